// Softmax cross entropy of the last layer, the logits not kept, and its gradients.
//
//   z_tv = scale x_t . W_v,  lse_t = log sum_v exp z_tv
//   loss_t = lse_t - (1 - eps) z_t,target - eps / V sum_v z_tv
//   g_tv = dloss_t scale (exp(z_tv - lse_t) - (1 - eps) [v = target] - eps / V),  dx = g W,  dW = g^T x
//
// Forward: a tile of products leaves each row's maximum, sum of exponentials and sum of logits over
// its columns; a second launch joins them.  Backward: a piece of the vocabulary at a time, the
// products again, their gradient g in bf16 terms, and the two products with it, whose operands lie
// across the reduction: they are transposed on the way out of LDS (written a second time, transposed,
// g took 130 of 447 us for 4096 x 32000 of it, and the table's and x's transposes 50).
//
// A bf16 output takes g in one bf16 term, whose rounding is of the size of the output's own: 2.4e-3 of the
// norm off where the output's rounding alone leaves 1.7e-3; a second term would double the products with g
// and its writes.  An fp32 tensor in such a product is cut to two terms (16 bits: 2^-8 of the output's
// rounding).  An fp32 output takes three bf16 terms of g (4096 tokens on 32000 x 1024 bf16, fp32 gradient of the table:
// 4.5e-7 of its norm off in 1400 us for both gradients, with two terms 2.6e-6 in 1147; the exact g in an
// fp32 library product 1.1e-6).
#include "cross_entropy_plan.hpp"
#include "luq_launch.hpp"

namespace luq {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kMost = 3.40282347e38f;   // kMost: fp32's largest number

__device__ __forceinline__ int64_t target_of(const void* targets, int i64, int64_t t) {
  return i64 ? static_cast<const int64_t*>(targets)[t] : static_cast<const int32_t*>(targets)[t];
}

// Terms of v: bf16 numbers whose sum it is to 8 bits a term.  What is not finite has one term.
template <int N>
__device__ __forceinline__ void terms(float v, uint16_t (&h)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint16_t b = from_f32<uint16_t>(v);
    if ((b & 0x7FFF) == 0x7F80 && fabsf(v) < __builtin_inff()) b -= 1;   // not rounded up to infinity
    h[i] = b;
    const float rest = v - to_f32(b);
    v = fabsf(v) < __builtin_inff() ? rest : 0.0f;
  }
}

typedef uint32_t v4w __attribute__((ext_vector_type(4)));

// N terms of eight elements, 16 bytes a term.
template <int N>
__device__ __forceinline__ void terms8(const float (&v)[8], v4w (&w)[N]) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    uint16_t a[N], b[N];
    terms<N>(v[k], a);
    terms<N>(v[k + 1], b);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i][k / 2] = (uint32_t)a[i] | (uint32_t)b[i] << 16;
  }
}

// ---- operands laid out: terms of a matrix, its rows a multiple of eight long

struct PackArgs {
  const void* src;      // [rows][cols]
  int64_t rows, cols;
  const void* targets;  // rows whose target is not in [0, vocab) become 0, or NULL
  int i64;
  int64_t vocab;
  uint16_t* out;
  int64_t width, ld, plane;   // width: cols, up to a multiple of eight
  __device__ __forceinline__ bool kept(int64_t row) const {
    if (!targets) return true;
    const int64_t y = target_of(targets, i64, row);
    return y >= 0 && y < vocab;
  }
};

template <typename T, int N>
__global__ __launch_bounds__(256) void pack_rows_kernel(PackArgs a) {
  const int64_t pieces = a.width / 8;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < a.rows * pieces; at += (int64_t)gridDim.x * 256) {
    const int64_t row = at / pieces, c = (at - row * pieces) * 8;
    float v[8];
    if (a.kept(row)) load_row<8>(static_cast<const T*>(a.src) + row * a.cols + c, a.cols - c, v);
    else
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    v4w w[N];
    terms8<N>(v, w);
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<v4w*>(a.out + i * a.plane + row * a.ld + c) = w[i];
  }
}

// ---- the products

// Where a lane's sums lie: row `row(i)` of the matrix, columns col(j, q) .. + 3 in registers 4q .. 4q + 3.
template <typename Tile>
struct Lane {
  int64_t row0, col0;
  __device__ __forceinline__ Lane(int64_t m0, int64_t n0) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    row0 = m0 + (wave / Tile::WN) * Tile::TM * 32 + (lane & 31);
    col0 = n0 + (wave % Tile::WN) * Tile::TN * 32 + 4 * (lane >> 5);
  }
  __device__ __forceinline__ int64_t row(int i) const { return row0 + i * 32; }
  __device__ __forceinline__ int64_t col(int j, int q) const { return col0 + j * 32 + 8 * q; }
};

struct LossArgs {
  const void* targets;
  int i64;
  int64_t T, V;
  float scale;
  int smoothed;    // whether the sum of logits is asked for
  float* part;     // [tiles of columns][3][T]: maximum, sum of exponentials (over its own), sum of logits
  float* at_target;
};

// Parts of a row joined, one after the other.  The maximum is a logit as it is rounded for the target too, and
// its exponential is 1: the sum is no less than 1, and a loss without smoothing no less than 0.
struct RowSum {
  float top = -kMost, sum = 0.0f, all = 0.0f;
  __device__ __forceinline__ void add(float m, float s, float z) {
    const float next = fmaxf(top, m);
    sum = sum * __builtin_amdgcn_exp2f((top - next) * kLog2e) + s * __builtin_amdgcn_exp2f((m - next) * kLog2e);
    top = next;
    all += z;
  }
};

template <typename Tile>
__global__ __launch_bounds__(Tile::kThreads) void loss_tile_kernel(Bf16Product g, LossArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[Tile::kLds];
  int tm, tn;
  bf16_tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * Tile::BM, n0 = (int64_t)tn * Tile::BN;
  Tile tile;
  tile.template run<false, false>(g, m0, n0, 0, g.pairs.count * (int)((g.K + Tile::BK - 1) / Tile::BK), lds);
  const Lane<Tile> at(m0, n0);
  const float c = a.scale * kLog2e;
  const int half = (threadIdx.x & 63) >> 5;
  const int64_t cols0 = at.col0 - 4 * half;   // of the wave
  if (n0 + Tile::BN > a.V) {
    // columns beyond the table: nothing, whatever the sign of the scale
    const float none = c < 0.0f ? __builtin_inff() : -__builtin_inff();
#pragma unroll
    for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
      for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (at.col(j, e / 4) + e % 4 >= a.V) tile.acc[i][j][e] = none;
  }
  // a row's sums of each wave, joined at the end: [3][waves][rows of the tile]
  float* const red = reinterpret_cast<float*>(lds) + (threadIdx.x >> 6) % Tile::WN * Tile::BM;
  constexpr int kNext = Tile::WN * Tile::BM;
#pragma unroll
  for (int i = 0; i < Tile::TM; ++i) {
    const int64_t row = at.row(i);
    const int64_t y = row < a.T ? target_of(a.targets, a.i64, row) : -1;
    float all = 0.0f;
    if (a.smoothed) {
#pragma unroll
      for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) all += at.col(j, e / 4) + e % 4 < a.V ? tile.acc[i][j][e] : 0.0f;
      all += __shfl_xor(all, 32, kWave);
    }
    const int mine = y >= cols0 && y < cols0 + Tile::TN * 32 ? (int)(y - cols0) - 4 * half : -8;
    if (__ballot(mine != -8)) {   // a target among the wave's columns
#pragma unroll
      for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (mine == j * 32 + 8 * (e / 4) + e % 4) a.at_target[row] = tile.acc[i][j][e] * a.scale;
    }
    float top = tile.acc[i][0][0];
    if (c < 0.0f) {
#pragma unroll
      for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fminf(top, tile.acc[i][j][e]);
    } else {
#pragma unroll
      for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, tile.acc[i][j][e]);
    }
    const float other = __shfl_xor(top, 32, kWave);
    top = c < 0.0f ? fminf(fminf(top, other), kMost) : fmaxf(fmaxf(top, other), -kMost);   // (columns beyond the table)
    float sum = 0.0f;
    // differences of products, before the scale: exact near the maximum, and 0 there, however large it is
#pragma unroll
    for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f((tile.acc[i][j][e] - top) * c);
    sum += __shfl_xor(sum, 32, kWave);
    if (half == 0) {
      float* const out = red + (row - m0);
      out[0] = top * a.scale;
      out[kNext] = sum;
      out[2 * kNext] = all * a.scale;
    }
  }
  __syncthreads();
  static_assert(Tile::BM <= Tile::kThreads, "a thread a row");
  const int64_t row = m0 + threadIdx.x;
  if (threadIdx.x >= Tile::BM || row >= a.T) return;
  const float* const in = reinterpret_cast<const float*>(lds) + threadIdx.x;
  RowSum r;
#pragma unroll
  for (int w = 0; w < Tile::WN; ++w) r.add(in[w * Tile::BM], in[kNext + w * Tile::BM], in[2 * kNext + w * Tile::BM]);
  float* const out = a.part + (int64_t)tn * 3 * a.T + row;
  out[0] = r.top;
  out[a.T] = r.sum;
  if (a.smoothed) out[2 * a.T] = r.all;
}

// (hipcc leaves the host's side of the tiles' kernels out unless asked for)
template __global__ void loss_tile_kernel<BigTile>(Bf16Product, LossArgs);
template __global__ void loss_tile_kernel<SmallTile>(Bf16Product, LossArgs);
template __global__ void loss_tile_kernel<DeepTile>(Bf16Product, LossArgs);
template __global__ void loss_tile_kernel<ThinTile>(Bf16Product, LossArgs);

// The outputs of a row from its sums.
struct LossOut {
  float smoothing;
  float* loss;
  float* lse;
  __device__ __forceinline__ void put(const LossArgs& a, int64_t row, const RowSum& r) const {
    const int64_t y = target_of(a.targets, a.i64, row);
    const bool kept = y >= 0 && y < a.V;
    const float rest = logf(r.sum);
    lse[row] = kept ? r.top + rest : 0.0f;
    // differences to the maximum first: the loss keeps its bits however far from 0 the logits are
    const float behind = kept ? r.top - a.at_target[row] : 0.0f;
    loss[row] = y < 0              ? 0.0f
                : !kept            ? __builtin_nanf("")
                : smoothing > 0.0f ? rest + (1.0f - smoothing) * behind + smoothing * (r.top - r.all / (float)a.V)
                                   : rest + behind;
  }
};

// The rows' parts joined: 64 rows a workgroup, its 16 waves every 16th part.
__global__ __launch_bounds__(1024) void loss_join_kernel(LossArgs a, int64_t parts, LossOut out) {
  __shared__ float red[3][16][kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * kWave + lane;
  RowSum r;
  if (row < a.T) {
    constexpr int U = 4;
    for (int64_t p = wave; p < parts; p += 16 * U) {
      float m[U], s[U], z[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t q = p + 16 * u;
        const float* const src = a.part + (q < parts ? q : p) * 3 * a.T + row;
        m[u] = q < parts ? src[0] : -kMost;
        s[u] = q < parts ? src[a.T] : 0.0f;
        z[u] = a.smoothed && q < parts ? src[2 * a.T] : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) r.add(m[u], s[u], z[u]);
    }
  }
  red[0][wave][lane] = r.top;
  red[1][wave][lane] = r.sum;
  red[2][wave][lane] = r.all;
  __syncthreads();
  if (wave != 0 || row >= a.T) return;
  RowSum all;
  for (int w = 0; w < 16; ++w) all.add(red[0][w][lane], red[1][w][lane], red[2][w][lane]);
  out.put(a, row, all);
}

// The same for few rows: a workgroup a row (the loss of 128 rows on 50021 x 1024: 30.3 us, 33.4 with 64
// rows a workgroup; of 256 rows 40 with either: the parts are read four bytes at a time here).
__global__ __launch_bounds__(1024) void loss_join_few_kernel(LossArgs a, int64_t parts, LossOut out) {
  __shared__ float red[3][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x;
  RowSum r;
  for (int64_t p = threadIdx.x; p < parts; p += 1024) {
    const float* const src = a.part + p * 3 * a.T + row;
    r.add(src[0], src[a.T], a.smoothed ? src[2 * a.T] : 0.0f);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    const float m = __shfl_xor(r.top, d, kWave), s = __shfl_xor(r.sum, d, kWave), z = __shfl_xor(r.all, d, kWave);
    r.add(m, s, z);
  }
  if (lane == 0) {
    red[0][wave] = r.top;
    red[1][wave] = r.sum;
    red[2][wave] = r.all;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  RowSum all;
  for (int w = 0; w < 16; ++w) all.add(red[0][w], red[1][w], red[2][w]);
  out.put(a, row, all);
}
constexpr int64_t kFewRows = 128;

// ---- backward

// A slab of a wave's sums in LDS: 32 rows of its columns in fp32, read in pieces of eight along the rows.
template <typename Tile>
struct Slab {
  static constexpr int kCols = Tile::TN * 32, kPitch = kCols + 4, kItems = 32 * kCols / 8 / 64;
  static_assert((size_t)Tile::WM * Tile::WN * 32 * kPitch * 4 <= (size_t)Tile::kLds, "slabs fit in the stages' place");
  float* e;
  __device__ __forceinline__ explicit Slab(uint8_t* lds) {
    e = reinterpret_cast<float*>(lds) + (threadIdx.x >> 6) * 32 * kPitch;
  }
  __device__ __forceinline__ void put(int j, int q, const float (&v)[4]) {
    const int lane = threadIdx.x & 63;
    typedef float f4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<f4*>(e + (lane & 31) * kPitch + j * 32 + 8 * q + 4 * (lane >> 5)) = f4{v[0], v[1], v[2], v[3]};
  }
  __device__ __forceinline__ void row8(int row, int c, float (&v)[8]) const { load_pack(e + row * kPitch + c, v); }
};

// The same in bf16.
template <typename Tile>
struct HalfSlab {
  static constexpr int kCols = Tile::TN * 32, kPitch = kCols * 2 + 8, kItems = 32 * kCols / 8 / 64;
  static_assert((size_t)Tile::WM * Tile::WN * 32 * kPitch <= (size_t)Tile::kLds, "slabs fit in the stages' place");
  typedef uint32_t v2w __attribute__((ext_vector_type(2)));
  uint8_t* e;
  int lane;
  __device__ __forceinline__ explicit HalfSlab(uint8_t* lds) : lane(threadIdx.x & 63) {
    e = lds + (threadIdx.x >> 6) * 32 * kPitch;
  }
  // the lane's four columns of its row, and what rounding to bf16 leaves of them
  __device__ __forceinline__ void put(int j, int q, float* v) const {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    v2w w;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[2 * k], v[2 * k + 1]}, bf2));
      v[2 * k] -= __uint_as_float(w[k] << 16);
      v[2 * k + 1] -= __uint_as_float(w[k] & 0xFFFF0000u);
    }
    *reinterpret_cast<v2w*>(e + (lane & 31) * kPitch + (j * 32 + 8 * q + 4 * (lane >> 5)) * 2) = w;
  }
  __device__ __forceinline__ v4w row8(int row, int c) const {
    const v2w* const p = reinterpret_cast<const v2w*>(e + row * kPitch + c * 2);
    const v2w a = p[0], b = p[1];
    return v4w{a[0], a[1], b[0], b[1]};
  }
};

struct GradArgs {
  const void* targets;
  int i64;
  int64_t T, V;        // V: of the whole table
  int64_t v0, cols;    // the piece: its first row of the table, and how many
  float scale, smoothing;
  const float* dloss;
  const float* lse;
  uint16_t* g;         // [terms][T][ld]: columns up to the next multiple of eight are written
  int64_t ld, plane;
  int terms;
};

template <typename Tile>
__global__ __launch_bounds__(Tile::kThreads) void grad_tile_kernel(Bf16Product g, GradArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[Tile::kLds];
  int tm, tn;
  bf16_tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * Tile::BM, n0 = (int64_t)tn * Tile::BN;
  Tile tile;
  tile.template run<false, false>(g, m0, n0, 0, g.pairs.count * (int)((g.K + Tile::BK - 1) / Tile::BK), lds);
  const Lane<Tile> at(m0, n0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t rows0 = m0 + (wave / Tile::WN) * Tile::TM * 32, cols0 = n0 + (wave % Tile::WN) * Slab<Tile>::kCols;
  const float each = a.smoothing / (float)a.V;
  const bool whole = n0 + Tile::BN <= a.cols;
  const HalfSlab<Tile> slab(lds);
#pragma unroll
  for (int i = 0; i < Tile::TM; ++i) {
    const int64_t row = at.row(i);
    const int64_t y = row < a.T ? target_of(a.targets, a.i64, row) : -1;
    const bool kept = y >= 0 && y < a.V;
    const float up = kept ? a.dloss[row] * a.scale : 0.0f, base = kept ? a.lse[row] : 0.0f;
    const bool any_out = !whole || __ballot(!kept);
    const int64_t rel = y - a.v0 - cols0;
    const int mine = kept && rel >= 0 && rel < HalfSlab<Tile>::kCols ? (int)rel - 4 * (lane >> 5) : -8;
    const bool any_target = __ballot(mine != -8);
    float v[Tile::TN][16];
#pragma unroll
    for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {   // the difference first: near the maximum it is exact
        v[j][e] = __builtin_amdgcn_exp2f(fmaf(tile.acc[i][j][e], a.scale, -base) * kLog2e) - each;
        if (any_target && mine == j * 32 + 8 * (e / 4) + e % 4) v[j][e] -= 1.0f - a.smoothing;
        v[j][e] *= up;
        if (any_out) v[j][e] = kept && at.col(j, e / 4) + e % 4 < a.cols ? v[j][e] : 0.0f;   // whatever the row holds
      }
    for (int n = 0; n < a.terms; ++n) {
#pragma unroll
      for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) slab.put(j, q, &v[j][4 * q]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int u = 0; u < HalfSlab<Tile>::kItems; ++u) {
        const int item = lane + u * 64, r = item / (HalfSlab<Tile>::kCols / 8), c = item % (HalfSlab<Tile>::kCols / 8) * 8;
        const int64_t gr = rows0 + i * 32 + r, gc = cols0 + c;
        if (gr < a.T && gc < a.cols) *reinterpret_cast<v4w*>(a.g + n * a.plane + gr * a.ld + gc) = slab.row8(r, c);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

template __global__ void grad_tile_kernel<BigTile>(Bf16Product, GradArgs);
template __global__ void grad_tile_kernel<SmallTile>(Bf16Product, GradArgs);
template __global__ void grad_tile_kernel<DeepTile>(Bf16Product, GradArgs);
template __global__ void grad_tile_kernel<ThinTile>(Bf16Product, GradArgs);

// Where a product's sums go: partial sums (fp32, one matrix a split, added to when `add`), or an
// output of type fp32 or bf16, added to when `add`; `before` (fp32) is added too.
struct OutArgs {
  int64_t M, N;
  float* part;
  void* out;
  int bf16, add;
  const float* before;   // what earlier pieces left, added to the sums, or NULL
  const void* targets;   // rows whose target is not in [0, vocab) become 0, or NULL
  int i64;
  int64_t vocab;
  int chunk;             // stages of a split
  __device__ __forceinline__ bool kept(int64_t row) const {
    if (!targets) return true;
    const int64_t y = target_of(targets, i64, row);
    return y >= 0 && y < vocab;
  }
  template <typename T>
  __device__ __forceinline__ void put(int64_t row, int64_t col, float (&v)[8]) const {
    T* const p = static_cast<T*>(out) + row * N + col;
    if (add) {
      float old[8];
      load_row<8>(p, N - col, old);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += old[k];
    }
    if (!kept(row))
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    store_row<8>(p, N - col, v);
  }
};

// CA: A lies across the reduction (g^T); B does in both products.
template <typename Tile, bool CA>
__global__ __launch_bounds__(Tile::kThreads) void out_tile_kernel(Bf16Product g, OutArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[Tile::kLds];
  int tm, tn;
  bf16_tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * Tile::BM, n0 = (int64_t)tn * Tile::BN;
  const int stages = g.pairs.count * (int)((g.K + Tile::BK - 1) / Tile::BK);
  const int beg = blockIdx.y * a.chunk, end = min(beg + a.chunk, stages);
  Tile tile;
  tile.template run<CA, true>(g, m0, n0, beg, end, lds);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t rows0 = m0 + (wave / Tile::WN) * Tile::TM * 32, cols0 = n0 + (wave % Tile::WN) * Slab<Tile>::kCols;
  Slab<Tile> slab(lds);
#pragma unroll
  for (int i = 0; i < Tile::TM; ++i) {
#pragma unroll
    for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float v[4] = {tile.acc[i][j][4 * q], tile.acc[i][j][4 * q + 1], tile.acc[i][j][4 * q + 2], tile.acc[i][j][4 * q + 3]};
        slab.put(j, q, v);
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the other lanes' parts of the slab
#pragma unroll
    for (int u = 0; u < Slab<Tile>::kItems; ++u) {
      const int item = lane + u * 64, r = item / (Slab<Tile>::kCols / 8), c = item % (Slab<Tile>::kCols / 8) * 8;
      const int64_t row = rows0 + i * 32 + r, col = cols0 + c;
      if (row >= a.M || col >= a.N) continue;
      float v[8];
      slab.row8(r, c, v);
      if (a.before) {
        float old[8];
        load_row<8>(a.before + row * a.N + col, a.N - col, old);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += old[k];
      }
      if (a.part) {
        float* const p = a.part + ((int64_t)blockIdx.y * a.M + row) * a.N + col;
        if (a.add) {
          float old[8];
          load_row<8>(p, a.N - col, old);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] += old[k];
        }
        store_row<8>(p, a.N - col, v);
      } else if (a.bf16) {
        a.put<uint16_t>(row, col, v);
      } else {
        a.put<float>(row, col, v);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // read before the next rows are put there
  }
}

template __global__ void out_tile_kernel<BigTile, false>(Bf16Product, OutArgs);
template __global__ void out_tile_kernel<SmallTile, false>(Bf16Product, OutArgs);
template __global__ void out_tile_kernel<DeepTile, false>(Bf16Product, OutArgs);
template __global__ void out_tile_kernel<DeepTile, true>(Bf16Product, OutArgs);
template __global__ void out_tile_kernel<BigTile, true>(Bf16Product, OutArgs);
template __global__ void out_tile_kernel<SmallTile, true>(Bf16Product, OutArgs);

// The splits' sums, in order, to the output.
__global__ __launch_bounds__(256) void out_join_kernel(OutArgs a, const float* __restrict__ part, int splits) {
  const int64_t pieces = (a.N + 7) / 8;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < a.M * pieces; at += (int64_t)gridDim.x * 256) {
    const int64_t row = at / pieces, col = (at - row * pieces) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int s = 0; s < splits; ++s) {
      float w[8];
      load_row<8>(part + ((int64_t)s * a.M + row) * a.N + col, a.N - col, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += w[k];
    }
    if (a.bf16) a.put<uint16_t>(row, col, v);
    else a.put<float>(row, col, v);
  }
}

// ---- host side

void pack_rows(const PackArgs& a, int bf16, hipStream_t st) {
  const int64_t need = ceil_div(a.rows * (a.width / 8), 256);
  const dim3 grid((unsigned)(need < 16384 ? need : 16384));
  if (bf16) hipLaunchKernelGGL((pack_rows_kernel<uint16_t, 1>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((pack_rows_kernel<float, 3>), grid, dim3(256), 0, st, a);
}

// The operands of the logits' product, laid out if need be.
Bf16Product logits_product(const CrossEntropyArgs& a, const Layout& l, bool back, uint8_t* ws, hipStream_t st) {
  Bf16Product g;
  g.A = {static_cast<const uint16_t*>(a.x), a.T, a.D, 0};
  g.B = {static_cast<const uint16_t*>(a.table), a.V, a.D, 0};
  if (l.pack_x) {
    uint16_t* const out = reinterpret_cast<uint16_t*>(ws + l.x_rows);
    pack_rows({a.x, a.T, a.D, back ? a.targets : nullptr, a.i64, a.V, out, l.D8, l.ld, a.T * l.ld}, a.x_bf16, st);
    g.A = {out, a.T, l.ld, a.T * l.ld};
  }
  if (l.pack_t) {
    uint16_t* const out = reinterpret_cast<uint16_t*>(ws + l.t_rows);
    pack_rows({a.table, a.V, a.D, nullptr, 0, 0, out, l.D8, l.ld, a.V * l.ld}, a.t_bf16, st);
    g.B = {out, a.V, l.ld, a.V * l.ld};
  }
  g.pairs = pairs_of(l.xn, l.tn);
  g.K = l.pack_x || l.pack_t ? l.D8 : a.D;
  return g;
}

void place(Bf16Product& g, int64_t M, int64_t N, Edge edge) {
  with_tile(edge, [&](auto tile) {
    g.tiles_m = (int)ceil_div(M, decltype(tile)::BM);
    g.tiles_n = (int)ceil_div(N, decltype(tile)::BN);
  });
}

template <typename Tile>
void loss_tiles(const Bf16Product& g, const LossArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((loss_tile_kernel<Tile>), dim3((unsigned)g.tiles_m * g.tiles_n), dim3(Tile::kThreads), 0, st, g, a);
}
template <typename Tile>
void grad_tiles(const Bf16Product& g, const GradArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((grad_tile_kernel<Tile>), dim3((unsigned)g.tiles_m * g.tiles_n), dim3(Tile::kThreads), 0, st, g, a);
}
template <typename Tile, bool CA>
void out_tiles(const Bf16Product& g, const OutArgs& a, int splits, hipStream_t st) {
  hipLaunchKernelGGL((out_tile_kernel<Tile, CA>), dim3((unsigned)g.tiles_m * g.tiles_n, splits), dim3(Tile::kThreads), 0, st, g, a);
}

template <bool CA>
void out_product(Bf16Product g, OutArgs o, Choice c, hipStream_t st) {
  place(g, o.M, o.N, c.edge);
  const int stages = g.pairs.count * (int)ceil_div(g.K, kStage);
  o.chunk = (int)ceil_div(stages, c.splits);
  if (c.edge == Edge::kBig) out_tiles<BigTile, CA>(g, o, c.splits, st);
  else if (c.edge == Edge::kDeep) out_tiles<DeepTile, CA>(g, o, c.splits, st);
  else out_tiles<SmallTile, CA>(g, o, c.splits, st);
}

void out_join(const OutArgs& o, const float* part, int splits, hipStream_t st) {
  const int64_t need = ceil_div(o.M * ceil_div(o.N, 8), 256);
  hipLaunchKernelGGL(out_join_kernel, dim3((unsigned)(need < 16384 ? need : 16384)), dim3(256), 0, st, o, part, splits);
}

template <typename T>
__global__ void zero_kernel(T* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) p[i] = 0;
}

}  // namespace

size_t cross_entropy_fwd_workspace_bytes(int64_t T, int64_t V, int64_t D, int x_bf16, int t_bf16) {
  Layout l(T, V, D, x_bf16, t_bf16, false);
  l.forward();
  return l.bytes;
}

size_t cross_entropy_bwd_workspace_bytes(int64_t T, int64_t V, int64_t D, int x_bf16, int t_bf16, int g_bf16) {
  Layout l(T, V, D, x_bf16, t_bf16, true);
  l.backward(x_bf16, g_bf16);
  return l.bytes;
}

hipError_t launch_cross_entropy_fwd(const CrossEntropyArgs& a, float* loss, float* lse, void* ws, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  Layout l(a.T, a.V, a.D, a.x_bf16, a.t_bf16, false);
  l.forward();
  uint8_t* const w = static_cast<uint8_t*>(ws);
  Bf16Product g = logits_product(a, l, false, w, st);
  place(g, a.T, a.V, l.z.edge);
  const LossArgs la{a.targets, a.i64, a.T, a.V, a.scale, a.smoothing > 0.0f, reinterpret_cast<float*>(w + l.part),
                    reinterpret_cast<float*>(w + l.at_target)};
  if (l.z.edge == Edge::kBig) loss_tiles<BigTile>(g, la, st);
  else if (l.z.edge == Edge::kSmall) loss_tiles<SmallTile>(g, la, st);
  else if (l.z.edge == Edge::kDeep) loss_tiles<DeepTile>(g, la, st);
  else loss_tiles<ThinTile>(g, la, st);
  const LossOut out{a.smoothing, loss, lse};
  if (a.T <= kFewRows) hipLaunchKernelGGL(loss_join_few_kernel, dim3((unsigned)a.T), dim3(1024), 0, st, la, l.parts, out);
  else hipLaunchKernelGGL(loss_join_kernel, dim3((unsigned)ceil_div(a.T, 64)), dim3(1024), 0, st, la, l.parts, out);
  return hipGetLastError();
}

hipError_t launch_cross_entropy_bwd(const CrossEntropyArgs& a, const float* dloss, const float* lse, int accumulate,
                                    void* dx, void* dtable, int g_bf16, void* ws, hipStream_t st) {
  if (a.T == 0) {
    if (accumulate) return hipSuccess;
    const int64_t n = a.V * a.D, need = ceil_div(n, 256);
    const dim3 grid((unsigned)(need < 16384 ? need : 16384));
    if (g_bf16) hipLaunchKernelGGL((zero_kernel<uint16_t>), grid, dim3(256), 0, st, static_cast<uint16_t*>(dtable), n);
    else hipLaunchKernelGGL((zero_kernel<float>), grid, dim3(256), 0, st, static_cast<float*>(dtable), n);
    return hipGetLastError();
  }
  Layout l(a.T, a.V, a.D, a.x_bf16, a.t_bf16, true);
  l.backward(a.x_bf16, g_bf16);
  uint8_t* const w = static_cast<uint8_t*>(ws);
  auto half = [&](size_t at) { return reinterpret_cast<uint16_t*>(w + at); };
  Bf16Product z = logits_product(a, l, true, w, st);
  const Bf16Planes table = z.B;
  for (int64_t p = 0; p < l.pieces; ++p) {
    const int64_t v0 = p * l.piece, cols = a.V - v0 < l.piece ? a.V - v0 : l.piece;
    // g of the piece
    z.B = {table.p + v0 * table.ld, cols, table.ld, table.plane};
    place(z, a.T, cols, l.z.edge);
    const GradArgs ga{a.targets, a.i64, a.T, a.V, v0, cols, a.scale, a.smoothing, dloss, lse, half(l.g), l.piece, a.T * l.piece, l.g_terms()};
    if (l.z.edge == Edge::kBig) grad_tiles<BigTile>(z, ga, st);
    else if (l.z.edge == Edge::kSmall) grad_tiles<SmallTile>(z, ga, st);
    else if (l.z.edge == Edge::kDeep) grad_tiles<DeepTile>(z, ga, st);
    else grad_tiles<ThinTile>(z, ga, st);
    const Bf16Planes grad{half(l.g), a.T, l.piece, a.T * l.piece};
    // dx += g W
    Bf16Product x;
    x.A = grad;
    x.B = z.B;
    x.pairs = pairs_of(l.g_x, l.tx);
    x.K = up8(cols);
    float* const sums = l.sums_x ? reinterpret_cast<float*>(w + l.sum_x) : nullptr;
    const bool last = p + 1 == l.pieces && l.by_x.splits == 1;   // writes dx itself
    OutArgs ox{a.T, a.D, last ? nullptr : sums, dx, a.x_bf16, last ? 0 : p > 0, last ? sums : nullptr, a.targets, a.i64, a.V, 0};
    out_product<false>(x, ox, l.by_x, st);
    // dW = g^T x
    Bf16Product t;
    t.A = grad;
    t.B = z.A;
    t.pairs = pairs_of(l.g_w, l.xt);
    t.K = a.T;
    uint8_t* const rows = static_cast<uint8_t*>(dtable) + (size_t)v0 * a.D * (g_bf16 ? 2 : 4);
    OutArgs ow{cols, a.D, nullptr, rows, g_bf16, accumulate, nullptr, nullptr, 0, 0, 0};
    if (l.by_w.splits > 1) {
      OutArgs part = ow;
      part.part = reinterpret_cast<float*>(w + l.sum_w);
      part.add = 0;
      out_product<true>(t, part, l.by_w, st);
      out_join(ow, part.part, l.by_w.splits, st);
    } else {
      out_product<true>(t, ow, l.by_w, st);
    }
  }
  if (l.by_x.splits > 1) {
    const OutArgs ox{a.T, a.D, nullptr, dx, a.x_bf16, 0, nullptr, a.targets, a.i64, a.V, 0};
    out_join(ox, reinterpret_cast<const float*>(w + l.sum_x), l.by_x.splits, st);
  }
  return hipGetLastError();
}

}  // namespace luq
