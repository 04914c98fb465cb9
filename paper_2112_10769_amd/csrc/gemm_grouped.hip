// 4-bit products grouped by expert: the tile kernel of gemm_kernel.hpp on ragged groups
// whose sizes only the device knows.
//
//   rows  (forward, activation gradient)  C[m][n] = s * s_w[e] * sum_k A[m][k] B_e[n][k],
//         m in group e: every group is a product of its own, of M_e = offsets[e + 1] -
//         offsets[e] rows.
//   depth (weight gradient)  C_e[m][n] = s * sum_k A[m][k] B[n][k], k in group e.
//
// The grid covers the most tiles that T rows in so many groups can make; a workgroup finds
// its group from the offsets and leaves if there is none for it.
//
// Rows: bound by the tile kernel (8192 rows of 8 experts, 4096 -> 16384: 513 us, 2.14 POPS)
// or by the weights' codes (16 rows of 16 experts, 4096 -> 4096: 20 us, 4.2 TB/s).  Depth:
// short reductions are bound by the output (16 experts, 1024 -> 4096 over 16384 rows: 107 us,
// 268 MB written).
#include "grouped_plan.hpp"

namespace luq {

namespace {

// ---- groups of rows --------------------------------------------------------------------

struct RowsArgs {
  const uint8_t* A;
  const uint8_t* B;
  const int32_t* offsets;
  int experts, tiles_n, vec, scales;
  int64_t T, N, K;
  int64_t w_row, w_expert;   // bytes
  const float* alpha;
  const float* bscale;
  float* C;
};

// One tile as the tile kernel sees it, moved to the origin: M rows of A from A, N rows of
// B from B.
struct RowsTile {
  static constexpr bool kMaskK = false, kStream = false;
  const uint8_t* A;
  const uint8_t* B;
  int64_t a_plane, M, N, K, ldb, ldc;
  int rows_a, rows_b;        // rows inside the tile
  const float* alpha;
  const float* bscale;
  float* C;
  int vec;
  __device__ __forceinline__ void place(int, int, int64_t& m0, int64_t& n0, int64_t& kbeg, int64_t& kend) const {
    m0 = n0 = kbeg = 0;
    kend = K;
  }
  __device__ __forceinline__ int64_t row_a(bool i8) const { return i8 ? K : K >> 1; }
  __device__ __forceinline__ int64_t row_b() const { return ldb; }
  __device__ __forceinline__ int range_a(int64_t row) const { return (int)(rows_a * row); }
  // the last row ends where its codes do
  __device__ __forceinline__ int range_b(int64_t row) const { return (int)((rows_b - 1) * row + (K >> 1)); }
  __device__ __forceinline__ bool sums() const { return false; }
  __device__ __forceinline__ uint32_t* out() const { return reinterpret_cast<uint32_t*>(C); }
  __device__ __forceinline__ int64_t row_c() const { return ldc; }
};

// Rows of group e (e = experts: the rows after the last group), kept inside the batch
// whatever the offsets hold.
__device__ __forceinline__ void group_bounds(const int32_t* offsets, int experts, int T, int e, int& lo, int& hi) {
  lo = min(max(offsets[e], 0), T);
  hi = e < experts ? min(max(offsets[e + 1], lo), T) : T;
}

struct GroupTile {
  int group, lo, rows, tm, tn;   // the group, its first row and number of rows, the tile in it
};

// Tile of workgroup bid: tiles are numbered group by group, and within a group in columns
// of 8 tile-rows; each of the 8 XCDs takes a run of them, as in tile_coords.  Every wave
// scans the offsets for itself, 64 groups at a time, twice (512 -> 512, 16 rows: 64
// experts 7 us, 4096 36, the difference the scans; 8192 rows: 10.4 and 1960, in 33 rounds of
// workgroups).  False: no tile is left for bid.
__device__ __forceinline__ bool find_tile(const int32_t* offsets, int experts, int T, int bm, int tiles_n, int bid,
                                          GroupTile& g) {
  const int lane = threadIdx.x & 63;
  auto tiles_of = [&](int e, int& lo, int& rows) -> uint32_t {   // at most 2^25
    int hi = 0;
    lo = rows = 0;
    if (e <= experts) {
      group_bounds(offsets, experts, T, e, lo, hi);
      rows = hi - lo;
    }
    return (uint32_t)((rows + bm - 1) / bm);
  };
  // offsets that decrease can ask for more tiles than the grid has: those are left out
  int64_t rows_total = 0;
  for (int base = 0; base <= experts; base += 64) {
    int lo, rows;
    uint32_t n = tiles_of(base + lane, lo, rows);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) n += (uint32_t)__shfl_xor((int)n, d, 64);
    rows_total += (uint32_t)__builtin_amdgcn_readfirstlane((int)n);
  }
  const int total = (int)min(rows_total * tiles_n, (int64_t)gridDim.x);
  if (bid >= total) return false;
  const int xcd = bid & 7, q = total >> 3, r = total & 7;
  int L = xcd * q + min(xcd, r) + (bid >> 3);
  uint32_t before = 0;   // tile-rows of the groups before
  const uint32_t row = (uint32_t)(L / tiles_n);
  for (int base = 0; base <= experts; base += 64) {
    int lo, rows;
    const uint32_t n = tiles_of(base + lane, lo, rows);
    uint32_t sum = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t up = (uint32_t)__shfl_up((int)sum, d, 64);
      if (lane >= d) sum += up;
    }
    const uint64_t past = __ballot(before + sum > row);
    if (past) {
      const int at = __builtin_ctzll(past);
      g.group = base + at;
      g.lo = __builtin_amdgcn_readlane(lo, at);
      g.rows = __builtin_amdgcn_readlane(rows, at);
      const int ntm = __builtin_amdgcn_readlane((int)n, at);
      L -= ((int)before + __builtin_amdgcn_readlane((int)sum, at) - ntm) * tiles_n;
      constexpr int G = 8;
      const int first = (L / (G * tiles_n)) * G, size = min(ntm - first, G);
      const int in = L - first * tiles_n;
      g.tm = first + in % size;
      g.tn = in / size;
      return true;
    }
    before += (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
  }
  return false;
}

template <int AC, bool BSIGNED, bool FULLK, int PF, typename S>
__global__ __launch_bounds__(S::THREADS, S::OCC) void grouped_rows_kernel(RowsArgs a) {
  GroupTile g;
  if (!find_tile(a.offsets, a.experts, (int)a.T, S::BM, a.tiles_n, blockIdx.x, g)) return;
  const int64_t m0 = (int64_t)g.lo + (int64_t)g.tm * S::BM, n0 = (int64_t)g.tn * S::BN;
  const int64_t m = g.rows - (int64_t)g.tm * S::BM, n = a.N - n0;
  float* const C = a.C + m0 * a.N + n0;
  if (g.group == a.experts) {   // rows of no group
    const int rows = (int)min(m, (int64_t)S::BM), cols = (int)min(n, (int64_t)S::BN);
    for (int r = threadIdx.x / 64; r < rows; r += S::NW)
      for (int c = threadIdx.x & 63; c < cols; c += 64) C[r * a.N + c] = 0.0f;
    return;
  }
  RowsTile t;
  t.A = a.A + m0 * (AC == kAcSum2 ? a.K : a.K >> 1);
  t.B = a.B + g.group * a.w_expert + n0 * a.w_row;
  t.a_plane = 0;
  t.M = m;
  t.N = n;
  t.K = a.K;
  t.ldb = a.w_row;
  t.ldc = a.N;
  t.rows_a = (int)min(m, (int64_t)S::BM);
  t.rows_b = (int)min(n, (int64_t)S::BN);
  t.alpha = a.alpha;
  t.bscale = a.bscale + (a.scales == 1 ? 0 : g.group);
  t.C = C;
  t.vec = a.vec;
  gemm_tile<AC, 1, BSIGNED, FULLK, PF, S>(t);
}

// ---- groups of the reduction -------------------------------------------------------------

struct DepthArgs {
  const uint8_t* A;
  const uint8_t* B;
  const int32_t* offsets;
  int experts, tiles_m, tiles_n, splits, vec;
  int64_t T, M, N;
  const float* alpha;
  const float* bscale;
  float* C;
  int32_t* partial;   // [splits][experts][M][N], or null
};

// A group's k range is read from a multiple of 128 codes on (64 bytes; 128 of the int8 sums),
// as the stages of an ungrouped product are: the codes before the group are cleared.
constexpr int kDepthAlign = 128;

// STREAM: the gradient is next read by the optimizer, after the rest of the backward pass, and
// goes around the caches (16 experts, 1024 -> 4096, 16384 rows: 128 -> 117 us; 512 -> 1024
// over 8192 rows 19.0 -> 16.9) where its rows are whole 128-byte lines: parts of a line must
// meet in L2 (17 experts, 2744 -> 3648 over 96 rows: 251 us streamed, 152 not).  The rows'
// products are read by a quantizer next and stay in the caches (2048 x 4096: streamed, 23.4 ->
// 21.5 us alone, but 40.2 -> 40.6 with the quantizer).
template <bool STREAM>
struct DepthTile {
  static constexpr bool kMaskK = true, kStream = STREAM;
  const uint8_t* A;
  const uint8_t* B;
  int64_t a_plane, M, N, T, klo, kend;
  int64_t ldc;
  int rows_a, rows_b;
  const float* alpha;
  const float* bscale;
  uint32_t* C;
  int vec;
  bool part;
  __device__ __forceinline__ void place(int, int, int64_t& m0, int64_t& n0, int64_t& kb, int64_t& ke) const {
    m0 = n0 = 0;
    kb = klo & ~(int64_t)(kDepthAlign - 1);
    ke = kend;
  }
  __device__ __forceinline__ int64_t row_a(bool i8) const { return i8 ? T : T >> 1; }
  __device__ __forceinline__ int64_t row_b() const { return T >> 1; }
  __device__ __forceinline__ int range_a(int64_t row) const { return (int)(rows_a * row); }
  __device__ __forceinline__ int range_b(int64_t row) const { return (int)(rows_b * row); }
  __device__ __forceinline__ bool sums() const { return part; }
  __device__ __forceinline__ uint32_t* out() const { return C; }
  __device__ __forceinline__ int64_t row_c() const { return ldc; }
};

template <int AC, bool BSIGNED, int PF, typename S, bool STREAM>
__global__ __launch_bounds__(S::THREADS, S::OCC) void grouped_depth_kernel(DepthArgs a) {
  // Groups differ in length, so each of the 8 XCDs takes an eighth of every group's tiles (a
  // run of whole groups for each left XCDs waiting for the one with the longest)
  const int per = a.tiles_m * a.tiles_n, share = (per + 7) / 8;
  const int xcd = blockIdx.x & 7, at = (int)(blockIdx.x >> 3), e = at / share;
  const int L = xcd * share + at - e * share;
  if (L >= per) return;
  constexpr int G = 8;
  const int first = (L / (G * a.tiles_n)) * G, size = min(a.tiles_m - first, G);
  const int in = L - first * a.tiles_n;
  const int64_t m0 = (int64_t)(first + in % size) * S::BM, n0 = (int64_t)(in / size) * S::BN;
  int lo, hi;
  group_bounds(a.offsets, a.experts, (int)a.T, e, lo, hi);
  if (a.splits > 1) {   // whole stages a split, at most kMaxExactK
    const int kb = lo & ~(kDepthAlign - 1), stages = (hi - kb + S::BK - 1) / S::BK;
    const int chunk = (stages + a.splits - 1) / a.splits * S::BK;
    const int from = kb + (int)blockIdx.y * chunk;
    hi = min(hi, from + chunk);
    lo = min(max(lo, from), hi);
  }
  DepthTile<STREAM> t;
  t.A = a.A + m0 * (AC == kAcSum2 ? a.T : a.T >> 1);
  t.B = a.B + n0 * (a.T >> 1);
  t.a_plane = 0;
  t.M = a.M - m0;
  t.N = a.N - n0;
  t.T = a.T;
  t.klo = lo;
  t.kend = hi;
  t.ldc = a.N;
  t.rows_a = (int)min(t.M, (int64_t)S::BM);
  t.rows_b = (int)min(t.N, (int64_t)S::BN);
  t.alpha = a.alpha;
  t.bscale = a.bscale;
  t.vec = a.vec;
  t.part = a.partial != nullptr;
  const int64_t slab = ((int64_t)blockIdx.y * a.experts + e) * a.M * a.N + m0 * a.N + n0;
  t.C = t.part ? reinterpret_cast<uint32_t*>(a.partial + slab) : reinterpret_cast<uint32_t*>(a.C + slab);
  gemm_tile<AC, 1, BSIGNED, true, PF, S>(t);
}

// ---- launch ------------------------------------------------------------------------------

template <typename S, int AC, bool BSIGNED>
void launch_rows_tile(RowsArgs a, GemmTile tile, hipStream_t st) {
  a.tiles_n = (int)((a.N + S::BN - 1) / S::BN);
  const dim3 grid((unsigned)rows_grid(tile, a.T, a.N, a.experts));
  if (a.K % S::BK == 0)
    hipLaunchKernelGGL((grouped_rows_kernel<AC, BSIGNED, true, prefetch_depth<S, AC, 1, BSIGNED, true>(), S>), grid, dim3(S::THREADS), 0, st, a);
  else
    hipLaunchKernelGGL((grouped_rows_kernel<AC, BSIGNED, false, prefetch_depth<S, AC, 1, BSIGNED, false>(), S>), grid, dim3(S::THREADS), 0, st, a);
}

template <int AC, bool BSIGNED>
hipError_t launch_rows(const RowsArgs& a, hipStream_t st) {
  const GemmTile tile = plan_rows(a.T, a.N, a.K, a.experts);
  switch (tile) {
    case kTile256x256: launch_rows_tile<Tile256x256, AC, BSIGNED>(a, tile, st); break;
    case kTile128x128: launch_rows_tile<Tile128x128, AC, BSIGNED>(a, tile, st); break;
    case kTile64x128: launch_rows_tile<Tile64x128, AC, BSIGNED>(a, tile, st); break;
    case kTile32x64: launch_rows_tile<Tile32x64, AC, BSIGNED>(a, tile, st); break;
    case kTile32x32: launch_rows_tile<Tile32x32, AC, BSIGNED>(a, tile, st); break;
    default: launch_rows_tile<Tile64x64k1, AC, BSIGNED>(a, tile, st); break;
  }
  return hipGetLastError();
}

template <typename S, int AC, bool BSIGNED>
void launch_depth_tile(DepthArgs a, GemmTile tile, hipStream_t st) {
  a.tiles_m = (int)((a.M + S::BM - 1) / S::BM);
  a.tiles_n = (int)((a.N + S::BN - 1) / S::BN);
  const dim3 grid((unsigned)depth_grid(tile, a.M, a.N, a.experts), (unsigned)a.splits);
  constexpr int kPf = prefetch_depth<S, AC, 1, BSIGNED, true>();
  if (!a.partial && a.N % 32 == 0 && ((uintptr_t)a.C & 127) == 0)
    hipLaunchKernelGGL((grouped_depth_kernel<AC, BSIGNED, kPf, S, true>), grid, dim3(S::THREADS), 0, st, a);
  else
    hipLaunchKernelGGL((grouped_depth_kernel<AC, BSIGNED, kPf, S, false>), grid, dim3(S::THREADS), 0, st, a);
}

template <int AC, bool BSIGNED>
hipError_t launch_depth(DepthArgs a, GemmTile tile, hipStream_t st) {
  a.vec = (a.N % 4) == 0 && (((uintptr_t)(a.partial ? (void*)a.partial : (void*)a.C)) & 15) == 0;
  switch (tile) {
    case kTile256x256: launch_depth_tile<Tile256x256, AC, BSIGNED>(a, tile, st); break;
    case kTile128x256: launch_depth_tile<Tile128x256, AC, BSIGNED>(a, tile, st); break;
    case kTile128x128: launch_depth_tile<Tile128x128, AC, BSIGNED>(a, tile, st); break;
    case kTile64x128: launch_depth_tile<Tile64x128, AC, BSIGNED>(a, tile, st); break;
    case kTile32x64: launch_depth_tile<Tile32x64, AC, BSIGNED>(a, tile, st); break;
    default: launch_depth_tile<Tile64x64k1, AC, BSIGNED>(a, tile, st); break;
  }
  if (a.splits > 1)
    launch_split_reduce(a.partial, a.splits, a.experts * a.M * a.N,
                        EpilogueScale<AC, 1, BSIGNED>{a.alpha, a.bscale}, a.C, st);
  return hipGetLastError();
}

}  // namespace

// fp32 outputs of 256 GiB; the largest tile has the fewest workgroups.
static constexpr int64_t kMostOutputs = (int64_t)1 << 36;

hipError_t launch_grouped_rows(GroupedA kind, const uint8_t* A, const float* alpha, const uint8_t* B, int64_t w_row,
                               int64_t w_expert, const float* bscale, int64_t scales, int b_signed,
                               const int32_t* offsets, int64_t experts, int64_t T, int64_t N, int64_t K, float* C,
                               hipStream_t st) {
  RowsArgs a;
  a.A = A;
  a.B = B;
  a.offsets = offsets;
  a.experts = (int)experts;
  a.tiles_n = 0;
  a.vec = (N % 4) == 0 && ((uintptr_t)C & 15) == 0;
  a.scales = (int)scales;
  a.T = T;
  a.N = N;
  a.K = K;
  a.w_row = w_row / 2;
  a.w_expert = w_expert / 2;
  a.alpha = alpha;
  a.bscale = bscale;
  a.C = C;
  switch (kind) {
    case GroupedA::kLuq: return b_signed ? launch_rows<kAcLuq, true>(a, st) : launch_rows<kAcLuq, false>(a, st);
    case GroupedA::kSums: return b_signed ? launch_rows<kAcSum2, true>(a, st) : launch_rows<kAcSum2, false>(a, st);
    case GroupedA::kInt4S: return b_signed ? launch_rows<kAcInt4S, true>(a, st) : launch_rows<kAcInt4S, false>(a, st);
    default: return b_signed ? launch_rows<kAcInt4U, true>(a, st) : launch_rows<kAcInt4U, false>(a, st);
  }
}

bool grouped_rows_fit(int64_t T, int64_t N, int64_t experts) {
  return T * N <= kMostOutputs && rows_grid(kTile256x256, T, N, experts) < kMostWorkgroups;
}

bool grouped_depth_fits(int64_t T, int64_t M, int64_t N, int64_t experts) {
  const int64_t outputs = experts * M * N;
  if (outputs > kMostOutputs || depth_grid(kTile256x256, M, N, experts) >= kMostWorkgroups) return false;
  if (T <= kMaxExactK) return true;
  // the launch that adds the splits takes 4 outputs a thread of whole groups of 4, or one
  return T <= kMostDepth && T % kDepthAlign == 0 && outputs < (int64_t)1 << (outputs % 4 == 0 ? 34 : 32);
}

size_t grouped_depth_workspace_bytes(int64_t T, int64_t M, int64_t N, int64_t experts) {
  const int splits = plan_depth(T, M, N, experts).splits;
  return splits > 1 ? (size_t)splits * experts * M * N * sizeof(int32_t) : 0;
}

hipError_t launch_grouped_depth(GroupedA kind, const uint8_t* A, const float* alpha, const uint8_t* B,
                                const float* bscale, int b_signed, const int32_t* offsets, int64_t experts, int64_t T,
                                int64_t M, int64_t N, float* C, void* ws, hipStream_t st) {
  DepthArgs a;
  a.A = A;
  a.B = B;
  a.offsets = offsets;
  a.experts = (int)experts;
  a.tiles_m = a.tiles_n = a.vec = 0;
  const DepthPlan p = plan_depth(T, M, N, experts);
  a.splits = p.splits;
  a.T = T;
  a.M = M;
  a.N = N;
  a.alpha = alpha;
  a.bscale = bscale;
  a.C = C;
  a.partial = a.splits > 1 ? static_cast<int32_t*>(ws) : nullptr;
  if (kind == GroupedA::kSums)
    return b_signed ? launch_depth<kAcSum2, true>(a, p.tile, st) : launch_depth<kAcSum2, false>(a, p.tile, st);
  return b_signed ? launch_depth<kAcLuq, true>(a, p.tile, st) : launch_depth<kAcLuq, false>(a, p.tile, st);
}

}  // namespace luq
