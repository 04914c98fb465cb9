// Embedding lookup with scaling, and the gradient of its table.
//
//   out[i] = scale * table[ids[i]]        dtable[v] = scale * sum over ids[i] = v of dout[i]
//
// Both are bound by memory: the lookup reads and writes a row per id (16384 rows of 1024
// bf16: 9.1 us, 4.9 TB/s), the gradient reads a row per id and writes the table once (65536
// rows of 1024 bf16 into 50021, on other buffers each call: 84 us, of them 74 the sums and the
// cleared rows, 4.7 TB/s; 50 with what the caches hold).  The gradient takes the positions grouped by id
// (group_ids.hip), so that every row of the table has one writer and its sum one order.
#include <algorithm>
#include <type_traits>

#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

// ---- lookup ------------------------------------------------------------------------------

// A row is taken by 2^log_lanes lanes of each block along y, kRows rows of a lane group in
// flight together.
template <typename ID, typename TT, typename OT, int kRows>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const ID* __restrict__ ids, int64_t n,
                                                            const TT* __restrict__ table, int64_t vocab, int64_t dim,
                                                            float scale, OT* __restrict__ out, int log_lanes) {
  constexpr int V = kPack<TT, OT>;
  const int lanes = 1 << log_lanes, groups = 256 >> log_lanes;
  const int64_t first = ((int64_t)blockIdx.x * groups + (threadIdx.x >> log_lanes)) * kRows;
  int64_t id[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) id[r] = first + r < n ? (int64_t)ids[first + r] : -1;
  const int64_t step = (int64_t)gridDim.y * lanes * V;
  for (int64_t c = ((int64_t)blockIdx.y * lanes + (threadIdx.x & (lanes - 1))) * V; c < dim; c += step) {
    const PackAt<V> at((int)c, (int)dim);
    RowPack<TT, V> raw[kRows];
    if (dim >= V) {
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (id[r] >= 0 && id[r] < vocab) raw[r].load(table + id[r] * dim + at.begin);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (first + r >= n) continue;
      const bool row = id[r] >= 0 && id[r] < vocab;
      const float none = id[r] >= 0 ? __builtin_nanf("") : 0.0f;   // off the table, or padding
      OT* const dst = out + (first + r) * dim;
      if (dim >= V) {
        float v[V];
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = row ? __fmul_rn(raw[r].get(k), scale) : none;
        store_pack(dst + at.begin, v);
      } else {
        for (int k = 0; k < (int)dim; ++k)
          dst[k] = from_f32<OT>(row ? __fmul_rn(to_f32(table[id[r] * dim + k]), scale) : none);
      }
    }
  }
}

// ---- gradient ----------------------------------------------------------------------------
//
// The sorted positions are cut into pieces of equal length whatever the ids are, so that a
// frequent id costs no more than rare ones.  A wave sums one piece over its slab of columns:
// the lanes hold the piece's positions and ids, which are wave-uniform in the loop, and two
// batches of rows are in flight (a narrow row takes fewer elements a lane, not fewer lanes:
// several pieces a wave, whose ids end at different rows, took 60000 rows of 64 35 us).  Ids that begin and end inside the piece are written at
// once; the sum of an id that continues from the piece before (the head) or into the next
// (the tail) goes to the workspace, and a second launch adds tail and heads in order.

struct Span {
  int32_t id, last;   // the id that a piece hands on (-1: none), and the piece it ends in
};

struct GradArgs {
  const int32_t* order;
  const int32_t* offsets;
  int64_t n, vocab, dim;
  float scale;
  int accumulate;
  float* dtable;
  Span* spans;         // [pieces]
  float* partial;      // [pieces][2][dim]: heads and tails
  int piece;           // positions per piece, at most a wave's lanes
  int64_t pieces;
  int slabs;           // slabs of 64 V columns
  int64_t sum_blocks;  // blocks that sum; those after them clear the rows of ids that do not occur
  int clear_rows;      // rows of the table that a clearing wave looks at, at most 16
};

// The elements of a pack that are its own.
template <int V>
__device__ __forceinline__ void store_own(float* row, const PackAt<V>& at, const float (&v)[V]) {
  if (at.shared == 0) {
    store_pack(row + at.begin, v);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (at.own(k)) row[at.begin + k] = v[k];
  }
}

// The row of the table that an id names: the scaled sum, or that added to it.  Elements that
// two packs share are stored by one of them, as the other may add to what it wrote.
template <int V>
__device__ __forceinline__ void write_row(const GradArgs& a, int64_t id, const PackAt<V>& at, float (&sum)[V]) {
  float* const row = a.dtable + id * a.dim;
#pragma unroll
  for (int k = 0; k < V; ++k) sum[k] *= a.scale;
  if (a.accumulate) {
    float old[V];
    load_pack(row + at.begin, old);
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] += old[k];
  }
  store_own(row, at, sum);
}

template <typename ID, typename GT, int V>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const GT* __restrict__ dout, const ID* __restrict__ ids,
                                                            GradArgs a) {
  constexpr int U = V * sizeof(GT) >= 16 ? 8 : 16;   // rows of a batch
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int64_t)blockIdx.x >= a.sum_blocks) {
    const int64_t v0 = (((int64_t)blockIdx.x - a.sum_blocks) * 4 + wave) * a.clear_rows;
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    // the rows' offsets at once: nothing but stores is left in the loop.  They go around the
    // caches, which the rows of dout need (each call on other buffers: 65536 rows of 1024 bf16
    // into 50021 97 -> 87 us, 4096 rows into 30000 36 -> 29, 2048 rows of 512 into 8000 15.1 -> 13.1),
    // also where rows are no whole lines (65536 of 1001 97 -> 91, 16 of 65 fp32 into 200000 21 ->
    // 17, 16384 of 510 42 either way; but 8192 of 4098 bf16 into 32000 132 -> 148)
    const int32_t from = v0 + lane <= a.vocab && lane <= a.clear_rows ? a.offsets[v0 + lane] : 0;
    const int32_t to = __shfl_down(from, 1, 64);
    uint64_t empty = __ballot(lane < a.clear_rows && v0 + lane < a.vocab && from >= to);
    for (; empty; empty &= empty - 1) {
      float* const dst = a.dtable + (v0 + __builtin_ctzll(empty)) * a.dim;
      for (int64_t c = lane * 4; c < a.dim; c += 256) {
        if (c + 4 <= a.dim) stream_pack(dst + c, zero);
        else store_row<4>(dst + c, a.dim - c, zero);
      }
    }
    return;
  }
  const int64_t job = (int64_t)blockIdx.x * 4 + wave, p = job / a.slabs;
  if (p >= a.pieces) return;
  const int64_t c = ((job - p * a.slabs) * 64 + lane) * V;
  const PackAt<V> at((int)c, (int)a.dim);   // dim >= V
  const int64_t count = min(max((int64_t)a.offsets[a.vocab], (int64_t)0), a.n);   // positions that have a group
  const int64_t q0 = p * a.piece;
  const int len = (int)max((int64_t)0, min((int64_t)a.piece, count - q0));
  // lane k: position and id of the piece's k-th row, id -1 if there is none
  int pos = 0, ident = -1;
  if (lane < len) {
    pos = a.order[q0 + lane];
    if (pos >= 0 && pos < a.n) {
      const int64_t id = (int64_t)ids[pos];
      if (id >= 0 && id < a.vocab) ident = (int)id;
    }
  }
  // the last id goes on behind the piece; the first one came from before it
  const int first_id = __builtin_amdgcn_readlane(ident, 0);
  const int last_id = len > 0 ? __builtin_amdgcn_readlane(ident, len - 1) : -1;
  const int64_t end = last_id >= 0 ? (int64_t)a.offsets[last_id + 1] : 0;
  const bool onward = end > q0 + len;
  bool head = first_id >= 0 && a.offsets[first_id] < q0;
  if (c == 0)   // a piece inside an id's run hands nothing on: it is a head as a whole
    a.spans[p] = onward && !(head && first_id == last_id)
                     ? Span{last_id, (int)min((end - 1) / a.piece, a.pieces - 1)}
                     : Span{-1, 0};
  int cur = first_id;
  float sum[V];
#pragma unroll
  for (int k = 0; k < V; ++k) sum[k] = 0.0f;
  auto flush = [&](bool last) {
    if (cur >= 0 && at.any()) {
      if (head) store_pack(a.partial + 2 * p * a.dim + at.begin, sum);
      else if (last && onward) store_pack(a.partial + (2 * p + 1) * a.dim + at.begin, sum);
      else write_row<V>(a, cur, at, sum);
    }
    head = false;
  };
  RowPack<GT, V> row[2][U];
  auto fetch = [&](int buf, int q) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q + u < len && __builtin_amdgcn_readlane(ident, q + u) >= 0 && at.any())
        row[buf][u].load(dout + (int64_t)__builtin_amdgcn_readlane(pos, q + u) * a.dim + at.begin);
  };
  auto add = [&](int buf, int q) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q + u < len) {
        const int id = __builtin_amdgcn_readlane(ident, q + u);
        if (id != cur) {
          flush(false);
          cur = id;
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] = 0.0f;
        }
        if (id >= 0) {
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] += row[buf][u].get(k);
        }
      }
  };
  if (len == 0) return;
  fetch(0, 0);
  for (int q = 0; q < len; q += 2 * U) {
    fetch(1, q + U);
    add(0, q);
    fetch(0, q + 2 * U);
    add(1, q + U);
  }
  flush(true);
}

// A workgroup for each piece and 64 V columns: where the piece hands an id on, its eight
// waves add an eighth of the later pieces' heads each, and their sums meet in LDS.
template <int V>
__global__ __launch_bounds__(512) void embedding_join_kernel(GradArgs a) {
  constexpr int W = 8, U = 8;
  __shared__ float part[W][64][V];
  const int64_t p = blockIdx.x;
  const Span span = a.spans[p];
  if (span.id < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const PackAt<V> at(((int)blockIdx.y * 64 + lane) * V, (int)a.dim);
  const int64_t heads = span.last - p, from = p + 1 + heads * wave / W, to = p + 1 + heads * (wave + 1) / W;
  float sum[V];
#pragma unroll
  for (int k = 0; k < V; ++k) sum[k] = 0.0f;
  if (at.any()) {
    if (wave == 0) load_pack(a.partial + (2 * p + 1) * a.dim + at.begin, sum);
    for (int64_t h = from; h < to; h += U) {
      float v[U][V];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (h + u < to) load_pack(a.partial + 2 * (h + u) * a.dim + at.begin, v[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (h + u < to)
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] += v[u][k];
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) part[wave][lane][k] = sum[k];
  __syncthreads();
  if (wave == 0 && at.any()) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      sum[k] = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) sum[k] += part[w][lane][k];
    }
    write_row<V>(a, span.id, at, sum);
  }
}

// log2 of the lanes a row of dim elements gets, pack elements each.
int row_lanes(int64_t dim, int pack, int most) {
  int l = 0;
  while (l < most && ((int64_t)pack << l) < dim) ++l;
  return l;
}

// Positions per piece: enough pieces to fill the machine, and no fewer than 16 positions (65536
// rows of 1024 bf16: 64 positions 100 us, 32 89, 16 94; 16384 rows: 16 positions 38, 8 44), or 8
// where 16 leave most of it idle and a piece's chain of loads and stores is what the launch
// waits for (4000 rows of 2048 fp32: 16 positions 28.3 us, 8 26.2, 4 30.8; 300 of 4096: 24.6,
// 22.2, 22.6; 8000 of 512 24.4, 23.1; but 30000 of 256 33.8, 34.6).
int grad_piece(int64_t n, int64_t dim) {
  const int64_t waves_per_piece = (dim + 255) / 256;
  int piece = 64;
  while (piece > 16 && n / piece * waves_per_piece < 8192) piece /= 2;
  if (piece == 16 && n < 16384 && n / 16 * waves_per_piece < 2048) piece = 8;
  return piece;
}

}  // namespace

hipError_t launch_embedding_fwd(const void* ids, int i64, int64_t n, const void* table, int t_bf16, int64_t vocab,
                                int64_t dim, float scale, void* out, int o_bf16, hipStream_t st) {
  auto launch = [&](auto id, auto tt, auto ot) {
    using ID = decltype(id);
    using TT = decltype(tt);
    using OT = decltype(ot);
    const int log_lanes = row_lanes(dim, kPack<TT, OT>, 8);
    const int64_t groups = 256 >> log_lanes, pass = (int64_t)kPack<TT, OT> << log_lanes;
    auto go = [&](auto kernel, int64_t rows, int64_t along) {
      // a grid holds below 2^32 threads
      const int64_t most = ((int64_t)1 << 23) * groups * rows;
      for (int64_t at = 0; at < n; at += most) {
        const int64_t m = n - at < most ? n - at : most;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((m + groups * rows - 1) / (groups * rows)), (unsigned)along),
                           dim3(256), 0, st, static_cast<const ID*>(ids) + at, m, static_cast<const TT*>(table), vocab,
                           dim, scale, static_cast<OT*>(out) + at * dim, log_lanes);
      }
    };
    // few rows: a block for every 256 packs of each, so that no load waits for another
    const int64_t along = (dim + pass - 1) / pass;
    if (n >= 4096 * groups) go(embedding_fwd_kernel<ID, TT, OT, 4>, 4, 1);
    else go(embedding_fwd_kernel<ID, TT, OT, 1>, 1, n < 1024 && along < 65536 ? along : 1);
  };
  auto types = [&](auto id) {
    if (t_bf16) o_bf16 ? launch(id, uint16_t{}, uint16_t{}) : launch(id, uint16_t{}, float{});
    else o_bf16 ? launch(id, float{}, uint16_t{}) : launch(id, float{}, float{});
  };
  i64 ? types(int64_t{}) : types(int32_t{});
  return hipGetLastError();
}

size_t embedding_grad_workspace_bytes(int64_t n, int64_t dim) {
  const int64_t piece = grad_piece(n, dim), pieces = (n + piece - 1) / piece;
  return (size_t)pieces * (sizeof(Span) + 2 * (size_t)dim * sizeof(float));
}

hipError_t launch_embedding_grad(const void* dout, int g_bf16, const void* ids, int i64, const int32_t* order,
                                 const int32_t* offsets, int64_t n, int64_t vocab, int64_t dim, float scale,
                                 int accumulate, float* dtable, void* ws, hipStream_t st) {
  GradArgs a;
  a.order = order;
  a.offsets = offsets;
  a.n = n;
  a.vocab = vocab;
  a.dim = dim;
  a.scale = scale;
  a.accumulate = accumulate;
  a.dtable = dtable;
  a.piece = grad_piece(n, dim);
  a.pieces = (n + a.piece - 1) / a.piece;
  a.spans = static_cast<Span*>(ws);
  a.partial = reinterpret_cast<float*>(a.spans + a.pieces);
  auto launch = [&](auto id, auto gt) {
    using ID = decltype(id);
    using GT = decltype(gt);
    auto sum = [&](auto pack) {
      constexpr int V = decltype(pack)::value;
      a.slabs = (int)((dim + 64 * V - 1) / (64 * V));
      a.sum_blocks = (a.pieces * a.slabs + 3) / 4;
      // 32 KB a wave, or a row (16 rows of 7136: 28 us for 381 rows of the table)
      a.clear_rows = dim < 8192 ? (int)std::min<int64_t>(16, 8192 / dim) : 1;
      const int64_t clear = accumulate ? 0 : (vocab + 4 * a.clear_rows - 1) / (4 * a.clear_rows);
      if (a.sum_blocks + clear > 0)
        hipLaunchKernelGGL((embedding_sum_kernel<ID, GT, V>), dim3((unsigned)(a.sum_blocks + clear)), dim3(256), 0, st,
                           static_cast<const GT*>(dout), static_cast<const ID*>(ids), a);
    };
    constexpr int kMost = kPack<GT, GT>;
    if (dim <= 64) sum(std::integral_constant<int, 1>{});
    else if (dim <= 128) sum(std::integral_constant<int, 2>{});
    else if (dim <= 256 || kMost == 4) sum(std::integral_constant<int, 4>{});
    else sum(std::integral_constant<int, kMost>{});
    if (a.pieces > 1) {
      auto join = [&](auto kernel, int64_t cols) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(a.pieces - 1), (unsigned)((dim + cols - 1) / cols)), dim3(512), 0, st, a);
      };
      dim < 4 ? join(embedding_join_kernel<1>, 64) : join(embedding_join_kernel<4>, 256);
    }
  };
  if (i64) g_bf16 ? launch(int64_t{}, uint16_t{}) : launch(int64_t{}, float{});
  else g_bf16 ? launch(int32_t{}, uint16_t{}) : launch(int32_t{}, float{});
  return hipGetLastError();
}

}  // namespace luq
