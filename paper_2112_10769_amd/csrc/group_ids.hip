// Positions grouped by id: a stable sort of (id, position) and the offsets of every id in
// the result.
//
// Up to kRankKeys ids of fewer than 2^18 groups (an id and a position share a word): one
// launch, every position's rank counted against all ids.  Beyond, a least-significant-digit
// radix sort.  Each pass sorts by one digit of at most 9 bits: a histogram of every block's range, then
// a scatter in which every block derives its bases from all blocks' histograms (so no
// launch is spent on a scan) and ranks its keys by ballots, wave by wave in order of
// position.  Nothing depends on the order in which blocks or atomics run: the histogram's
// LDS atomics only count.
//
// Ids outside [0, groups) get the key `groups`, which sorts last.
//
// Bound by latency: 509 ids take 3.5 us, 65536 of 50021 22 us in five launches (27 traced, 4
// to 6 each); 8 ids of 262144 groups, three passes, 25 us a call against 13 of 262143.
#include "luq_device.hpp"
#include "luq_launch.hpp"

namespace luq {

namespace {

constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kItems = 1, kPiece = kSortThreads * kItems;   // keys a block ranks at a time
constexpr int kMaxSortBlocks = 128;

// Where a pass reads its keys from.
enum Source { kIds32, kIds64, kKeys };

struct SortPass {
  const void* keys;      // ids or keys
  const int32_t* pos;    // positions of the keys, or null: the keys are in order of position
  int64_t n, per;        // per: keys a block covers, a multiple of kPiece
  uint32_t groups;
  int shift, bits, blocks;
};

template <int SRC>
__device__ __forceinline__ uint32_t load_key(const SortPass& a, int64_t i) {
  if constexpr (SRC == kKeys) return static_cast<const uint32_t*>(a.keys)[i];
  const int64_t id = SRC == kIds32 ? (int64_t)static_cast<const int32_t*>(a.keys)[i]
                                   : static_cast<const int64_t*>(a.keys)[i];
  return id >= 0 && id < (int64_t)a.groups ? (uint32_t)id : a.groups;
}

template <int SRC>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass a, uint32_t* counts) {
  __shared__ uint32_t hist[kBins];
  const int bins = 1 << a.bits;
  for (int d = threadIdx.x; d < bins; d += kSortThreads) hist[d] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * a.per, hi = min(lo + a.per, a.n);
  for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads)
    atomicAdd(&hist[(load_key<SRC>(a, i) >> a.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += kSortThreads) counts[(int64_t)blockIdx.x * bins + d] = hist[d];
}

// Exclusive prefix sums of one value per thread over the block; scratch holds a word per wave.
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t* scratch) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  uint32_t sum = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint32_t up = (uint32_t)__shfl_up((int)sum, d, kWave);
    if (lane >= d) sum += up;
  }
  if (lane == kWave - 1) scratch[wave] = sum;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += scratch[w];
  __syncthreads();
  return before + sum - v;
}

template <int SRC>
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortPass a, const uint32_t* counts,
                                                                   uint32_t* out_keys, int32_t* out_pos) {
  __shared__ uint32_t base[kBins];
  __shared__ uint32_t count[kSortWaves][kBins];
  __shared__ uint32_t scratch[kSortWaves];
  __shared__ uint32_t totals[kSortThreads], befores[kSortThreads];
  const int bins = 1 << a.bits, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t lo = (int64_t)blockIdx.x * a.per, hi = min(lo + a.per, a.n);
  // wave w ranks the keys [w * 64 * kItems, ...) of a piece, 64 at a time; the next piece's
  // are read ahead, the first one's while the histograms come
  uint32_t next_key[kItems];
  int32_t next_pos[kItems];
  auto fetch = [&](int64_t piece) {
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int64_t i = piece + (wave * kItems + k) * kWave + lane;
      next_key[k] = i < hi ? load_key<SRC>(a, i) : 0;
      next_pos[k] = i < hi && a.pos ? a.pos[i] : (int32_t)i;
    }
  };
  fetch(lo);
  // where this block's keys of digit d begin: all smaller digits, then the blocks before
  // (the block's threads share the blocks of a digit, 16 histograms in flight each)
  const int d0 = threadIdx.x, shares = kSortThreads >> a.bits, share = threadIdx.x >> a.bits;
  uint32_t total = 0, before = 0;
  for (int b0 = share * 16; b0 < a.blocks; b0 += shares * 16) {
    uint32_t c[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) c[k] = b0 + k < a.blocks ? counts[(b0 + k) * bins + (d0 & (bins - 1))] : 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (b0 + k < (int)blockIdx.x) before += c[k];
      total += c[k];
    }
  }
  totals[threadIdx.x] = total;
  befores[threadIdx.x] = before;
  __syncthreads();
  total = before = 0;
  if (d0 < bins)
    for (int k = 0; k < shares; ++k) {
      total += totals[(k << a.bits) + d0];
      before += befores[(k << a.bits) + d0];
    }
  const uint32_t smaller = block_prefix(total, scratch);
  if (d0 < bins) base[d0] = smaller + before;
  for (int64_t piece = lo; piece < hi; piece += kPiece) {
    for (int w = 0; w < kSortWaves; ++w)
      if (d0 < bins) count[w][d0] = 0;
    __syncthreads();
    uint32_t key[kItems], rank[kItems];
    int32_t pos[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      key[k] = next_key[k];
      pos[k] = next_pos[k];
    }
    if (piece + kPiece < hi) fetch(piece + kPiece);
    volatile uint32_t* mine = count[wave];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int64_t i = piece + (wave * kItems + k) * kWave + lane;
      const bool in = i < hi;
      const uint32_t d = (key[k] >> a.shift) & (bins - 1);
      uint64_t same = __ballot(in);
      for (int bit = 0; bit < a.bits; ++bit) {
        const uint64_t set = __ballot((d >> bit) & 1);
        same &= (d >> bit) & 1 ? set : ~set;
      }
      const uint64_t below = same & ((1ull << lane) - 1);
      const uint32_t first = in ? mine[d] : 0;
      rank[k] = first + __popcll(below);
      // all lanes have read the count before the lowest lane of the digit raises it
      if (in && below == 0) mine[d] = first + __popcll(same);
    }
    __syncthreads();
    if (d0 < bins) {
      uint32_t run = base[d0];
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = count[w][d0];
        count[w][d0] = run;
        run += c;
      }
      base[d0] = run;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int64_t i = piece + (wave * kItems + k) * kWave + lane;
      if (i < hi) {
        const uint32_t at = count[wave][(key[k] >> a.shift) & (bins - 1)] + rank[k];
        out_keys[at] = key[k];
        out_pos[at] = pos[k];
      }
    }
    __syncthreads();
  }
}

// The offsets from the sorted keys: a block takes 64 of them into LDS, and its 256 threads
// fill the offsets from the key before its first up to its last, each by bisection (few keys
// a block: rare ids lie far apart).  One key past the end is `groups`.  Where these offsets are
// more than kWideOffsets, the first blocks fill them instead: a wave for every kSpread ids
// finds where its ids' keys are (the whole sort with one block for each wide range, and so:
// 65536 ids of 50021, most of them small, 52 and 27 us; all alike 39 and 26; of 2^20 442 and
// 33; evenly spread 23 both).
constexpr int kOffsetKeys = 64, kWideOffsets = 4096, kSpread = 1024;
static_assert(kOffsetKeys == kWave && kSpread < kWideOffsets, "see spread_offsets");

// Offsets of the ids [v0, v0 + kSpread) among those of wide ranges.  There are two such ranges
// at most, those of the first and the last id, as any other lies between these.
__device__ __forceinline__ void spread_offsets(const uint32_t* __restrict__ keys, int64_t n, uint32_t groups, int64_t v0,
                                               int32_t* offsets) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t v1 = min(v0 + kSpread - 1, (int64_t)groups);
  // keys below v0 and below v1, by probes of 64 keys each
  int64_t at[2] = {0, 0}, left[2] = {n, n};
  while (left[0] > 0 || left[1] > 0) {
    uint32_t key[2];
    int64_t step[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      step[i] = (left[i] + kWave - 1) / kWave;
      const int64_t p = (lane + 1) * step[i] - 1;
      key[i] = p >= 0 && p < left[i] ? keys[at[i] + p] : 0xFFFFFFFFu;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t below = __popcll(__ballot((int64_t)key[i] < (i ? v1 : v0))) * step[i];
      at[i] += below;
      left[i] = max((int64_t)0, min(step[i] - 1, left[i] - below));
    }
  }
  int64_t done = -1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t p0 = at[i] / kOffsetKeys * kOffsetKeys;
    if (p0 == done) break;
    done = p0;
    const uint32_t key = p0 + lane < n ? keys[p0 + lane] : groups;
    const int64_t prev = p0 > 0 ? (int64_t)keys[p0 - 1] : -1, last = (uint32_t)__shfl((int)key, kOffsetKeys - 1, kWave);
    if (last - prev <= kWideOffsets) continue;
    const int64_t end = min(last, v1);
    for (int64_t v = max(prev + 1, v0); v <= end; v += kWave) {
      int below = 0;   // of the keys; the last is not
#pragma unroll
      for (int d = kOffsetKeys / 2; d >= 1; d >>= 1)
        if ((int64_t)(uint32_t)__shfl((int)key, below + d - 1, kWave) < v + lane) below += d;
      if (v + lane <= end) offsets[v + lane] = (int32_t)(p0 + below);
    }
  }
}

__global__ __launch_bounds__(256) void group_offsets_kernel(const uint32_t* __restrict__ keys, int64_t n, uint32_t groups,
                                                            int32_t* offsets, int spread_blocks) {
  if ((int)blockIdx.x < spread_blocks) {
    const int64_t v0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / kWave) * kSpread;
    if (v0 <= (int64_t)groups) spread_offsets(keys, n, groups, v0, offsets);
    return;
  }
  __shared__ uint32_t k[kOffsetKeys];
  const int64_t p0 = ((int64_t)blockIdx.x - spread_blocks) * kOffsetKeys, p = p0 + threadIdx.x;
  if (threadIdx.x < kOffsetKeys) k[threadIdx.x] = p < n ? keys[p] : groups;
  const int64_t prev = p0 > 0 ? (int64_t)keys[p0 - 1] : -1;
  __syncthreads();
  const int64_t last = k[kOffsetKeys - 1];
  if (last - prev > kWideOffsets) return;
  for (int64_t v = prev + 1 + threadIdx.x; v <= last; v += 256) {
    int at = 0;   // keys below v; the last is not
#pragma unroll
    for (int d = kOffsetKeys / 2; d >= 1; d >>= 1)
      if (k[at + d - 1] < (uint32_t)v) at += d;
    offsets[v] = (int32_t)(p0 + at);
  }
}

// Few ids: a block ranks 16 positions, each by 64 threads that compare it with a 64th of
// all of them.  A position's word is (key, position) + 1, so that its rank is the number of
// smaller words, and the largest of those is its predecessor: where that has a smaller key,
// the position is the first of its group and the offsets between the two are filled with its
// rank, by a wave or, where they are many, by the block (16 ids of 250000: 41 us by a wave, 13).
// n^2 comparisons of four instructions: 4096 ids are 1.7 us of the machine's VALU.
constexpr int kRankBits = 13, kRankKeys = 1 << kRankBits, kRanked = 16;

// offsets[v] = value for v in [from, to).
struct Fill {
  int32_t from, to, value;
};

template <int SRC>
__global__ __launch_bounds__(1024) void rank_kernel(SortPass a, int32_t* order, int32_t* offsets) {
  __shared__ __attribute__((aligned(16))) uint32_t words[kRankKeys];
  __shared__ uint32_t rank_s[kRanked], prev_s[kRanked];
  __shared__ Fill fill[kRanked + 1];
  const int n = (int)a.n, steps = (n + 255) / 256;
  for (int i = threadIdx.x; i < steps * 256; i += 1024)
    words[i] = i < n ? (load_key<SRC>(a, i) << kRankBits) + i + 1 : 0xFFFFFFFFu;
  if (threadIdx.x < kRanked) rank_s[threadIdx.x] = prev_s[threadIdx.x] = 0;
  __syncthreads();
  const int slot = threadIdx.x % kRanked, part = threadIdx.x / kRanked;
  const int i = blockIdx.x * kRanked + slot;
  const uint32_t mine = i < n ? words[i] : 0;
  uint32_t rank = 0, prev = 0;
  for (int k = 0; k < steps; ++k) {
    const uint4 w = *reinterpret_cast<const uint4*>(words + (k * 64 + part) * 4);
    for (const uint32_t v : {w.x, w.y, w.z, w.w}) {
      const bool less = v < mine;
      rank += less;
      prev = max(prev, less ? v : 0u);
    }
  }
#pragma unroll
  for (int d = kRanked; d < kWave; d <<= 1) {
    rank += (uint32_t)__shfl_xor((int)rank, d, kWave);
    prev = max(prev, (uint32_t)__shfl_xor((int)prev, d, kWave));
  }
  if ((threadIdx.x & (kWave - 1)) < kRanked) {
    atomicAdd(&rank_s[slot], rank);
    atomicMax(&prev_s[slot], prev);
  }
  __syncthreads();
  if (threadIdx.x < kRanked) {
    const bool in = i < n;
    rank = rank_s[slot];
    prev = prev_s[slot];
    const int32_t key = in ? (int32_t)((mine - 1) >> kRankBits) : 0;
    const int32_t prev_key = prev ? (int32_t)((prev - 1) >> kRankBits) : -1;
    if (in) order[rank] = i;
    fill[slot] = in ? Fill{prev_key + 1, key + 1, (int32_t)rank} : Fill{0, 0, 0};
    // after the last id, unless positions without a group (key = groups) have filled them
    if (slot == 0) fill[kRanked] = Fill{0, 0, 0};
  }
  __syncthreads();
  if (threadIdx.x < kRanked && i < n && (int)rank == n - 1) fill[kRanked] = Fill{fill[slot].to, (int32_t)a.groups + 1, n};
  __syncthreads();
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const Fill range = fill[min(lane, kRanked)];
  const bool many = range.to - range.from > 4 * kWave;
  for (uint64_t todo = __ballot(lane <= kRanked && (many || (lane & (kRanked - 1)) == wave)); todo; todo &= todo - 1) {
    const int s = __builtin_ctzll(todo);
    const bool all = __shfl((int)many, s, kWave);
    const Fill f = fill[s];
    for (int v = f.from + (all ? (int)threadIdx.x : lane); v < f.to; v += all ? 1024 : kWave) offsets[v] = f.value;
  }
}

struct SortPlan {
  int passes, bits, blocks;   // passes = 0: ranked in one launch
  int64_t per;
};

SortPlan plan_sort(int64_t n, int64_t groups) {
  int bits = 1;
  while ((groups >> bits) != 0) ++bits;   // keys 0 .. groups
  SortPlan p{};
  if (n <= kRankKeys && bits + kRankBits < 32) return p;
  p.passes = (bits + kDigitBits - 1) / kDigitBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  const int64_t pieces = (n + kPiece - 1) / kPiece;
  const int64_t per = (pieces + kMaxSortBlocks - 1) / kMaxSortBlocks;
  p.per = per * kPiece;
  p.blocks = (int)((pieces + per - 1) / (per > 0 ? per : 1));
  return p;
}

size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

}  // namespace

// Two sets of keys and positions, and the blocks' histograms.
size_t group_ids_workspace_bytes(int64_t n, int64_t groups) {
  const SortPlan p = plan_sort(n, groups);
  if (n == 0 || p.passes == 0) return 0;
  return 4 * round256((size_t)n * 4) + (size_t)p.blocks * kBins * 4;
}

hipError_t launch_group_ids(const void* ids, int i64, int64_t n, int64_t groups, int32_t* order, int32_t* offsets,
                            void* ws, hipStream_t st) {
  uint8_t* w = static_cast<uint8_t*>(ws);
  const size_t part = round256((size_t)n * 4);
  const uint32_t* sorted = nullptr;
  const SortPlan p = plan_sort(n, groups);
  SortPass a{};
  a.keys = ids;
  a.n = n;
  a.groups = (uint32_t)groups;
  if (n > 0 && p.passes == 0) {
    const dim3 grid((unsigned)((n + kRanked - 1) / kRanked));
    if (i64) hipLaunchKernelGGL((rank_kernel<kIds64>), grid, dim3(1024), 0, st, a, order, offsets);
    else hipLaunchKernelGGL((rank_kernel<kIds32>), grid, dim3(1024), 0, st, a, order, offsets);
    return hipGetLastError();
  }
  if (n > 0) {
    uint32_t* const counts = reinterpret_cast<uint32_t*>(w + 4 * part);
    a.per = p.per;
    a.bits = p.bits;
    a.blocks = p.blocks;
    for (int pass = 0; pass < p.passes; ++pass) {
      a.shift = pass * p.bits;
      uint32_t* const keys = reinterpret_cast<uint32_t*>(w + 2 * (pass & 1) * part);
      int32_t* const pos = pass + 1 == p.passes ? order : reinterpret_cast<int32_t*>(w + (2 * (pass & 1) + 1) * part);
      auto launch = [&](auto count, auto scatter) {
        hipLaunchKernelGGL(count, dim3(p.blocks), dim3(kSortThreads), 0, st, a, counts);
        hipLaunchKernelGGL(scatter, dim3(p.blocks), dim3(kSortThreads), 0, st, a, counts, keys, pos);
      };
      if (pass > 0) launch(sort_count_kernel<kKeys>, sort_scatter_kernel<kKeys>);
      else if (i64) launch(sort_count_kernel<kIds64>, sort_scatter_kernel<kIds64>);
      else launch(sort_count_kernel<kIds32>, sort_scatter_kernel<kIds32>);
      a.keys = keys;
      a.pos = pos;
      sorted = keys;
    }
  }
  // no range is wide if all ids together are not
  const int spread = groups + 1 > kWideOffsets ? (int)(groups / (4 * kSpread) + 1) : 0;
  hipLaunchKernelGGL(group_offsets_kernel, dim3((unsigned)(spread + n / kOffsetKeys + 1)), dim3(256), 0, st, sorted, n,
                     (uint32_t)groups, offsets, spread);
  return hipGetLastError();
}

}  // namespace luq
