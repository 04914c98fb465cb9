// Choice of experts: scores, the top k of them, weights; and the gradient of the logits.
//
//   s = softmax(l) or sigmoid(l),  c = s + bias,  w_k = scale s_k (/ sum of the chosen s)
//
// 8 to 64 lanes a row, each with NE neighbouring experts.  The choice is k times the largest
// key of the row (a key is a value as an unsigned number of the same order): of the lanes that
// hold it the first has the lowest index.  Without a bias, and with groups ranked by their
// largest expert, the order of c is that of the logits, whose keys need no exponential.
//
// Otherwise c is a sum, and which of two nearly equal ones is larger must not hang on a rounding:
// the row is chosen in fp32 first, and again in 64 bits where two values that the choice
// compared are nearer to each other than fp32's errors.  How many rows that are depends on the values.
// Of 16384 rows of 256 fp32 logits of deviation 1.2 in 8 groups by two it is 1 to 4 of 1000 (15 us a call).
// Equal values are near too: of bf16 logits without a bias or with one of zeros a third of the rows (34 us).
// So are scores that saturate: with a bias of 0.001 and logits of deviation 4 2% to 13% of the rows (19 to
// 25 us), without a bias at 8 a third (softmax, 34 us) or all (sigmoid, 42 us: no values take longer).
//
// Where a key's lowest bits are free (a bf16 logit's, or those of a sum, whose neighbours are looked
// at again anyway) they hold the expert's place, in the row or in the lane: taking an expert out is
// then a comparison for each key, without a branch.
//
// Bound by instructions, not by memory (16384 rows of 256 experts in 8 groups, top 8: 15 us, their
// 16.8 MB would take 3.4; a wave a row with the choice in 64 bits took 57, in fp32 with the largest of a
// lane's keys looked for at each choice 23): many rows take as few lanes as 16 experts a lane allow, few
// rows as many.  A row chosen again is waited for: 3.5 us at the end of a call that has one.
#include <type_traits>

#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

constexpr int kRouteWaves = 4, kMaxPer = 64, kMaxTop = 64;

// Keys: unsigned numbers in the order of the values; 0 is no value's (-inf is barred).
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);   // -0 is 0
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t key_of(double v) {
  const uint64_t b = __double_as_longlong(v + 0.0);
  return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(uint64_t k) {
  return __longlong_as_double(k >> 63 ? k ^ 0x8000000000000000ull : ~k);
}

// A reduction over the LPR lanes of a row, in registers; every lane gets the result.
template <int LPR, typename V, typename F>
__device__ __forceinline__ V row_reduce(V v, F f) {
  static_assert(sizeof(V) == 4, "a word");
  auto step = [&](uint32_t other) { v = f(v, __builtin_bit_cast(V, other)); };
  auto bits = [&]() { return __builtin_bit_cast(uint32_t, v); };
  step(__builtin_amdgcn_update_dpp(0, bits(), 0xB1, 0xF, 0xF, true));                     // lanes 1 0 3 2
  step(__builtin_amdgcn_update_dpp(0, bits(), 0x4E, 0xF, 0xF, true));                     // lanes 2 3 0 1
  if constexpr (LPR >= 8) step(__builtin_amdgcn_update_dpp(0, bits(), 0x141, 0xF, 0xF, true));    // eight reversed
  if constexpr (LPR >= 16) step(__builtin_amdgcn_update_dpp(0, bits(), 0x140, 0xF, 0xF, true));   // sixteen reversed
  if constexpr (LPR >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(bits(), bits(), false, false);
    const uint32_t x = s[0], y = s[1];   // (a bit cast of a vector's element takes the first)
    v = f(__builtin_bit_cast(V, x), __builtin_bit_cast(V, y));
  }
  if constexpr (LPR >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(bits(), bits(), false, false);
    const uint32_t x = s[0], y = s[1];   // (a bit cast of a vector's element takes the first)
    v = f(__builtin_bit_cast(V, x), __builtin_bit_cast(V, y));
  }
  return v;
}
template <int LPR>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  return row_reduce<LPR>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
template <int LPR>
__device__ __forceinline__ float row_max(float v) {
  return row_reduce<LPR>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LPR>
__device__ __forceinline__ float row_min(float v) {
  return row_reduce<LPR>(v, [](float a, float b) { return fminf(a, b); });
}
template <int LPR>
__device__ __forceinline__ float row_total(float v) {
  return row_reduce<LPR>(v, [](float a, float b) { return a + b; });
}
// The lanes of this lane's row that say yes, the row's first lane in bit 0.
template <int LPR>
__device__ __forceinline__ uint64_t row_ballot(bool yes) {
  const uint64_t all = __ballot(yes);
  if constexpr (LPR == kWave) return all;
  return all >> (threadIdx.x & (kWave - 1) & ~(LPR - 1)) & ((1ull << LPR) - 1);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
  return v;
}

// The first of the lanes that hold a wave's largest key, or -1 if all are 0.
__device__ __forceinline__ int wave_first(uint64_t key) {
  const uint32_t high = (uint32_t)(key >> 32), most = row_max<kWave>(high);
  if (most == 0) return -1;   // (no value's key has a high word of 0)
  uint64_t who = __ballot(high == most);
  if (who & (who - 1)) {
    const uint32_t low = high == most ? (uint32_t)key : 0, most_low = row_max<kWave>(low);
    who = __ballot(high == most && low == most_low);
  }
  return __builtin_ctzll(who);
}

// A number that is neither NaN nor +inf.
__device__ __forceinline__ bool sound(float v) { return v < __builtin_inff(); }

// Adds a pair (the first of it the larger) to the two largest keys.
template <typename K>
__device__ __forceinline__ void put_key(K& first, K& second, K k1, K k2) {
  second = max(max(min(first, k1), second), k2);
  first = max(first, k1);
}

// The choice of a row in 64 bits, by a wave; lane t has experts t * NE .. t * NE + NE - 1.
// keys: [E] in LDS; list: the choices, in LDS.  The row holds no NaN and no +inf.
template <typename T, int NE>
__device__ void route_exact(const RouteArgs& a, int64_t row, uint64_t* keys, int* list) {
  const int lane = threadIdx.x & (kWave - 1), e0 = lane * NE, left = a.E - e0;
  const T* const src = static_cast<const T*>(a.logits) + row * a.E + e0;
  float l[NE], top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    l[i] = i < left ? to_f32(src[i]) : -__builtin_inff();
    top = fmaxf(top, l[i]);
  }
  top = row_max<kWave>(top);
  uint64_t key[NE];
  double s[NE], total = 0.0;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    if (a.sigmoid) {
      s[i] = 1.0 / (1.0 + exp(-(double)l[i]));
    } else {
      s[i] = l[i] > -__builtin_inff() ? exp((double)l[i] - (double)top) : 0.0;
      total += s[i];
    }
  }
  if (!a.sigmoid) total = wave_sum64(total);
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    if (!a.sigmoid) s[i] = s[i] / total;
    const double c = a.bias && i < left ? s[i] + (double)a.bias[e0 + i] : s[i];
    key[i] = l[i] > -__builtin_inff() && c > -__builtin_inf() ? key_of(c) : 0;
  }
  if (a.groups > 1) {
    const int size = a.E / a.groups, lanes = size / NE;
    const bool whole = size % NE == 0 && (lanes & (lanes - 1)) == 0;
    uint64_t first = 0, second = 0;
    if (whole) {   // groups of a power of two of lanes
#pragma unroll
      for (int i = 0; i < NE; ++i) put_key<uint64_t>(first, second, key[i], 0);
      for (int d = 1; d < lanes; d *= 2)
        put_key<uint64_t>(first, second, __shfl_xor((unsigned long long)first, d, kWave),
                          __shfl_xor((unsigned long long)second, d, kWave));
    } else {       // lane g reads group g
#pragma unroll
      for (int i = 0; i < NE; ++i)
        if (i < left) keys[e0 + i] = key[i];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (lane < a.groups)
        for (int i = 0; i < size; ++i) put_key<uint64_t>(first, second, keys[lane * size + i], 0);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    const uint64_t rank = a.best == 2 && second ? key_of(value_of(first) + value_of(second)) : first;
    // groups before this lane's, by rank and then by place
    const int step = whole ? lanes : 1, mine = lane / step;
    int before = 0;
    for (int g = 0; g < a.groups; ++g) {
      const uint64_t r = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(rank >> 32), g * step) << 32 |
                         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)rank, g * step);
      before += r > rank || (r == rank && g < mine);
    }
    const uint64_t kept = __ballot(before < a.top_groups && mine < a.groups);
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (i < left && !(kept >> ((e0 + i) / size * step) & 1)) key[i] = 0;
  }
  // without a bias the order within the groups is that of the logits, also where scores round to the same
  // number (a sigmoid's above 37 to 1, a softmax's 745 below the largest to 0)
  if (!a.bias) {
#pragma unroll
    for (int i = 0; i < NE; ++i) key[i] = key[i] ? key_of((double)l[i]) : 0;
  }
  uint64_t best = 0;
  int at = 0;
  auto local = [&]() {
    best = key[0];
    at = 0;
#pragma unroll
    for (int i = 1; i < NE; ++i)
      if (key[i] > best) {
        best = key[i];
        at = i;
      }
  };
  local();
  for (int k = 0; k < a.K; ++k) {
    const int who = wave_first(best);
    if (lane == max(who, 0)) {
      list[k] = who >= 0 ? e0 + at : -1;
#pragma unroll
      for (int i = 0; i < NE; ++i)
        if (i == at) key[i] = 0;
      local();
    }
  }
}

// How much two values of c in fp32 may be off, together: a sigmoid is off by 5 u (its exponential
// by (2 |l| + 2) u of itself, of which s (1 - s) remains, a sum and a reciprocal by 3 u), a softmax by
// 60 u of itself (an exponential of d by (3 |d| + 2) u of itself, the sum's terms as much on average,
// the additions and the division), for which the row's largest score stands.  The addition of the bias is
// off by u |c| more.
__device__ __forceinline__ float near_of(bool sigmoid, float most_score) {
  return sigmoid ? 0x1p-20f : 0x1p-17f * most_score;
}
constexpr float kNearSum = 0x1p-23f;   // 2 u

// The comparisons of an odd-even merge sort of N keys.
template <int N>
struct SortNetwork {
  int count = 0, first[N > 1 ? N * 4 : 1] = {}, second[N > 1 ? N * 4 : 1] = {};
  constexpr SortNetwork() {
    for (int p = 1; p < N; p *= 2)
      for (int d = p; d >= 1; d /= 2)
        for (int b = d % p; b + d < N; b += 2 * d)
          for (int i = 0; i < d; ++i)
            if (i + b + d < N && (i + b) / (2 * p) == (i + b + d) / (2 * p)) {
              first[count] = i + b;
              second[count++] = i + b + d;
            }
  }
};
// Descending.
template <int N>
__device__ __forceinline__ void sort_keys(uint32_t (&k)[N]) {
  constexpr SortNetwork<N> net;
#pragma unroll
  for (int i = 0; i < net.count; ++i) {
    const uint32_t x = k[net.first[i]], y = k[net.second[i]];
    k[net.first[i]] = max(x, y);
    k[net.second[i]] = min(x, y);
  }
}

// LPR lanes a row, NE experts a lane: lane j has experts j * NE .. j * NE + NE - 1.  SUM: c is a sum.
// dynamic LDS, with groups: a region a wave for the keys of its rows, or of a row in 64 bits.
template <int LPR>
__host__ __device__ constexpr int route_wave_bytes(int E) {
  return (kWave / LPR > 2 ? kWave / LPR * 4 : 8) * E;
}
// ONE: fewer choices than lanes.
template <typename T, int LPR, int NE, bool SUM, bool ONE>
__global__ __launch_bounds__(kRouteWaves * kWave) void route_fwd_kernel(RouteArgs a, int32_t* __restrict__ chosen,
                                                                        float* __restrict__ weights) {
  constexpr int kRows = kWave / LPR, kList = LPR * NE < kMaxTop ? LPR * NE : kMaxTop, kMine = ONE ? 1 : (kList + LPR - 1) / LPR;
  // the place that a key holds: of sixteen free bits the one in the row (equal keys are then in the
  // order of their places), else the one in the lane
  constexpr bool kPacked = SUM || sizeof(T) == 2, kInRow = !SUM && sizeof(T) == 2;
  constexpr uint32_t kPlace = kInRow ? LPR * NE - 1 : kPacked ? NE - 1 : 0;
  static_assert((NE & (NE - 1)) == 0 && LPR * NE <= 65536, "a place in the lowest bits");
  // a lane's keys in order, the largest first: taking one out moves the others up
  constexpr bool kSorted = kPacked && NE <= 16;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds_keys[];
  __shared__ int lists[SUM ? kRouteWaves : 1][kMaxTop];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & (LPR - 1);
  const int64_t row0 = ((int64_t)blockIdx.x * (blockDim.x / kWave) + wave) * kRows, row = row0 + lane / LPR;
  if (row0 >= a.T) return;
  const bool in = row < a.T;
  const int e0 = j * NE, left = in ? a.E - e0 : 0;
  uint8_t* const region = lds_keys + wave * route_wave_bytes<LPR>(a.E);
  const T* const src = static_cast<const T*>(a.logits) + row * a.E;
  float l[NE];
  if (left >= NE) {
    RowPack<T, NE> pack;
    pack.load(src + e0);
#pragma unroll
    for (int i = 0; i < NE; ++i) l[i] = pack.get(i);
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i) l[i] = i < left ? to_f32(src[e0 + i]) : -__builtin_inff();
  }
  bool good = true, near = false;
  float top = l[0];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    good &= sound(l[i]);
    top = fmaxf(top, l[i]);
  }
  top = row_max<LPR>(top);
  constexpr float kLog2e = 1.44269504088896341f;
  uint32_t key[NE];
  float tolerance = 0.0f;
  auto pack_place = [&](uint32_t k, int i) { return kPacked ? (k & ~kPlace) | (kPlace - (kInRow ? e0 + i : i)) : k; };
  if constexpr (SUM) {
    float s[NE], b[NE], share = 1.0f;
    if (a.sigmoid) {
#pragma unroll
      for (int i = 0; i < NE; ++i) s[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-l[i] * kLog2e));
    } else {
      float total = 0.0f;
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        s[i] = l[i] > -__builtin_inff() ? __builtin_amdgcn_exp2f((l[i] - top) * kLog2e) : 0.0f;
        total += s[i];
      }
      share = 1.0f / row_total<LPR>(total);
    }
    if (a.bias && left >= NE) {
      RowPack<float, NE> pack;
      pack.load(a.bias + e0);
#pragma unroll
      for (int i = 0; i < NE; ++i) b[i] = pack.get(i);
    } else {
#pragma unroll
      for (int i = 0; i < NE; ++i) b[i] = a.bias && i < left ? a.bias[e0 + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const float sum = fmaf(s[i], share, b[i]);
      const float c = l[i] > -__builtin_inff() ? sum : -__builtin_inff();
      good &= sound(c);
      key[i] = c > -__builtin_inff() ? pack_place(key_of(c), i) : 0;
    }
    tolerance = near_of(a.sigmoid, share);
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i) key[i] = l[i] > -__builtin_inff() ? pack_place(key_of(l[i]), i) : 0;
  }
  const bool bad = row_ballot<LPR>(!good) != 0;
  // of a key with a place, the least and the largest value that it may stand for
  auto least = [&](uint32_t k) { return value_of(k & ~kPlace); };
  auto largest = [&](uint32_t k) { return value_of(k | kPlace); };
  // the rank of this lane's group: of whole lanes, a power of two of them, in registers; else lane g
  // of the row reads group g.  Ranks are values without places; each has the error of its sums.
  const int size = a.groups > 1 ? a.E / a.groups : 0, lanes = size / NE;
  const bool grouped = a.groups > 1, whole = size % NE == 0 && (lanes & (lanes - 1)) == 0;
  auto rank_of = [&](uint32_t first, uint32_t second) {
    if constexpr (SUM) {
      if (a.best == 2 && second) return key_of(least(first) + least(second));
    }
    return first & ~kPlace;
  };
  // the least that a rank may stand for, and the largest
  auto rank_error = [&](uint32_t first, uint32_t second) {
    return kNearSum * (fabsf(least(first)) + (a.best == 2 && second ? 2.0f * fabsf(least(second)) : 0.0f));
  };
  auto rank_least = [&](uint32_t rank, uint32_t first, uint32_t second) {
    return rank ? value_of(rank) - rank_error(first, second) : __builtin_inff();
  };
  auto rank_largest = [&](uint32_t rank, uint32_t first, uint32_t second) {
    return rank ? largest(first) + (a.best == 2 && second ? largest(second) : 0.0f) + rank_error(first, second) : -__builtin_inff();
  };
  if (grouped && !whole) {
    uint32_t* const mine = reinterpret_cast<uint32_t*>(region) + lane / LPR * a.E;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (i < left) mine[e0 + i] = key[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // groups beyond the row's lanes: a lane takes every LPR-th
    constexpr int kPerLane = kMaxTop / LPR;
    uint32_t ranks[kPerLane];
    float lows[kPerLane], highs[kPerLane];
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) {
      const int g = j + q * LPR;
      uint32_t first = 0, second = 0;
      if (in && g < a.groups)
        for (int i = 0; i < size; ++i) put_key<uint32_t>(first, second, mine[g * size + i], 0);
      ranks[q] = rank_of(first, second);
      lows[q] = rank_least(ranks[q], first, second);
      highs[q] = rank_largest(ranks[q], first, second);
    }
    uint64_t kept = 0;
    float low = __builtin_inff();
    for (int n = 0; n < a.top_groups; ++n) {
      uint32_t best = 0;
      int at = 0;
#pragma unroll
      for (int q = 0; q < kPerLane; ++q)
        if (ranks[q] > best) {
          best = ranks[q];
          at = q;
        }
      const uint32_t most = row_max<LPR>(best);
      // the lowest group of those: by q first, then by lane
      const uint64_t who = row_ballot<LPR>(best == most);
      int g = 1 << 20;
      for (uint64_t w = most ? who : 0; w; w &= w - 1) {
        const int t = __builtin_ctzll(w);
        g = min(g, t + LPR * __shfl(at, (lane & ~(LPR - 1)) + t, kWave));
      }
      if (most == 0) continue;
      kept |= 1ull << g;
#pragma unroll
      for (int q = 0; q < kPerLane; ++q)
        if (g == j + q * LPR) {
          low = fminf(low, lows[q]);
          ranks[q] = 0;
          highs[q] = -__builtin_inff();
        }
    }
    if constexpr (SUM) {
      float high = highs[0];
#pragma unroll
      for (int q = 1; q < kPerLane; ++q) high = fmaxf(high, highs[q]);
      high = row_max<LPR>(high);
      near |= high > -__builtin_inff() && row_min<LPR>(low) - high <= 2.0f * tolerance;
    }
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (i < left && !(kept >> ((e0 + i) / size) & 1)) key[i] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  if constexpr (kSorted) sort_keys(key);
  if (grouped && whole) {
    uint32_t first = 0, second = 0;
    if constexpr (kSorted) {
      first = key[0];
      second = NE > 1 ? key[NE > 1] : 0;
    } else {
#pragma unroll
      for (int i = 0; i < NE; ++i) put_key<uint32_t>(first, second, key[i], 0);
    }
#pragma unroll
    for (int d = 1; d < LPR; d *= 2)
      if (d < lanes) put_key<uint32_t>(first, second, __shfl_xor(first, d, kWave), __shfl_xor(second, d, kWave));
    uint32_t rank = rank_of(first, second);
    if (e0 >= a.E) rank = 0;
    // groups before ours, by rank and then by place
    const int mine = j / lanes;
    int before = 0;
    for (int g = 0; g < a.groups; ++g) {
      const uint32_t r = __shfl(rank, (lane & ~(LPR - 1)) + g * lanes, kWave);
      before += r > rank || (r == rank && g < mine);
    }
    const bool kept = before < a.top_groups;
    if constexpr (SUM) {
      const float low = row_min<LPR>(kept ? rank_least(rank, first, second) : __builtin_inff());
      const float high = row_max<LPR>(kept ? -__builtin_inff() : rank_largest(rank, first, second));
      near |= high > -__builtin_inff() && low - high <= 2.0f * tolerance;
    }
    if (!kept)
#pragma unroll
      for (int i = 0; i < NE; ++i) key[i] = 0;
  }
  // the choices, the k-th in lane k mod LPR; with SUM one more, for its distance
  int expert[kMine];
#pragma unroll
  for (int q = 0; q < kMine; ++q) expert[q] = -1;
  // whether the values of two keys, one behind the other, cannot be told apart
  auto too_near = [&](uint32_t k1, uint32_t k2) {
    const float v = least(k1), w = largest(k2);
    return v - w <= tolerance + kNearSum * (fabsf(v) + fabsf(w));
  };
  uint32_t last = 0, taken = 0;
  for (int k = 0; k < a.K + SUM; ++k) {
    uint32_t best = key[0];
    int at = 0;
    if constexpr (!kSorted) {
#pragma unroll
      for (int i = 1; i < NE; ++i) {
        if constexpr (!kPacked) at = key[i] > best ? i : at;
        best = max(best, key[i]);
      }
    }
    const uint32_t most = row_max<LPR>(best);
    if constexpr (SUM) {
      if constexpr (ONE) {
        taken = k == j ? most : taken;   // looked at afterwards, all at once
      } else {
        near |= k > 0 && most && too_near(last, most);
        last = most;
      }
      if (k == a.K) break;
    }
    int first = 0, index;
    if constexpr (!kInRow) {
      const uint64_t who = row_ballot<LPR>(best == most);
      first = LPR <= 32 ? __builtin_ctz((uint32_t)who) : __builtin_ctzll(who);
    }
    if constexpr (kPacked) {
      index = (int)(kPlace - (most & kPlace)) + first * NE;
      const bool out = kInRow ? best == most : j == first;
      if constexpr (kSorted) {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          const uint32_t up = i + 1 < NE ? key[i + 1 < NE ? i + 1 : i] : 0, here = key[i];   // (values: of places it makes an index)
          key[i] = out ? up : here;
        }
      } else {
#pragma unroll
        for (int i = 0; i < NE; ++i) key[i] = out && key[i] == most ? 0 : key[i];
      }
    } else {
      index = __shfl(at, (lane & ~(LPR - 1)) + first, kWave) + first * NE;
#pragma unroll
      for (int i = 0; i < NE; ++i) key[i] = j == first && i == at ? 0 : key[i];
    }
#pragma unroll
    for (int q = 0; q < kMine; ++q)
      if (k == j + q * LPR && most) expert[q] = index;
  }
  if constexpr (SUM && ONE) {
    const uint32_t behind = __shfl_down(taken, 1, kWave);
    near |= j < a.K && behind && too_near(taken, behind);
  }
  if constexpr (SUM) {
    // rows where two values are too near to tell, one after the other by the whole wave
    const bool row_near = row_ballot<LPR>(near) != 0;
    uint64_t again = __ballot(in && !bad && row_near && j == 0);
    while (again) {
      const int r = __builtin_ctzll(again) / LPR;
      again &= again - 1;
      route_exact<T, (LPR * NE + kWave - 1) / kWave>(a, row0 + r, reinterpret_cast<uint64_t*>(region), lists[wave]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int q = 0; q < kMine; ++q)
        if (lane / LPR == r && j + q * LPR < a.K) expert[q] = lists[wave][j + q * LPR];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
  if (!in) return;
  float logit[kMine], w[kMine], most = -__builtin_inff(), total = 0.0f;
#pragma unroll
  for (int q = 0; q < kMine; ++q) {
    if (bad) expert[q] = -1;
    logit[q] = expert[q] < 0 ? -__builtin_inff() : to_f32(src[expert[q]]);
    most = fmaxf(most, logit[q]);
  }
  // of shares only ratios count: scores over the largest of them, or over e^top where all are small
  const float ref = a.renorm ? (a.sigmoid ? fminf(row_max<LPR>(most), 0.0f) : row_max<LPR>(most)) : a.sigmoid ? 0.0f : top;
#pragma unroll
  for (int q = 0; q < kMine; ++q) {
    const float v = logit[q];
    w[q] = expert[q] < 0 ? 0.0f
           : !a.sigmoid  ? expf(v - ref)
           : v > 0.0f    ? 1.0f / (1.0f + expf(-v))
                         : expf(v - ref) / (1.0f + expf(v));
    total += w[q];
  }
  if (a.renorm) {
    total = row_total<LPR>(total);
  } else if (a.sigmoid) {
    total = 1.0f;
  } else {
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < NE; ++i) total += l[i] > -__builtin_inff() ? expf(l[i] - top) : 0.0f;
    total = row_total<LPR>(total);
  }
#pragma unroll
  for (int q = 0; q < kMine; ++q) {
    const int k = j + q * LPR;
    if (k >= a.K) break;
    chosen[row * a.K + k] = expert[q];
    weights[row * a.K + k] = bad ? __builtin_nanf("") : expert[q] < 0 ? 0.0f : w[q] / total * a.scale;
  }
}

// ---- backward: lane k of a row holds the k-th choice's gradient; every expert adds those that are its own

// NE elements at p, of which the row has `left`.
template <int NE, typename T>
__device__ __forceinline__ void store_elements(T* p, int left, const float (&v)[NE]) {
  constexpr int V = sizeof(T) == 4 ? 4 : 8;
  if constexpr (NE >= V) {
#pragma unroll
    for (int i = 0; i < NE; i += V) {
      float w[V];
#pragma unroll
      for (int k = 0; k < V; ++k) w[k] = v[i + k];
      store_row<V>(p + i, left - i, w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (i < left) p[i] = from_f32<T>(v[i]);
  }
}

template <typename T, int LPR, int NE>
__global__ __launch_bounds__(kRouteWaves * kWave) void route_bwd_kernel(RouteArgs a, const float* __restrict__ dweights,
                                                                        const int32_t* __restrict__ chosen, T* dlogits) {
  constexpr int kRows = kWave / LPR, kList = LPR * NE < kMaxTop ? LPR * NE : kMaxTop, kMine = (kList + LPR - 1) / LPR;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & (LPR - 1), row_lane = lane - j;
  const int64_t row = ((int64_t)blockIdx.x * kRouteWaves + wave) * kRows + lane / LPR;
  const bool in = row < a.T;
  const int e0 = j * NE, left = in ? a.E - e0 : 0;
  const T* const src = static_cast<const T*>(a.logits) + row * a.E;
  float l[NE];
  if (left >= NE) {
    RowPack<T, NE> pack;
    pack.load(src + e0);
#pragma unroll
    for (int i = 0; i < NE; ++i) l[i] = pack.get(i);
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i) l[i] = i < left ? to_f32(src[e0 + i]) : -__builtin_inff();
  }
  // the choices of lane j: j, j + LPR, ..; their logits are read before any lane writes (dlogits may
  // be logits, and a row's lanes are of one wave)
  int expert[kMine];
  float d[kMine], mine[kMine], most = -__builtin_inff();
  bool any = false;
#pragma unroll
  for (int q = 0; q < kMine; ++q) {
    const int k = j + q * LPR;
    expert[q] = in && k < a.K ? chosen[row * a.K + k] : -1;
    if (expert[q] < 0 || expert[q] >= a.E) expert[q] = -1;
    d[q] = expert[q] < 0 ? 0.0f : dweights[row * a.K + k] * a.scale;
    mine[q] = expert[q] < 0 ? -__builtin_inff() : to_f32(src[expert[q]]);
    most = fmaxf(most, mine[q]);
    any |= expert[q] >= 0;
  }
  float top = l[0];
#pragma unroll
  for (int i = 1; i < NE; ++i) top = fmaxf(top, l[i]);
  top = row_max<LPR>(top);
  float grad[kMine];   // of the choice's score; with renorm times the score's derivative
  if (a.renorm) {
    most = row_max<LPR>(most);
    const float ref = a.sigmoid ? fminf(most, 0.0f) : most;
    float s[kMine], rest[kMine], total = 0.0f, all = 0.0f;   // score over e^ref; 1 - score
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      s[q] = 0.0f;
      rest[q] = 1.0f;
      if (expert[q] >= 0) {
        const float low = expf(-fabsf(mine[q]));
        if (!a.sigmoid) {
          s[q] = expf(mine[q] - ref);
        } else if (mine[q] > 0.0f) {
          s[q] = 1.0f / (1.0f + low);
          rest[q] = low / (1.0f + low);
        } else {
          s[q] = expf(mine[q] - ref) / (1.0f + low);
          rest[q] = 1.0f / (1.0f + low);
        }
      }
      total += s[q];
    }
    total = row_total<LPR>(total);
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      s[q] = expert[q] >= 0 ? s[q] / total : 0.0f;
      all += d[q] * s[q];
    }
    all = row_total<LPR>(all);
#pragma unroll
    for (int q = 0; q < kMine; ++q) grad[q] = expert[q] >= 0 ? s[q] * (d[q] - all) * rest[q] : 0.0f;
  } else {
#pragma unroll
    for (int q = 0; q < kMine; ++q) grad[q] = d[q];
  }
  float out[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) out[i] = 0.0f;
  for (int k = 0; k < a.K; ++k) {
    int e = 0;
    float g = 0.0f;
#pragma unroll
    for (int q = 0; q < kMine; ++q)
      if (k / LPR == q) {
        e = __shfl(expert[q], row_lane + (k & (LPR - 1)), kWave) - e0;
        g = __shfl(grad[q], row_lane + (k & (LPR - 1)), kWave);
      }
#pragma unroll
    for (int i = 0; i < NE; ++i) out[i] += e == i ? g : 0.0f;
  }
  if (!a.renorm && a.sigmoid) {
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const float low = expf(-fabsf(l[i])), s = 1.0f / (1.0f + low);
      out[i] = out[i] == 0.0f ? 0.0f : out[i] * (s * (low * s));
    }
  } else if (!a.renorm) {
    float s[NE], total = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      s[i] = l[i] > -__builtin_inff() ? expf(l[i] - top) : 0.0f;
      total += s[i];
    }
    total = row_total<LPR>(total);
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      s[i] /= total;
      dot += s[i] * out[i];
    }
    dot = row_total<LPR>(dot);
    // a row without a choice: zeros, whatever its logits
    const bool some = row_ballot<LPR>(any) != 0;
#pragma unroll
    for (int i = 0; i < NE; ++i) out[i] = some ? s[i] * (out[i] - dot) : 0.0f;
  }
  if (left > 0) store_elements<NE>(dlogits + row * a.E + e0, left, out);
}

// Logits that fill the machine with 16 experts a lane (8192 rows of 256 experts: 11.2 us, 15.3 with 4 a
// lane; 16384 of 128: 11.6 and 13.5; 4096 of 128: 10.3 and 8.2; 1024 of 256: 6.0 and 4.9).
constexpr int64_t kManyLogits = 5 << 18;

// Calls f with the lanes a row takes and the experts a lane.
template <bool MANY, typename F>
void with_row_shape(int E, F f) {
  using std::integral_constant;
  if constexpr (MANY) {
    if (E > 64 && E <= 128) return f(integral_constant<int, 8>{}, integral_constant<int, 16>{});
    if (E > 128 && E <= 256) return f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    if (E > 256 && E <= 512) return f(integral_constant<int, 32>{}, integral_constant<int, 16>{});
  }
  if (E <= 8) f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  else if (E <= 16) f(integral_constant<int, 8>{}, integral_constant<int, 2>{});
  else if (E <= 32) f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
  else if (E <= 64) f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  else if (E <= 128) f(integral_constant<int, 32>{}, integral_constant<int, 4>{});
  else if (E <= 256) f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  else if (E <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  else if (E <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
  else f(integral_constant<int, 64>{}, integral_constant<int, kMaxPer>{});
}

}  // namespace

hipError_t launch_route_fwd(const RouteArgs& a, int bf16, int32_t* chosen, float* weights, hipStream_t st) {
  // without a bias and without sums the logits' order is the scores'
  const bool sum = a.bias || (a.groups > 1 && a.best == 2);
  const int waves = a.groups > 1 && a.E > 512 ? 1 : kRouteWaves;
  auto go = [&](auto lpr, auto ne) {
    constexpr int LPR = decltype(lpr)::value, NE = decltype(ne)::value;
    const int rows = waves * (kWave / LPR);
    const size_t lds = a.groups > 1 ? (size_t)waves * route_wave_bytes<LPR>(a.E) : 0;
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((a.T + rows - 1) / rows)), dim3(waves * kWave), lds, st, a, chosen, weights);
    };
    auto typed = [&](auto elem, auto one) {
      using T = decltype(elem);
      constexpr bool ONE = decltype(one)::value;
      sum ? launch(route_fwd_kernel<T, LPR, NE, true, ONE>) : launch(route_fwd_kernel<T, LPR, NE, false, ONE>);
    };
    auto counted = [&](auto one) { bf16 ? typed(uint16_t{}, one) : typed(float{}, one); };
    if (a.K < LPR) counted(std::true_type{});
    else counted(std::false_type{});
  };
  if (a.T * a.E >= kManyLogits) with_row_shape<true>(a.E, go);
  else with_row_shape<false>(a.E, go);
  return hipGetLastError();
}

hipError_t launch_route_bwd(const RouteArgs& a, int bf16, const float* dweights, const int32_t* chosen, void* dlogits,
                            hipStream_t st) {
  // (8111 rows of 160 experts: 7 us with 16 experts a lane)
  with_row_shape<false>(a.E, [&](auto lpr, auto ne) {
    constexpr int LPR = decltype(lpr)::value, NE = decltype(ne)::value, rows = kRouteWaves * (kWave / LPR);
    auto launch = [&](auto kernel, auto* out) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((a.T + rows - 1) / rows)), dim3(kRouteWaves * kWave), 0, st, a, dweights, chosen, out);
    };
    if (bf16) launch(route_bwd_kernel<uint16_t, LPR, NE>, static_cast<uint16_t*>(dlogits));
    else launch(route_bwd_kernel<float, LPR, NE>, static_cast<float*>(dlogits));
  });
  return hipGetLastError();
}

}  // namespace luq
