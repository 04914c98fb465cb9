// Choice of experts: scores, the top k of them, weights; and the gradient of the logits.
//
//   s = softmax(l) or sigmoid(l),  c = s + bias,  w_k = scale s_k (/ sum of the chosen s)
//
// A wave a row.  The choice is k times the largest key of the row: a key is c as an unsigned
// number of the same order.  Without a bias, and with groups ranked by their largest expert,
// the order of c is that of the logits, whose keys need no exponential; otherwise c is
// formed in 64 bits, so that two implementations that round differently choose alike.
#include <type_traits>

#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

constexpr int kRouteWaves = 4, kMaxPer = 64;

// Keys: unsigned numbers in the order of the values; 0 is no value's (-inf is barred).
__device__ __forceinline__ uint64_t key_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);   // -0 is 0
  return (uint64_t)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | 0xFFFFFFFFu;
}
__device__ __forceinline__ uint64_t key_of(double v) {
  const uint64_t b = __double_as_longlong(v + 0.0);
  return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
  return v;
}
__device__ __forceinline__ float wave_max32(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, kWave));
  return v;
}

// The largest key of a wave and the lowest index that has it (a lane's own are the largest of
// its keys and that one's index).
__device__ __forceinline__ void wave_best(uint64_t& key, int& index) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    const uint64_t k = __shfl_xor((unsigned long long)key, d, kWave);
    const int i = __shfl_xor(index, d, kWave);
    if (k > key || (k == key && i < index)) {
      key = k;
      index = i;
    }
  }
}

// A number that is neither NaN nor +inf.
__device__ __forceinline__ bool sound(float v) { return v < __builtin_inff(); }
__device__ __forceinline__ bool sound(double v) { return v < __builtin_inf(); }

// NE experts a lane: expert i of lane t is i * 64 + t.  WIDE: c in 64 bits.
template <typename T, int NE, bool WIDE>
__global__ __launch_bounds__(kRouteWaves * kWave) void route_fwd_kernel(RouteArgs a, int32_t* __restrict__ chosen,
                                                                        float* __restrict__ weights) {
  extern __shared__ uint64_t lds_keys[];   // [waves][E], with groups
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / kWave) + wave;
  if (row >= a.T) return;
  const T* const src = static_cast<const T*>(a.logits) + row * a.E;
  float l[NE];
  bool good = true;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = i * kWave + lane;
    l[i] = e < a.E ? to_f32(src[e]) : -__builtin_inff();
    good &= sound(l[i]);
  }
  float top = l[0];
#pragma unroll
  for (int i = 1; i < NE; ++i) top = fmaxf(top, l[i]);
  top = wave_max32(top);
  uint64_t key[NE];
  if constexpr (WIDE) {
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
    if (!a.sigmoid) {
      total = wave_sum64(total);
#pragma unroll
      for (int i = 0; i < NE; ++i) s[i] = s[i] / total;
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = i * kWave + lane;
      const double c = a.bias && e < a.E ? s[i] + (double)a.bias[e] : s[i];
      const bool barred = !(l[i] > -__builtin_inff()) || c == -__builtin_inf();
      good &= barred || sound(c);
      key[i] = barred ? 0 : key_of(c);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i) key[i] = l[i] > -__builtin_inff() ? key_of(l[i]) : 0;
  }
  if (__ballot(good) != ~0ull) {
    if (lane < a.K) {
      chosen[row * a.K + lane] = -1;
      weights[row * a.K + lane] = __builtin_nanf("");
    }
    return;
  }
  if (a.groups > 1) {
    // lane g ranks group g
    uint64_t* const mine = lds_keys + wave * a.E;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = i * kWave + lane;
      if (e < a.E) mine[e] = key[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int size = a.E / a.groups;
    uint64_t rank = 0;
    if (lane < a.groups) {
      uint64_t first = 0, second = 0;
      for (int j = 0; j < size; ++j) {
        const uint64_t k = mine[lane * size + j];
        if (k > first) {
          second = first;
          first = k;
        } else if (k > second) {
          second = k;
        }
      }
      rank = first;
      if constexpr (WIDE) {
        if (a.best == 2 && second) {
          auto value = [](uint64_t k) {
            return __longlong_as_double(k >> 63 ? k ^ 0x8000000000000000ull : ~k);
          };
          rank = key_of(value(first) + value(second));
        }
      }
    }
    uint64_t kept = 0;   // a bit for each group
    for (int j = 0; j < a.top_groups; ++j) {
      uint64_t k = rank;
      int g = lane;
      wave_best(k, g);
      if (k == 0) break;
      kept |= 1ull << g;
      if (lane == g) rank = 0;
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = i * kWave + lane;
      if (e < a.E && !(kept >> (e / size) & 1)) key[i] = 0;
    }
  }
  // lane k keeps the k-th choice
  int my_expert = -1;
  float my_logit = -__builtin_inff();
  for (int k = 0; k < a.K; ++k) {
    uint64_t best = key[0];
    int index = lane;
#pragma unroll
    for (int i = 1; i < NE; ++i)
      if (key[i] > best) {
        best = key[i];
        index = i * kWave + lane;
      }
    wave_best(best, index);
    if (best == 0) break;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (index == i * kWave + lane) {
        key[i] = 0;
        v = l[i];
      }
    v = __shfl(v, index & (kWave - 1), kWave);
    if (lane == k) {
      my_expert = index;
      my_logit = v;
    }
  }
  const bool have = my_expert >= 0;
  float w = 0.0f;
  if (a.renorm) {
    // of shares only ratios count: scores over the largest of them, or over e^top where all are small
    const float most = wave_max32(my_logit);
    if (a.sigmoid) {
      const float ref = fminf(most, 0.0f);
      w = !have ? 0.0f : my_logit > 0.0f ? 1.0f / (1.0f + expf(-my_logit)) : expf(my_logit - ref) / (1.0f + expf(my_logit));
    } else {
      w = have ? expf(my_logit - most) : 0.0f;
    }
    const float total = wave_sum(w);
    w = total > 0.0f ? w / total : 0.0f;
  } else if (a.sigmoid) {
    w = have ? 1.0f / (1.0f + expf(-my_logit)) : 0.0f;
  } else {
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < NE; ++i) total += l[i] > -__builtin_inff() ? expf(l[i] - top) : 0.0f;
    total = wave_sum(total);
    w = have ? expf(my_logit - top) / total : 0.0f;
  }
  if (lane < a.K) {
    chosen[row * a.K + lane] = my_expert;
    weights[row * a.K + lane] = w * a.scale;
  }
}

// ---- backward: lane k holds the k-th choice's gradient; every expert adds those that are its own

template <typename T, int NE>
__global__ __launch_bounds__(kRouteWaves * kWave) void route_bwd_kernel(RouteArgs a, const float* __restrict__ dweights,
                                                                        const int32_t* __restrict__ chosen, T* dlogits) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t row = (int64_t)blockIdx.x * kRouteWaves + wave;
  if (row >= a.T) return;
  const T* const src = static_cast<const T*>(a.logits) + row * a.E;
  float l[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = i * kWave + lane;
    l[i] = e < a.E ? to_f32(src[e]) : -__builtin_inff();
  }
  int expert = lane < a.K ? chosen[row * a.K + lane] : -1;
  if (expert < 0 || expert >= a.E) expert = -1;
  const bool have = expert >= 0;
  const float d = have ? dweights[row * a.K + lane] * a.scale : 0.0f;
  T* const dst = dlogits + row * a.E;
  const uint64_t some = __ballot(have);
  float out[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) out[i] = 0.0f;
  if (some) {
    // the choices' logits, from the row as it was read (dlogits may be logits)
    float mine = 0.0f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const float v = __shfl(l[i], expert & (kWave - 1), kWave);
      if (expert / kWave == i) mine = v;
    }
    if (!have) mine = -__builtin_inff();
    float top = l[0];
#pragma unroll
    for (int i = 1; i < NE; ++i) top = fmaxf(top, l[i]);
    top = wave_max32(top);
    float grad = d;      // of the choice's score; with renorm and softmax times the score
    if (a.renorm) {
      const float most = wave_max32(mine), ref = a.sigmoid ? fminf(most, 0.0f) : most;
      float s = 0.0f, rest = 1.0f;   // score over e^ref; 1 - score
      if (have) {
        const float low = expf(-fabsf(mine));
        if (!a.sigmoid) {
          s = expf(mine - ref);
        } else if (mine > 0.0f) {
          s = 1.0f / (1.0f + low);
          rest = low / (1.0f + low);
        } else {
          s = expf(mine - ref) / (1.0f + low);
          rest = 1.0f / (1.0f + low);
        }
      }
      const float total = wave_sum(s), share = s / total;
      const float all = wave_sum(have ? d * share : 0.0f);
      grad = have ? share * (d - all) * rest : 0.0f;
      for (int k = 0; k < a.K; ++k) {
        const int e = __shfl(expert, k, kWave);
        const float g = __shfl(grad, k, kWave);
#pragma unroll
        for (int i = 0; i < NE; ++i)
          if (e == i * kWave + lane) out[i] += g;
      }
    } else {
      for (int k = 0; k < a.K; ++k) {
        const int e = __shfl(expert, k, kWave);
        const float g = __shfl(grad, k, kWave);
#pragma unroll
        for (int i = 0; i < NE; ++i)
          if (e == i * kWave + lane) out[i] += g;
      }
      if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          const float low = expf(-fabsf(l[i])), s = 1.0f / (1.0f + low);
          out[i] = out[i] == 0.0f ? 0.0f : out[i] * (s * (low * s));
        }
      } else {
        float s[NE], total = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          s[i] = l[i] > -__builtin_inff() ? expf(l[i] - top) : 0.0f;
          total += s[i];
        }
        total = wave_sum(total);
#pragma unroll
        for (int i = 0; i < NE; ++i) {
          s[i] /= total;
          dot += s[i] * out[i];
        }
        dot = wave_sum(dot);
#pragma unroll
        for (int i = 0; i < NE; ++i) out[i] = s[i] * (out[i] - dot);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = i * kWave + lane;
    if (e < a.E) dst[e] = from_f32<T>(out[i]);
  }
}

// Calls f with the experts a lane holds.
template <typename F>
void with_per_lane(int E, F f) {
  const int n = (E + kWave - 1) / kWave;
  if (n <= 1) f(std::integral_constant<int, 1>{});
  else if (n <= 2) f(std::integral_constant<int, 2>{});
  else if (n <= 4) f(std::integral_constant<int, 4>{});
  else if (n <= 8) f(std::integral_constant<int, 8>{});
  else if (n <= 16) f(std::integral_constant<int, 16>{});
  else f(std::integral_constant<int, kMaxPer>{});
}

}  // namespace

hipError_t launch_route_fwd(const RouteArgs& a, int bf16, int32_t* chosen, float* weights, hipStream_t st) {
  // without a bias and without sums the logits' order is the scores'
  const bool wide = a.bias || (a.groups > 1 && a.best == 2);
  const int waves = a.groups > 1 && a.E > 512 ? 1 : kRouteWaves;
  const size_t lds = a.groups > 1 ? (size_t)waves * a.E * sizeof(uint64_t) : 0;
  with_per_lane(a.E, [&](auto ne) {
    constexpr int NE = decltype(ne)::value;
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((a.T + waves - 1) / waves)), dim3(waves * kWave), lds, st, a, chosen, weights);
    };
    if (bf16) wide ? go(route_fwd_kernel<uint16_t, NE, true>) : go(route_fwd_kernel<uint16_t, NE, false>);
    else wide ? go(route_fwd_kernel<float, NE, true>) : go(route_fwd_kernel<float, NE, false>);
  });
  return hipGetLastError();
}

hipError_t launch_route_bwd(const RouteArgs& a, int bf16, const float* dweights, const int32_t* chosen, void* dlogits,
                            hipStream_t st) {
  const unsigned blocks = (unsigned)((a.T + kRouteWaves - 1) / kRouteWaves);
  with_per_lane(a.E, [&](auto ne) {
    constexpr int NE = decltype(ne)::value;
    if (bf16)
      hipLaunchKernelGGL((route_bwd_kernel<uint16_t, NE>), dim3(blocks), dim3(kRouteWaves * kWave), 0, st, a, dweights, chosen,
                         static_cast<uint16_t*>(dlogits));
    else
      hipLaunchKernelGGL((route_bwd_kernel<float, NE>), dim3(blocks), dim3(kRouteWaves * kWave), 0, st, a, dweights, chosen,
                         static_cast<float*>(dlogits));
  });
  return hipGetLastError();
}

}  // namespace luq
