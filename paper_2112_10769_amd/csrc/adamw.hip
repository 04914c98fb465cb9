// AdamW over many tensors in one launch.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p - r wd p - r (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// The plan cuts every tensor into chunks of 4096 elements; a workgroup takes chunk after chunk, the
// next one's tensor looked up meanwhile in the plan's table, and has all of a chunk's loads in flight
// at once.  Bound by memory: 28 bytes an element with fp32 states and gradients (134 M elements: 720 us,
// 5.2 TB/s), 14 to 18 with states in 8 bits (51 M with bf16 gradients and a copy: 175 us, 4.7 TB/s).
//
// States in 8 bits are e4m3 codes of m and sqrt(v), 32 elements (eight lanes) sharing a power
// of two: the grid of codes does not move while the block's largest element stays in its
// binade.  Their form is kept short (148 instructions an element made 51 M of them take 239 us): a
// code is the top of a float whose smallest normal number is e4m3's, and roots and quotients are the
// hardware's, off by one unit of the last place or two.  They are rounded stochastically: of a step to
// the next code of 2^-4 to 2^-3 a v with b2 = 0.999 changes 10^-3 at most, which rounding to nearest
// would lose every time.
#include <math.h>

#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

constexpr int kGroupsPerCu = 16;
constexpr int kThreads = 256, kPer = 4, kGroups = kAdamwChunk / (kThreads * kPer);

struct AdamwArgs {
  const AdamwEntry* entries;
  const AdamwChunk* chunks;
  const float* lr;
  const int64_t* step;
  const float* grad_scale;
  int64_t count;
  double beta1, beta2, log_beta1, log_beta2;   // the logarithms to base 2
  float eps;
  uint32_t seed_lo, seed_hi;
};

// What all elements of a chunk have in common.
struct Common {
  float b1, c1, b2, c2, size, keep, root, eps, gs;
};

template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true)));
}

// The largest of the eight lanes that hold a block.
__device__ __forceinline__ float block_max(float v) {
  v = dpp_max<0xB1>(v);    // lanes 1 0 3 2
  v = dpp_max<0x4E>(v);    // lanes 2 3 0 1
  return dpp_max<0x141>(v);   // the eight lanes reversed
}

// Biased exponent of a block's power of two: its largest magnitude over 2^(scale - 127) is in
// [128, 256), so that the code above it is a finite one.  (The exponent field of a subnormal
// number is 0, of a block of zeros too.)
__device__ __forceinline__ int block_scale(float top) { return max((int)(__float_as_uint(top) >> 23) - 7, 0); }

// 2^(scale - 127).
__device__ __forceinline__ float scale_up(int scale) {
  return __uint_as_float(scale ? (uint32_t)scale << 23 : 0x00400000u);
}

__device__ __forceinline__ float finite_or_zero(float a) { return a < __builtin_inff() ? a : 0.0f; }

// The e4m3 code of magnitude a: of a over the block's power of two and over 2^120, so that e4m3's
// subnormal numbers are fp32's, the sign-less upper twelve bits; or the code above if the fraction
// between the two plus u / 2^16 reaches 1.  What is not finite becomes NaN; a NaN too comes in without
// its sign, whose bit the addition would carry out of the word.
__device__ __forceinline__ uint32_t encode(float a, int scale, uint32_t u) {
  const uint32_t bits = __float_as_uint(__builtin_amdgcn_ldexpf(a, 7 - scale));
  return min((bits + (u << 4)) >> 20, 0x7Fu);
}

// sqrt(v), off by a unit of the last place; the instruction takes a subnormal v as 0.
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v);
  return small ? r * 0x1p-32f : r;
}

// Up to four elements of any type at p, as they lie in memory.
typedef uint32_t u1_any __attribute__((aligned(1)));
template <typename T>
__device__ __forceinline__ void load4(const T* p, int left, float (&v)[4]) {
  if (left >= 4) {
    RowPack<T, 4> q;
    q.load(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = q.get(k);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = k < left ? to_f32(p[k]) : 0.0f;
  }
}
__device__ __forceinline__ uint32_t load4(const uint8_t* p, int left) {
  if (left >= 4) return *reinterpret_cast<const u1_any*>(p);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < left) w |= (uint32_t)p[k] << (8 * k);
  return w;
}
__device__ __forceinline__ void store4(float* p, int left, const float (&v)[4]) { store_row<4>(p, left, v); }
__device__ __forceinline__ void store4(uint16_t* p, int left, const float (&v)[4]) {
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    w[k] = (uint32_t)from_f32<uint16_t>(v[2 * k]) | (uint32_t)from_f32<uint16_t>(v[2 * k + 1]) << 16;
  if (left >= 4) {
    typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(2)));
    *reinterpret_cast<u2_any*>(p) = u2_any{w[0], w[1]};
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < left) p[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
  }
}
__device__ __forceinline__ void store4(uint8_t* p, int left, uint32_t w) {
  if (left >= 4) *reinterpret_cast<u1_any*>(p) = w;
  else
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < left) p[k] = (uint8_t)(w >> (8 * k));
}

// The four values of a word of e4m3 codes.
__device__ __forceinline__ void decode4(uint32_t w, float up, float (&v)[4]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = a[0] * up;
  v[1] = a[1] * up;
  v[2] = b[0] * up;
  v[3] = b[1] * up;
}

// The moments and the weights of four elements; r1 is the root of the new v.
template <bool EXACT>
__device__ __forceinline__ void update(const Common& c, const float (&g)[4], float (&p)[4], float (&m)[4], float (&v)[4],
                                       float (&r1)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float gk = g[k] * c.gs;
    m[k] = m[k] * c.b1 + gk * c.c1;
    v[k] = v[k] * c.b2 + gk * gk * c.c2;
    r1[k] = EXACT ? sqrtf(v[k]) : root_of(v[k]);
    const float under = r1[k] * c.root + c.eps;
    p[k] = p[k] * c.keep - (EXACT ? c.size * m[k] / under : c.size * m[k] * __builtin_amdgcn_rcpf(under));
  }
}

// WHOLE: all of the chunk's elements belong to the tensor.  Pointers are to the chunk's first element.
template <typename G, bool WHOLE>
__device__ __forceinline__ void chunk_f32(const AdamwEntry& e, const Common& c, int64_t start) {
  const int n = WHOLE ? kAdamwChunk : (int)(e.n - start);
  const G* const g = static_cast<const G*>(e.g) + start;
  float* const p = e.p + start;
  float* const m = static_cast<float*>(e.m) + start;
  float* const v = static_cast<float*>(e.v) + start;
  uint16_t* const copy = e.copy ? e.copy + start : nullptr;
  float gk[kGroups][4], pk[kGroups][4], mk[kGroups][4], vk[kGroups][4], r[4];
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int at = (i * kThreads + (int)threadIdx.x) * kPer, left = WHOLE ? kPer : n - at;
    if (left <= 0) continue;
    load4(g + at, left, gk[i]);
    load4(p + at, left, pk[i]);
    load4(m + at, left, mk[i]);
    load4(v + at, left, vk[i]);
  }
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int at = (i * kThreads + (int)threadIdx.x) * kPer, left = WHOLE ? kPer : n - at;
    if (left <= 0) continue;
    update<true>(c, gk[i], pk[i], mk[i], vk[i], r);
    store4(p + at, left, pk[i]);
    store4(m + at, left, mk[i]);
    store4(v + at, left, vk[i]);
    if (copy) store4(copy + at, left, pk[i]);
  }
}

template <typename G, bool WHOLE>
__device__ __forceinline__ void chunk_u8(const AdamwEntry& e, const Common& c, int64_t start, uint32_t tensor, uint32_t t,
                                         uint32_t k0, uint32_t k1) {
  const int n = WHOLE ? kAdamwChunk : (int)(e.n - start);
  const G* const g = static_cast<const G*>(e.g) + start;
  float* const p = e.p + start;
  uint8_t* const m = static_cast<uint8_t*>(e.m) + start;
  uint8_t* const v = static_cast<uint8_t*>(e.v) + start;
  uint8_t* const m_scale_at = e.m_scale + start / 32;
  uint8_t* const v_scale_at = e.v_scale + start / 32;
  uint16_t* const copy = e.copy ? e.copy + start : nullptr;
  float gk[kGroups][4], pk[kGroups][4];
  uint32_t mw[kGroups], vw[kGroups];
  int ms[kGroups], vs[kGroups];
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int at = (i * kThreads + (int)threadIdx.x) * kPer, left = WHOLE ? kPer : n - at;
    // lanes behind the tensor hold zeros: they take part in their block's maximum
    mw[i] = vw[i] = 0;
    ms[i] = vs[i] = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) gk[i][k] = pk[i][k] = 0.0f;
    if (left <= 0) continue;
    load4(g + at, left, gk[i]);
    load4(p + at, left, pk[i]);
    mw[i] = load4(m + at, left);
    vw[i] = load4(v + at, left);
    ms[i] = m_scale_at[at >> 5];
    vs[i] = v_scale_at[at >> 5];
  }
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int at = (i * kThreads + (int)threadIdx.x) * kPer, left = WHOLE ? kPer : n - at;
    float mk[4], vk[4], r[4];
    decode4(mw[i], scale_up(ms[i]), mk);
    decode4(vw[i], scale_up(vs[i]), vk);
#pragma unroll
    for (int k = 0; k < 4; ++k) vk[k] = vk[k] * vk[k];
    update<false>(c, gk[i], pk[i], mk, vk, r);
    // the blocks' largest magnitudes (NaN is passed over; an infinity is looked for again without it)
    float m_top = block_max(fmaxf(fmaxf(fabsf(mk[0]), fabsf(mk[1])), fmaxf(fabsf(mk[2]), fabsf(mk[3]))));
    float r_top = block_max(fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3])));
    if (__ballot(fmaxf(m_top, r_top) == __builtin_inff())) {
      m_top = r_top = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m_top = fmaxf(m_top, finite_or_zero(fabsf(mk[k])));
        r_top = fmaxf(r_top, finite_or_zero(r[k]));
      }
      m_top = block_max(m_top);
      r_top = block_max(r_top);
    }
    const int m_scale = block_scale(m_top), r_scale = block_scale(r_top);
    const uint64_t quad = (uint64_t)(start >> 2) + (uint32_t)(at >> 2);
    const U4 w = philox4x32_10(U4{(uint32_t)quad, (uint32_t)(quad >> 32), tensor, t}, k0, k1);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t mc = 0, rc = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t a = encode(fabsf(mk[k]), m_scale, u[k] & 0xFFFFu) | (__float_as_uint(mk[k]) >> 24 & 0x80u);
      // a root above 0 does not become 0: it divides
      const uint32_t b = max(encode(fabsf(r[k]), r_scale, u[k] >> 16), min(__float_as_uint(r[k]), 1u));
      mc |= a << (8 * k);
      rc |= b << (8 * k);
    }
    if (left <= 0) continue;
    store4(p + at, left, pk[i]);
    store4(m + at, left, mc);
    store4(v + at, left, rc);
    if ((threadIdx.x & 7) == 0) {
      m_scale_at[at >> 5] = (uint8_t)m_scale;
      v_scale_at[at >> 5] = (uint8_t)r_scale;
    }
    if (copy) store4(copy + at, left, pk[i]);
  }
}

template <typename G>
__device__ __forceinline__ void chunk(const AdamwEntry& e, const Common& c, const AdamwChunk& ch, uint32_t t, const AdamwArgs& a) {
  const int64_t start = (int64_t)ch.index * kAdamwChunk;
  const bool whole = e.n - start >= kAdamwChunk;
  if (e.state_bits == 32) {
    if (whole) chunk_f32<G, true>(e, c, start);
    else chunk_f32<G, false>(e, c, start);
  } else {
    if (whole) chunk_u8<G, true>(e, c, start, ch.tensor, t, a.seed_lo, a.seed_hi);
    else chunk_u8<G, false>(e, c, start, ch.tensor, t, a.seed_lo, a.seed_hi);
  }
}

__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwArgs a) {
  AdamwChunk ch = a.chunks[blockIdx.x];
  AdamwEntry e = a.entries[ch.tensor];
  const int64_t t = max(*a.step, (int64_t)1);
  const double lr = *a.lr;
  Common c;
  c.gs = a.grad_scale ? *a.grad_scale : 1.0f;
  if (!(fabsf(c.gs) < __builtin_inff())) return;
  c.b1 = (float)a.beta1;
  c.c1 = (float)(1.0 - a.beta1);
  c.b2 = (float)a.beta2;
  c.c2 = (float)(1.0 - a.beta2);
  c.root = (float)(1.0 / sqrt(1.0 - exp2((double)t * a.log_beta2)));
  c.eps = a.eps;
  const double bias = 1.0 - exp2((double)t * a.log_beta1);
  for (int64_t at = blockIdx.x;;) {
    const int64_t next = at + gridDim.x;
    AdamwChunk next_ch = ch;
    if (next < a.count) next_ch = a.chunks[next];
    const AdamwEntry next_e = a.entries[next_ch.tensor];
    const double rate = lr * (double)e.lr_scale;
    c.size = (float)(rate / bias);
    c.keep = (float)(1.0 - rate * (double)e.weight_decay);
    if (e.g_bf16) chunk<uint16_t>(e, c, ch, (uint32_t)t, a);
    else chunk<float>(e, c, ch, (uint32_t)t, a);
    if (next >= a.count) break;
    at = next;
    ch = next_ch;
    e = next_e;
  }
}

}  // namespace

hipError_t launch_adamw(const void* plan, int64_t count, int64_t chunks, const float* lr, const int64_t* step,
                        double beta1, double beta2, float eps, const float* grad_scale, uint64_t seed, hipStream_t st) {
  const AdamwEntry* const entries = static_cast<const AdamwEntry*>(plan);
  const AdamwArgs a{entries, reinterpret_cast<const AdamwChunk*>(entries + count), lr, step, grad_scale, chunks, beta1, beta2,
                    log2(beta1), log2(beta2), eps, (uint32_t)seed, (uint32_t)(seed >> 32)};
  // a workgroup takes several chunks of many: what they have in common (two powers in 64 bits) is a
  // third of the instructions of one
  const int64_t most = kGroupsPerCu * 256;
  hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)(chunks < most ? chunks : most)), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace luq
