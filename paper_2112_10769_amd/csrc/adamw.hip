// AdamW over many tensors in one launch.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p - r wd p - r (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// The plan cuts every tensor into chunks of 4096 elements; a workgroup takes a chunk, finds its
// tensor in the plan's table, and has all of its loads in flight at once.  Bound by memory: 28
// bytes an element with fp32 states and gradients, 14 to 18 with states in 8 bits.
//
// States in 8 bits are e4m3 codes of m and sqrt(v), 32 elements (eight lanes) sharing a power
// of two: the grid of codes does not move while the block's largest element stays in its
// binade.  They are rounded stochastically: of a step to the next code of 2^-4 to 2^-3 a v with
// b2 = 0.999 changes 10^-3 at most, which rounding to nearest would lose every time.
#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

constexpr int kThreads = 256, kPer = 4, kGroups = kAdamwChunk / (kThreads * kPer);

struct AdamwArgs {
  const AdamwEntry* entries;
  const AdamwChunk* chunks;
  const float* lr;
  const int64_t* step;
  const float* grad_scale;
  double beta1, beta2;
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

// 2^(scale - 127), and 2^(127 - scale): scale is at most 247, so that the second is normal.
__device__ __forceinline__ float scale_up(int scale) {
  return __uint_as_float(scale ? (uint32_t)scale << 23 : 0x00400000u);
}
__device__ __forceinline__ float scale_down(int scale) { return __uint_as_float((uint32_t)(254 - scale) << 23); }

__device__ __forceinline__ float finite_or_zero(float a) { return a < __builtin_inff() ? a : 0.0f; }

// The e4m3 code of magnitude a, y = a over the block's power of two (exact): the code below, or
// the one above it if the fraction between them plus u / 2^16 reaches 1.  Three bits of the
// significand are kept, below 2^-6 multiples of 2^-9; codes of both ranges follow each other.
__device__ __forceinline__ uint32_t encode(float a, float down, uint32_t u) {
  const float y = a * down;
  const uint32_t whole = ((__float_as_uint(y) + (u << 4)) >> 20) - (120u << 3);
  const uint32_t small = ((uint32_t)(fminf(y, 0x1p-6f) * 0x1p29f) + (u << 4)) >> 20;
  const uint32_t code = y < 0x1p-6f ? small : whole;
  return a < __builtin_inff() ? code : 0x7Fu;
}

// Up to four elements of any type at p, as they lie in memory.
typedef uint32_t u1_any __attribute__((aligned(1)));
template <typename T>
__device__ __forceinline__ void load4(const T* p, int64_t left, float (&v)[4]) {
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
__device__ __forceinline__ uint32_t load4(const uint8_t* p, int64_t left) {
  if (left >= 4) return *reinterpret_cast<const u1_any*>(p);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < left) w |= (uint32_t)p[k] << (8 * k);
  return w;
}
__device__ __forceinline__ void store4(float* p, int64_t left, const float (&v)[4]) { store_row<4>(p, left, v); }
__device__ __forceinline__ void store4(uint16_t* p, int64_t left, const float (&v)[4]) {
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
__device__ __forceinline__ void store4(uint8_t* p, int64_t left, uint32_t w) {
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
__device__ __forceinline__ void update(const Common& c, const float (&g)[4], float (&p)[4], float (&m)[4], float (&v)[4],
                                       float (&r1)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float gk = g[k] * c.gs;
    m[k] = m[k] * c.b1 + gk * c.c1;
    v[k] = v[k] * c.b2 + gk * gk * c.c2;
    r1[k] = sqrtf(v[k]);
    p[k] = p[k] * c.keep - c.size * m[k] / (r1[k] * c.root + c.eps);
  }
}

template <typename G>
__device__ __forceinline__ void chunk_f32(const AdamwEntry& e, const Common& c, int64_t start) {
  const G* const g = static_cast<const G*>(e.g);
  float* const m = static_cast<float*>(e.m);
  float* const v = static_cast<float*>(e.v);
  float gk[kGroups][4], pk[kGroups][4], mk[kGroups][4], vk[kGroups][4], r[4];
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int64_t at = start + (i * kThreads + threadIdx.x) * kPer, left = e.n - at;
    if (left <= 0) continue;
    load4(g + at, left, gk[i]);
    load4(e.p + at, left, pk[i]);
    load4(m + at, left, mk[i]);
    load4(v + at, left, vk[i]);
  }
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int64_t at = start + (i * kThreads + threadIdx.x) * kPer, left = e.n - at;
    if (left <= 0) continue;
    update(c, gk[i], pk[i], mk[i], vk[i], r);
    store4(e.p + at, left, pk[i]);
    store4(m + at, left, mk[i]);
    store4(v + at, left, vk[i]);
    if (e.copy) store4(e.copy + at, left, pk[i]);
  }
}

template <typename G>
__device__ __forceinline__ void chunk_u8(const AdamwEntry& e, const Common& c, int64_t start, uint32_t tensor, uint32_t t,
                                         uint32_t k0, uint32_t k1) {
  const G* const g = static_cast<const G*>(e.g);
  uint8_t* const m = static_cast<uint8_t*>(e.m);
  uint8_t* const v = static_cast<uint8_t*>(e.v);
  float gk[kGroups][4], pk[kGroups][4];
  uint32_t mw[kGroups], vw[kGroups];
  int ms[kGroups], vs[kGroups];
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int64_t at = start + (i * kThreads + threadIdx.x) * kPer, left = e.n - at;
    // lanes behind the tensor hold zeros: they take part in their block's maximum
    mw[i] = vw[i] = 0;
    ms[i] = vs[i] = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) gk[i][k] = pk[i][k] = 0.0f;
    if (left <= 0) continue;
    load4(g + at, left, gk[i]);
    load4(e.p + at, left, pk[i]);
    mw[i] = load4(m + at, left);
    vw[i] = load4(v + at, left);
    ms[i] = e.m_scale[at >> 5];
    vs[i] = e.v_scale[at >> 5];
  }
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int64_t at = start + (i * kThreads + threadIdx.x) * kPer, left = e.n - at;
    float mk[4], vk[4], r[4];
    decode4(mw[i], scale_up(ms[i]), mk);
    decode4(vw[i], scale_up(vs[i]), vk);
#pragma unroll
    for (int k = 0; k < 4; ++k) vk[k] = vk[k] * vk[k];
    update(c, gk[i], pk[i], mk, vk, r);
    float m_top = 0.0f, r_top = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m_top = fmaxf(m_top, finite_or_zero(fabsf(mk[k])));
      r_top = fmaxf(r_top, finite_or_zero(r[k]));
    }
    const int m_scale = block_scale(block_max(m_top)), r_scale = block_scale(block_max(r_top));
    const float m_down = scale_down(m_scale), r_down = scale_down(r_scale);
    const uint64_t quad = (uint64_t)at >> 2;
    const U4 w = philox4x32_10(U4{(uint32_t)quad, (uint32_t)(quad >> 32), tensor, t}, k0, k1);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t mc = 0, rc = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t a = encode(fabsf(mk[k]), m_down, u[k] & 0xFFFFu);
      if (a && mk[k] < 0.0f) a |= 0x80u;
      uint32_t b = encode(r[k], r_down, u[k] >> 16);
      if (r[k] > 0.0f && b == 0) b = 1;   // it divides
      mc |= a << (8 * k);
      rc |= b << (8 * k);
    }
    if (left <= 0) continue;
    store4(e.p + at, left, pk[i]);
    store4(m + at, left, mc);
    store4(v + at, left, rc);
    if ((threadIdx.x & 7) == 0) {
      e.m_scale[at >> 5] = (uint8_t)m_scale;
      e.v_scale[at >> 5] = (uint8_t)r_scale;
    }
    if (e.copy) store4(e.copy + at, left, pk[i]);
  }
}

__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwArgs a) {
  const AdamwChunk ch = a.chunks[blockIdx.x];
  const AdamwEntry e = a.entries[ch.tensor];
  const int64_t t = max(*a.step, (int64_t)1);
  Common c;
  c.gs = a.grad_scale ? *a.grad_scale : 1.0f;
  if (!(fabsf(c.gs) < __builtin_inff())) return;
  const double rate = (double)*a.lr * (double)e.lr_scale;
  c.b1 = (float)a.beta1;
  c.c1 = (float)(1.0 - a.beta1);
  c.b2 = (float)a.beta2;
  c.c2 = (float)(1.0 - a.beta2);
  c.size = (float)(rate / (1.0 - pow(a.beta1, (double)t)));
  c.keep = (float)(1.0 - rate * (double)e.weight_decay);
  c.root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)t)));
  c.eps = a.eps;
  const int64_t start = (int64_t)ch.index * kAdamwChunk;
  if (e.state_bits == 32) {
    if (e.g_bf16) chunk_f32<uint16_t>(e, c, start);
    else chunk_f32<float>(e, c, start);
  } else {
    if (e.g_bf16) chunk_u8<uint16_t>(e, c, start, ch.tensor, (uint32_t)t, a.seed_lo, a.seed_hi);
    else chunk_u8<float>(e, c, start, ch.tensor, (uint32_t)t, a.seed_lo, a.seed_hi);
  }
}

}  // namespace

hipError_t launch_adamw(const void* plan, int64_t count, int64_t chunks, const float* lr, const int64_t* step,
                        double beta1, double beta2, float eps, const float* grad_scale, uint64_t seed, hipStream_t st) {
  const AdamwEntry* const entries = static_cast<const AdamwEntry*>(plan);
  const AdamwArgs a{entries, reinterpret_cast<const AdamwChunk*>(entries + count), lr, step, grad_scale, beta1, beta2,
                    eps, (uint32_t)seed, (uint32_t)(seed >> 32)};
  hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace luq
