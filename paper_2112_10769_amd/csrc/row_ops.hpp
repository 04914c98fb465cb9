// Helpers of the kernels that work on rows of float tensors (layer norm, embedding):
// elements as fp32 whatever their type, and sums over a wave.
#pragma once

#include "luq_device.hpp"

namespace luq {

// A bfloat16 is held as its bits.
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// Rounded to nearest even; a NaN stays one.
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ uint16_t from_f32<uint16_t>(float v) {
  return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// V consecutive elements at p, which is aligned to its elements only: rows of any width
// begin anywhere, and the memory unit takes 16-byte accesses at any address.
typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(2)));

template <int V>
__device__ __forceinline__ void load_pack(const float* p, float (&v)[V]) {
  if constexpr (V < 4) {
    typedef float fv __attribute__((ext_vector_type(V), aligned(4)));
    const fv q = *reinterpret_cast<const fv*>(p);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = q[k];
    return;
  }
  typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int i = 0; i < V; i += 4) {
    const f4 q = *reinterpret_cast<const f4*>(p + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[i + k] = q[k];
  }
}
template <int V>
__device__ __forceinline__ void load_pack(const uint16_t* p, float (&v)[V]) {
  static_assert(V == 8, "one 16-byte piece");
  const u4_any q = *reinterpret_cast<const u4_any*>(p);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(q[k] << 16);
    v[2 * k + 1] = __uint_as_float(q[k] & 0xFFFF0000u);
  }
}
template <int V>
__device__ __forceinline__ void store_pack(float* p, const float (&v)[V]) {
  if constexpr (V < 4) {
    typedef float fv __attribute__((ext_vector_type(V), aligned(4)));
    fv q;
#pragma unroll
    for (int k = 0; k < V; ++k) q[k] = v[k];
    *reinterpret_cast<fv*>(p) = q;
    return;
  }
  typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int i = 0; i < V; i += 4) *reinterpret_cast<f4*>(p + i) = f4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}
template <int V>
__device__ __forceinline__ void store_pack(uint16_t* p, const float (&v)[V]) {
  static_assert(V == 8 || V == 1, "one 16-byte piece, or one element");
  if constexpr (V == 1) {
    *p = from_f32<uint16_t>(v[0]);
    return;
  }
  u4_any q;
#pragma unroll
  for (int k = 0; k < V / 2; ++k)
    q[k] = (uint32_t)from_f32<uint16_t>(v[2 * k]) | (uint32_t)from_f32<uint16_t>(v[2 * k + 1]) << 16;
  *reinterpret_cast<u4_any*>(p) = q;
}

// As store_pack, non-temporally.
__device__ __forceinline__ void stream_pack(float* p, const float (&v)[4]) {
  typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
  __builtin_nontemporal_store(f4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f4*>(p));
}

// The same for the `left` elements that a row has from p on: a whole pack, or its first
// elements (the others read as 0 and are not written).
template <int V, typename T>
__device__ __forceinline__ void load_row(const T* p, int64_t left, float (&v)[V]) {
  if (left >= V) {
    load_pack(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = k < left ? to_f32(p[k]) : 0.0f;
  }
}
template <int V, typename T>
__device__ __forceinline__ void store_row(T* p, int64_t left, const float (&v)[V]) {
  if (left >= V) {
    store_pack(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k < left) p[k] = from_f32<T>(v[k]);
  }
}

// A pack as it lies in memory, converted when it is used: loads of later rows are in flight
// in as few registers as they have bytes.
template <typename T, int V>
struct RowPack {
  static constexpr int kBytes = V * sizeof(T), W = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int k = 0; k < W; k += 4) {
        const u4_any q = reinterpret_cast<const u4_any*>(p)[k / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[k + i] = q[i];
      }
    } else if constexpr (kBytes == 8) {
      typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(2)));
      const u2_any q = *reinterpret_cast<const u2_any*>(p);
      w[0] = q[0];
      w[1] = q[1];
    } else if constexpr (kBytes == 4) {
      typedef uint32_t u1_any __attribute__((aligned(2)));
      w[0] = *reinterpret_cast<const u1_any*>(p);
    } else {
      w[0] = *p;
    }
  }
  __device__ __forceinline__ float get(int k) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
    return __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
  }
};

// A row of `cols` >= V columns in packs of V: the pack that begins at column c < cols lies at
// column begin = min(c, cols - V), so that the last one is whole too.  Its first `shared`
// elements are then the pack before's as well: they are left out of sums, and stored twice
// with the same value (a pack read element by element made every row wait for its loads).
template <int V>
struct PackAt {
  int begin, shared;   // shared = V: the row has no such pack
  __device__ __forceinline__ PackAt() {}
  __device__ __forceinline__ PackAt(int c, int cols) {   // below 2^24
    begin = min(c, cols - V);
    shared = min(c - begin, V);
  }
  __device__ __forceinline__ bool any() const { return shared < V; }
  __device__ __forceinline__ bool own(int k) const { return k >= shared; }
};

// Elements a lane takes at a time: 16 bytes of the narrower type.
template <typename A, typename B>
constexpr int kPack = sizeof(A) == 2 || sizeof(B) == 2 ? 8 : 4;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
  return v;
}

}  // namespace luq
