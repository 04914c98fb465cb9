// Embedding lookup with scaling, and the gradient of its table.
//
//   out[i] = scale * table[ids[i]]        dtable[v] = scale * sum over ids[i] = v of dout[i]
//
// Both are bound by memory: the lookup reads and writes a row per id, the gradient reads a
// row per id and writes the table once.  The gradient takes the positions grouped by id
// (group_ids.hip), so that every row of the table has one writer and its sum one order.
#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

template <typename ID, typename TT, typename OT>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const ID* ids, const TT* table, int64_t vocab, int64_t dim,
                                                            float scale, OT* out) {
  const int64_t i = blockIdx.x, id = ids[i];
  OT* const dst = out + i * dim;
  const TT* const src = table + id * dim;
  for (int64_t c = threadIdx.x; c < dim; c += 256) {
    float v = 0.0f;
    if (id >= vocab) v = __builtin_nanf("");
    else if (id >= 0) v = __fmul_rn(to_f32(src[c]), scale);
    dst[c] = from_f32<OT>(v);
  }
}

template <typename GT>
__global__ __launch_bounds__(256) void embedding_grad_kernel(const GT* dout, const int32_t* order, const int32_t* offsets,
                                                             int64_t n, int64_t dim, float scale, int accumulate,
                                                             float* dtable) {
  const int64_t v = blockIdx.x;
  const int64_t lo = min(max((int64_t)offsets[v], (int64_t)0), n), hi = min((int64_t)offsets[v + 1], n);
  float* const dst = dtable + v * dim;
  if (accumulate && lo >= hi) return;
  for (int64_t c = threadIdx.x; c < dim; c += 256) {
    float s = 0.0f;
    for (int64_t p = lo; p < hi; ++p) {
      const int64_t i = order[p];
      if (i >= 0 && i < n) s += to_f32(dout[i * dim + c]);
    }
    s *= scale;
    dst[c] = accumulate ? dst[c] + s : s;
  }
}

}  // namespace

hipError_t launch_embedding_fwd(const void* ids, int i64, int64_t n, const void* table, int t_bf16, int64_t vocab,
                                int64_t dim, float scale, void* out, int o_bf16, hipStream_t st) {
  auto launch = [&](auto id, auto tt, auto ot) {
    using ID = decltype(id);
    using TT = decltype(tt);
    using OT = decltype(ot);
    hipLaunchKernelGGL((embedding_fwd_kernel<ID, TT, OT>), dim3((unsigned)n), dim3(256), 0, st,
                       static_cast<const ID*>(ids), static_cast<const TT*>(table), vocab, dim, scale,
                       static_cast<OT*>(out));
  };
  auto types = [&](auto id) {
    if (t_bf16) o_bf16 ? launch(id, uint16_t{}, uint16_t{}) : launch(id, uint16_t{}, float{});
    else o_bf16 ? launch(id, float{}, uint16_t{}) : launch(id, float{}, float{});
  };
  i64 ? types(int64_t{}) : types(int32_t{});
  return hipGetLastError();
}

size_t embedding_grad_workspace_bytes(int64_t, int64_t) { return 0; }

hipError_t launch_embedding_grad(const void* dout, int g_bf16, const void*, int, const int32_t* order,
                                 const int32_t* offsets, int64_t n, int64_t vocab, int64_t dim, float scale,
                                 int accumulate, float* dtable, void*, hipStream_t st) {
  const dim3 grid((unsigned)vocab);
  if (g_bf16)
    hipLaunchKernelGGL((embedding_grad_kernel<uint16_t>), grid, dim3(256), 0, st, static_cast<const uint16_t*>(dout),
                       order, offsets, n, dim, scale, accumulate, dtable);
  else
    hipLaunchKernelGGL((embedding_grad_kernel<float>), grid, dim3(256), 0, st, static_cast<const float*>(dout), order,
                       offsets, n, dim, scale, accumulate, dtable);
  return hipGetLastError();
}

}  // namespace luq
