// Layer norm, forward and backward.
//
//   y = (x - mean) * rstd * gamma + beta,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   with xh = (x - mean) * rstd and a = dy * gamma:
//   dx = rstd * (a - mean(a) - xh * mean(a * xh)),  dgamma = sum dy * xh,  dbeta = sum dy
//
// Statistics and sums are fp32; the variance is taken from the differences to the mean, so
// that rows far from zero keep their digits.
#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

// Sum over a block of 256 threads; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float* scratch) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  return (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void layernorm_fwd_kernel(const T* x, int64_t cols, const float* gamma,
                                                            const float* beta, float eps, T* y, float* mean,
                                                            float* rstd) {
  __shared__ float scratch[4];
  const int64_t row = blockIdx.x;
  const T* const src = x + row * cols;
  T* const dst = y + row * cols;
  float s = 0.0f;
  for (int64_t c = threadIdx.x; c < cols; c += 256) s += to_f32(src[c]);
  const float mu = block_sum(s, scratch) / (float)cols;
  float q = 0.0f;
  for (int64_t c = threadIdx.x; c < cols; c += 256) {
    const float d = to_f32(src[c]) - mu;
    q += d * d;
  }
  const float r = 1.0f / sqrtf(block_sum(q, scratch) / (float)cols + eps);
  for (int64_t c = threadIdx.x; c < cols; c += 256) {
    const float xh = (to_f32(src[c]) - mu) * r;
    dst[c] = from_f32<T>(xh * (gamma ? gamma[c] : 1.0f) + (beta ? beta[c] : 0.0f));
  }
  if (threadIdx.x == 0) {
    if (mean) mean[row] = mu;
    if (rstd) rstd[row] = r;
  }
}

template <typename G, typename T>
__global__ __launch_bounds__(256) void layernorm_dx_kernel(const G* dy, const T* x, const float* mean, const float* rstd,
                                                           const float* gamma, int64_t cols, G* dx) {
  __shared__ float scratch[4];
  const int64_t row = blockIdx.x;
  const float mu = mean[row], r = rstd[row];
  const G* const g = dy + row * cols;
  const T* const src = x + row * cols;
  float s1 = 0.0f, s2 = 0.0f;
  for (int64_t c = threadIdx.x; c < cols; c += 256) {
    const float a = to_f32(g[c]) * (gamma ? gamma[c] : 1.0f);
    s1 += a;
    s2 += a * ((to_f32(src[c]) - mu) * r);
  }
  s1 = block_sum(s1, scratch) / (float)cols;
  s2 = block_sum(s2, scratch) / (float)cols;
  for (int64_t c = threadIdx.x; c < cols; c += 256) {
    const float a = to_f32(g[c]) * (gamma ? gamma[c] : 1.0f);
    dx[row * cols + c] = from_f32<G>(r * (a - s1 - (to_f32(src[c]) - mu) * r * s2));
  }
}

// A workgroup sums 64 columns over all rows, its four waves every fourth row.
template <typename G, typename T>
__global__ __launch_bounds__(256) void layernorm_dgamma_kernel(const G* dy, const T* x, const float* mean,
                                                               const float* rstd, int64_t rows, int64_t cols,
                                                               float* dgamma, float* dbeta) {
  __shared__ float red[2][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float sg = 0.0f, sb = 0.0f;
  if (c < cols)
    for (int64_t row = wave; row < rows; row += 4) {
      const float g = to_f32(dy[row * cols + c]);
      sg += g * ((to_f32(x[row * cols + c]) - mean[row]) * rstd[row]);
      sb += g;
    }
  red[0][wave][lane] = sg;
  red[1][wave][lane] = sb;
  __syncthreads();
  if (wave == 0 && c < cols) {
    if (dgamma) dgamma[c] = (red[0][0][lane] + red[0][1][lane]) + (red[0][2][lane] + red[0][3][lane]);
    if (dbeta) dbeta[c] = (red[1][0][lane] + red[1][1][lane]) + (red[1][2][lane] + red[1][3][lane]);
  }
}

}  // namespace

hipError_t launch_layernorm_fwd(const void* x, int bf16, int64_t rows, int64_t cols, const float* gamma,
                                const float* beta, float eps, void* y, float* mean, float* rstd, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  const dim3 grid((unsigned)rows);
  if (bf16)
    hipLaunchKernelGGL((layernorm_fwd_kernel<uint16_t>), grid, dim3(256), 0, st, static_cast<const uint16_t*>(x), cols,
                       gamma, beta, eps, static_cast<uint16_t*>(y), mean, rstd);
  else
    hipLaunchKernelGGL((layernorm_fwd_kernel<float>), grid, dim3(256), 0, st, static_cast<const float*>(x), cols, gamma,
                       beta, eps, static_cast<float*>(y), mean, rstd);
  return hipGetLastError();
}

size_t layernorm_bwd_workspace_bytes(int64_t, int64_t) { return 0; }

hipError_t launch_layernorm_bwd(const void* dy, int g_bf16, const void* x, int bf16, const float* mean,
                                const float* rstd, const float* gamma, int64_t rows, int64_t cols, void* dx,
                                float* dgamma, float* dbeta, void*, hipStream_t st) {
  auto launch = [&](auto g, auto t) {
    using G = decltype(g);
    using T = decltype(t);
    // the column sums first: dx may be dy
    if (dgamma || dbeta)
      hipLaunchKernelGGL((layernorm_dgamma_kernel<G, T>), dim3((unsigned)((cols + 63) / 64)), dim3(256), 0, st,
                         static_cast<const G*>(dy), static_cast<const T*>(x), mean, rstd, rows, cols, dgamma, dbeta);
    if (rows > 0)
      hipLaunchKernelGGL((layernorm_dx_kernel<G, T>), dim3((unsigned)rows), dim3(256), 0, st,
                         static_cast<const G*>(dy), static_cast<const T*>(x), mean, rstd, gamma, cols,
                         static_cast<G*>(dx));
  };
  if (g_bf16) bf16 ? launch(uint16_t{}, uint16_t{}) : launch(uint16_t{}, float{});
  else bf16 ? launch(float{}, uint16_t{}) : launch(float{}, float{});
  return hipGetLastError();
}

}  // namespace luq
