// Layer norm, forward and backward.
//
//   y = (x - mean) * rstd * gamma + beta,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   with xh = (x - mean) * rstd and a = dy * gamma:
//   dx = rstd * (a - mean(a) - xh * mean(a * xh)),  dgamma = sum dy * xh,  dbeta = sum dy
//
// Bound by memory: the forward reads and writes a row once, the backward reads two and
// writes one.  A row stays in registers between its sums and its output, spread over a wave
// or a workgroup; a workgroup takes several rows, the next one's loads in flight while one
// is reduced, and keeps the weights (and the sums of their gradients) in registers for all
// of them.  Wider rows than registers hold are read again instead.
//
// Statistics and sums are fp32; the variance is taken from the differences to the mean, so
// that rows far from zero keep their digits.
#include <type_traits>

#include "luq_launch.hpp"
#include "row_ops.hpp"

namespace luq {

namespace {

// Sums of K values over the TPR threads of a row (a wave, or a workgroup of TPR); every
// thread gets them.  red belongs to this use: a workgroup that calls it again must have
// passed another barrier in between.
template <int TPR, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float (*red)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
  if constexpr (TPR > kWave) {
    if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) red[threadIdx.x / kWave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.0f;
#pragma unroll
      for (int w = 0; w < TPR / kWave; ++w) v[k] += red[w][k];
    }
  }
}

// Rows a workgroup works on at a time, and its threads.
template <int TPR>
constexpr int kRowsAtOnce = TPR > kWave ? 1 : 256 / TPR;
template <int TPR>
constexpr int kThreads = TPR > kWave ? TPR : 256;

// A thread's CH packs of a row: pack i of thread t holds the columns from (i * TPR + t) * V on.
template <typename T, int V, int TPR, int CH>
struct RowRaw {
  RowPack<T, V> pack[CH];
  __device__ __forceinline__ void load(const T* row, int64_t cols, int t) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t c = (int64_t)(i * TPR + t) * V;
      pack[i].load(row + c, cols - c);
    }
  }
  __device__ __forceinline__ float get(int i, int k) const { return pack[i].get(k); }
};

template <typename T, int TPR, int CH>
__global__ __launch_bounds__(kThreads<TPR>) void layernorm_fwd_kernel(const T* x, int64_t rows, int64_t cols,
                                                                      const float* __restrict__ gamma,
                                                                      const float* __restrict__ beta, float eps, T* y,
                                                                      float* __restrict__ mean,
                                                                      float* __restrict__ rstd) {
  constexpr int V = kPack<T, T>, R = kRowsAtOnce<TPR>;
  __shared__ float red1[TPR / kWave][1], red2[TPR / kWave][1];
  const int t = threadIdx.x & (TPR - 1);
  const float inv = 1.0f / (float)cols;
  float g[CH][V], b[CH][V];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int64_t c = (int64_t)(i * TPR + t) * V;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      g[i][k] = 1.0f;
      b[i][k] = 0.0f;
    }
    if (gamma) load_row<V>(gamma + c, cols - c, g[i]);
    if (beta) load_row<V>(beta + c, cols - c, b[i]);
  }
  RowRaw<T, V, TPR, CH> next;
  int64_t row = (int64_t)blockIdx.x * R + (TPR > kWave ? 0 : threadIdx.x / TPR);
  const int64_t step = (int64_t)gridDim.x * R;
  if (row < rows) next.load(x + row * cols, cols, t);
  for (; row < rows; row += step) {
    const RowRaw<T, V, TPR, CH> cur = next;
    if (row + step < rows) next.load(x + (row + step) * cols, cols, t);
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) s[0] += cur.get(i, k);
    row_sum<TPR, 1>(s, red1);
    const float mu = s[0] * inv;
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t left = cols - (int64_t)(i * TPR + t) * V;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = k < left ? cur.get(i, k) - mu : 0.0f;
        q[0] = fmaf(d, d, q[0]);
      }
    }
    row_sum<TPR, 1>(q, red2);
    const float r = 1.0f / sqrtf(q[0] * inv + eps);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t c = (int64_t)(i * TPR + t) * V;
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = fmaf((cur.get(i, k) - mu) * r, g[i][k], b[i][k]);
      store_row<V>(y + row * cols + c, cols - c, v);
    }
    if (t == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = r;
    }
  }
}

// Rows wider than registers hold: read three times (from L2 after the first).
template <typename T>
__global__ __launch_bounds__(1024) void layernorm_fwd_wide_kernel(const T* x, int64_t rows, int64_t cols,
                                                                  const float* __restrict__ gamma,
                                                                  const float* __restrict__ beta, float eps, T* y,
                                                                  float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int V = kPack<T, T>, TPR = 1024;
  __shared__ float red1[TPR / kWave][1], red2[TPR / kWave][1];
  const float inv = 1.0f / (float)cols;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* const src = x + row * cols;
    float s[1] = {0.0f}, q[1] = {0.0f}, v[V];
    for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
      load_row<V>(src + c, cols - c, v);
#pragma unroll
      for (int k = 0; k < V; ++k) s[0] += v[k];
    }
    row_sum<TPR, 1>(s, red1);
    const float mu = s[0] * inv;
    for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
      load_row<V>(src + c, cols - c, v);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = k < cols - c ? v[k] - mu : 0.0f;
        q[0] = fmaf(d, d, q[0]);
      }
    }
    row_sum<TPR, 1>(q, red2);
    const float r = 1.0f / sqrtf(q[0] * inv + eps);
    for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
      float g[V], b[V];
      load_row<V>(src + c, cols - c, v);
      if (gamma) load_row<V>(gamma + c, cols - c, g);
      if (beta) load_row<V>(beta + c, cols - c, b);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = fmaf((v[k] - mu) * r, gamma ? g[k] : 1.0f, beta ? b[k] : 0.0f);
      store_row<V>(y + row * cols + c, cols - c, v);
    }
    if (threadIdx.x == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = r;
    }
  }
}

// ---- backward ----------------------------------------------------------------------------

struct BwdArgs {
  const float* mean;
  const float* rstd;
  const float* gamma;
  int64_t rows, cols;
  float* partial;   // [workgroups][2][cols]: each workgroup's sums for dgamma and dbeta
};

template <typename G, typename T, int TPR, int CH>
__global__ __launch_bounds__(kThreads<TPR>) void layernorm_bwd_kernel(const G* dy, const T* __restrict__ x, BwdArgs a,
                                                                      G* dx) {
  constexpr int V = kPack<G, T>, R = kRowsAtOnce<TPR>;
  // 1024 threads have 128 registers each: with 16 elements a thread the weight is read again
  // for every row and no row is fetched ahead (all of it kept spilled 174 to 220 registers)
  constexpr bool kTight = TPR == 1024 && CH * V > 8;
  __shared__ float red[2][TPR / kWave][2];
  const int t = threadIdx.x & (TPR - 1);
  const int64_t rows = a.rows, cols = a.cols;
  const float inv = 1.0f / (float)cols;
  float g[CH][V], dg[CH][V], db[CH][V];
  auto weight = [&](int i) {
    const int64_t c = (int64_t)(i * TPR + t) * V;
#pragma unroll
    for (int k = 0; k < V; ++k) g[i][k] = 1.0f;
    if (a.gamma) load_row<V>(a.gamma + c, cols - c, g[i]);
  };
#pragma unroll
  for (int i = 0; i < CH; ++i) {
#pragma unroll
    for (int k = 0; k < V; ++k) dg[i][k] = db[i][k] = 0.0f;
    if (!kTight) weight(i);
  }
  RowRaw<G, V, TPR, CH> next_dy;
  RowRaw<T, V, TPR, CH> next_x;
  float next_mu = 0.0f, next_r = 0.0f;
  auto fetch = [&](int64_t row) {
    next_dy.load(dy + row * cols, cols, t);
    next_x.load(x + row * cols, cols, t);
    next_mu = a.mean[row];
    next_r = a.rstd[row];
  };
  int64_t row = (int64_t)blockIdx.x * R + (TPR > kWave ? 0 : threadIdx.x / TPR);
  const int64_t step = (int64_t)gridDim.x * R;
  if (!kTight && row < rows) fetch(row);
  for (int phase = 0; row < rows; row += step, phase ^= 1) {
    if (kTight) fetch(row);
    const RowRaw<G, V, TPR, CH> cdy = next_dy;
    const RowRaw<T, V, TPR, CH> cx = next_x;
    const float mu = next_mu, r = next_r;
    if (!kTight && row + step < rows) fetch(row + step);
    float s[2] = {0.0f, 0.0f}, xh[CH][V], d[CH][V];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t left = cols - (int64_t)(i * TPR + t) * V;
      if (kTight) weight(i);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        xh[i][k] = k < left ? (cx.get(i, k) - mu) * r : 0.0f;
        const float dyk = cdy.get(i, k);
        dg[i][k] = fmaf(dyk, xh[i][k], dg[i][k]);
        db[i][k] += dyk;
        d[i][k] = dyk * g[i][k];
        s[0] += d[i][k];
        s[1] = fmaf(d[i][k], xh[i][k], s[1]);
      }
    }
    row_sum<TPR, 2>(s, red[phase]);
    const float m1 = s[0] * inv, m2 = s[1] * inv;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t c = (int64_t)(i * TPR + t) * V;
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = r * (d[i][k] - m1 - xh[i][k] * m2);
      store_row<V>(dx + row * cols + c, cols - c, v);
    }
  }
  float* const mine = a.partial + (int64_t)blockIdx.x * 2 * cols;
  if constexpr (TPR > kWave) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t c = (int64_t)(i * TPR + t) * V;
      store_row<V>(mine + c, cols - c, dg[i]);
      store_row<V>(mine + cols + c, cols - c, db[i]);
    }
  } else {
    // the waves' sums meet in LDS
    __shared__ float part[R][TPR * CH * V];
    const int wave = threadIdx.x / TPR;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (which) __syncthreads();
#pragma unroll
      for (int i = 0; i < CH; ++i)
        store_pack(&part[wave][(i * TPR + t) * V], which ? db[i] : dg[i]);
      __syncthreads();
      for (int64_t c = threadIdx.x; c < cols; c += 256) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < R; ++w) s += part[w][c];
        mine[which * cols + c] = s;
      }
    }
  }
}

// Rows wider than registers hold: read twice, the sums over rows kept in the workspace.
template <typename G, typename T>
__global__ __launch_bounds__(1024) void layernorm_bwd_wide_kernel(const G* dy, const T* __restrict__ x, BwdArgs a,
                                                                  G* dx) {
  constexpr int V = kPack<G, T>, TPR = 1024;
  __shared__ float red[2][TPR / kWave][2];
  const int64_t cols = a.cols;
  const float inv = 1.0f / (float)cols;
  float* const mine = a.partial + (int64_t)blockIdx.x * 2 * cols;
  bool first = true;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, first = false) {
    const float mu = a.mean[row], r = a.rstd[row];
    const G* const src = dy + row * cols;
    float s[2] = {0.0f, 0.0f}, v[V], w[V], g[V];
    for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
      load_row<V>(src + c, cols - c, v);
      load_row<V>(x + row * cols + c, cols - c, w);
      if (a.gamma) load_row<V>(a.gamma + c, cols - c, g);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = a.gamma ? v[k] * g[k] : v[k], xh = k < cols - c ? (w[k] - mu) * r : 0.0f;
        s[0] += d;
        s[1] = fmaf(d, xh, s[1]);
      }
    }
    row_sum<TPR, 2>(s, red[row / gridDim.x & 1]);
    const float m1 = s[0] * inv, m2 = s[1] * inv;
    for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
      float dg[V], db[V];
      load_row<V>(src + c, cols - c, v);
      load_row<V>(x + row * cols + c, cols - c, w);
      if (a.gamma) load_row<V>(a.gamma + c, cols - c, g);
      if (!first) {
        load_row<V>(mine + c, cols - c, dg);
        load_row<V>(mine + cols + c, cols - c, db);
      }
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = a.gamma ? v[k] * g[k] : v[k], xh = (w[k] - mu) * r;
        dg[k] = first ? v[k] * xh : fmaf(v[k], xh, dg[k]);
        db[k] = first ? v[k] : db[k] + v[k];
        v[k] = r * (d - m1 - xh * m2);
      }
      store_row<V>(mine + c, cols - c, dg);
      store_row<V>(mine + cols + c, cols - c, db);
      store_row<V>(dx + row * cols + c, cols - c, v);
    }
  }
}

// dgamma and dbeta (blockIdx.y) from the workgroups' sums: 64 columns a block, its 16 waves
// every 16th workgroup's sums, 8 of them in flight.
__global__ __launch_bounds__(1024) void layernorm_weight_kernel(const float* __restrict__ partial, int64_t parts,
                                                                int64_t cols, float* dgamma, float* dbeta) {
  __shared__ float red[16][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t c = (int64_t)blockIdx.x * kWave + lane;
  float* const out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  constexpr int U = 8;
  float s = 0.0f;
  const float* const src = partial + blockIdx.y * cols + c;
  if (c < cols)
    for (int64_t p = wave; p < parts; p += 16 * U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = p + 16 * u < parts ? src[(p + 16 * u) * 2 * cols] : 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) s += v[u];
    }
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) {
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += red[w][lane];
    out[c] = s;
  }
}

// Threads per row and packs per thread for rows of `packs` packs, at most `most` packs a
// thread: a wave's where that does, then workgroups of 256, 512 and 1024.  {0, 0}: too wide.
struct RowShape {
  int tpr, packs;
};
RowShape row_shape(int64_t packs, int most, bool few) {
  for (int tpr : {64, 256, 512, 1024}) {
    // few rows: one pack a thread as far as that goes
    const int cap = few && tpr < 1024 ? 1 : most;
    for (int n = 1; n <= cap; n *= 2)
      if (packs <= (int64_t)tpr * n) return {tpr, n};
  }
  return {0, 0};
}

constexpr int kCuCount = 256;

// Calls f with the shape's compile-time constants.
template <int MOST, typename F>
void with_shape(RowShape s, F f) {
  auto packs = [&](auto tpr) {
    switch (s.packs) {
      case 1: f(tpr, std::integral_constant<int, 1>{}); break;
      case 2: f(tpr, std::integral_constant<int, 2>{}); break;
      default:
        if constexpr (MOST >= 4) f(tpr, std::integral_constant<int, 4>{});
    }
  };
  switch (s.tpr) {
    case 64: packs(std::integral_constant<int, 64>{}); break;
    case 256: packs(std::integral_constant<int, 256>{}); break;
    case 512: packs(std::integral_constant<int, 512>{}); break;
    default: packs(std::integral_constant<int, 1024>{}); break;
  }
}

// Elements a thread holds: the forward needs the row twice and two weights (32 elements
// would be 160 registers), the backward the row twice, two weight sums and the weight.
constexpr int kElements = 16;

int64_t bwd_groups(int64_t rows, int64_t cols) {
  const int64_t at_once = cols <= 64 * kElements ? 4 : 1;
  const int64_t need = (rows + at_once - 1) / at_once;
  return need < 2 * kCuCount ? need : 2 * kCuCount;
}

}  // namespace

hipError_t launch_layernorm_fwd(const void* x, int bf16, int64_t rows, int64_t cols, const float* gamma,
                                const float* beta, float eps, void* y, float* mean, float* rstd, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  auto launch = [&](auto elem) {
    using T = decltype(elem);
    constexpr int V = kPack<T, T>;
    const RowShape s = row_shape((cols + V - 1) / V, kElements / V, rows < 2 * kCuCount);
    auto go = [&](auto kernel, int threads, int64_t at_once) {
      const int64_t need = (rows + at_once - 1) / at_once, most = 8 * kCuCount;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(need < most ? need : most)), dim3(threads), 0, st,
                         static_cast<const T*>(x), rows, cols, gamma, beta, eps, static_cast<T*>(y), mean, rstd);
    };
    if (s.tpr == 0) go(layernorm_fwd_wide_kernel<T>, 1024, 1);
    else
      with_shape<kElements / V>(s, [&](auto tpr, auto packs) {
        constexpr int TPR = decltype(tpr)::value;
        go(layernorm_fwd_kernel<T, TPR, decltype(packs)::value>, kThreads<TPR>, kRowsAtOnce<TPR>);
      });
  };
  bf16 ? launch(uint16_t{}) : launch(float{});
  return hipGetLastError();
}

size_t layernorm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  return (size_t)bwd_groups(rows, cols) * 2 * (size_t)cols * sizeof(float);
}

hipError_t launch_layernorm_bwd(const void* dy, int g_bf16, const void* x, int bf16, const float* mean,
                                const float* rstd, const float* gamma, int64_t rows, int64_t cols, void* dx,
                                float* dgamma, float* dbeta, void* ws, hipStream_t st) {
  const BwdArgs a{mean, rstd, gamma, rows, cols, static_cast<float*>(ws)};
  const int64_t groups = bwd_groups(rows, cols);
  auto launch = [&](auto grad, auto elem) {
    using G = decltype(grad);
    using T = decltype(elem);
    constexpr int V = kPack<G, T>;
    const RowShape s = row_shape((cols + V - 1) / V, kElements / V, false);
    auto go = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), 0, st, static_cast<const G*>(dy),
                         static_cast<const T*>(x), a, static_cast<G*>(dx));
    };
    if (s.tpr == 0) go(layernorm_bwd_wide_kernel<G, T>, 1024);
    else
      with_shape<kElements / V>(s, [&](auto tpr, auto packs) {
        constexpr int TPR = decltype(tpr)::value;
        go(layernorm_bwd_kernel<G, T, TPR, decltype(packs)::value>, kThreads<TPR>);
      });
  };
  if (rows > 0) {
    if (g_bf16) bf16 ? launch(uint16_t{}, uint16_t{}) : launch(uint16_t{}, float{});
    else bf16 ? launch(float{}, uint16_t{}) : launch(float{}, float{});
  }
  if (dgamma || dbeta)
    hipLaunchKernelGGL(layernorm_weight_kernel, dim3((unsigned)((cols + kWave - 1) / kWave), 2), dim3(1024), 0, st,
                       a.partial, groups, cols, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace luq
