// Layer norm, forward and backward.
//
//   y = (x - mean) * rstd * gamma + beta,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   with xh = (x - mean) * rstd and a = dy * gamma:
//   dx = rstd * (a - mean(a) - xh * mean(a * xh)),  dgamma = sum dy * xh,  dbeta = sum dy
//
// Bound by memory: the forward reads and writes a row once (8192 x 4096 fp32: 49 us, 5.5
// TB/s), the backward reads two and writes one (16384 x 4096 bf16: 80 us, 5.0 TB/s).  A row stays in registers between its sums and its output, spread over a wave
// or a workgroup; a workgroup takes several rows, the next one's loads in flight while one
// is reduced, and keeps the weights (and the sums of their gradients) in registers for all
// of them.  Wider rows than registers hold are read again instead.
//
// Statistics and sums are fp32; the variance is taken from the differences to the mean, so
// that rows far from zero keep their digits.  A mean that is large against these differences
// is corrected by their sum: the row's sum and its product with 1 / cols are off by some units
// in the last place, which rstd = 1 / sqrt(eps) made 0.5 of a row of -30000 throughout (1000
// columns).  A branch of its own: not taken it costs 200000 x 64 fp32 0.7 of 36 us and 2048 x
// 12000 bf16 1.2 of 28.6, a second sum for all rows 4 and 2.7.
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

// Where a thread's CH packs of a row lie: pack i of thread t begins at column (i * TPR + t) * V.
template <int V, int TPR, int CH>
struct RowAt {
  PackAt<V> at[CH];
  __device__ __forceinline__ RowAt(int t, int64_t cols) {
#pragma unroll
    for (int i = 0; i < CH; ++i) at[i] = PackAt<V>((i * TPR + t) * V, (int)cols);
  }
};

template <typename T, int V, int TPR, int CH>
struct RowRaw {
  RowPack<T, V> pack[CH];
  __device__ __forceinline__ void load(const T* row, const RowAt<V, TPR, CH>& col) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (col.at[i].any()) pack[i].load(row + col.at[i].begin);
  }
  __device__ __forceinline__ float get(int i, int k) const { return pack[i].get(k); }
};

// An fp32 vector over the columns, or a constant for NULL.
template <int V, int TPR, int CH>
__device__ __forceinline__ void load_vector(const float* p, float none, const RowAt<V, TPR, CH>& col, float (&v)[CH][V]) {
#pragma unroll
  for (int i = 0; i < CH; ++i) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[i][k] = none;
    if (p && col.at[i].any()) load_pack(p + col.at[i].begin, v[i]);
  }
}

// Whether a row's mean, off by some units in its last place, is off by much of its spread.
// The row's threads agree: they hold the same sums.
__device__ __forceinline__ bool far_from_zero(float mean, float var) { return mean * mean > 64.0f * var; }

// The mean and the variance from the sum of the differences to a first mean.
__device__ __forceinline__ void correct_mean(float& mean, float& var, float off) {
  mean += off;
  var = fmaxf(fmaf(-off, off, var), 0.0f);
}

template <typename T, int TPR, int CH>
__global__ __launch_bounds__(kThreads<TPR>) void layernorm_fwd_kernel(const T* x, int64_t rows, int64_t cols,
                                                                      const float* __restrict__ gamma,
                                                                      const float* __restrict__ beta, float eps, T* y,
                                                                      float* __restrict__ mean,
                                                                      float* __restrict__ rstd) {
  constexpr int V = kPack<T, T>, R = kRowsAtOnce<TPR>;
  __shared__ float red1[TPR / kWave][1], red2[TPR / kWave][1], red3[TPR / kWave][1];
  const int t = threadIdx.x & (TPR - 1);
  const float inv = 1.0f / (float)cols;
  const RowAt<V, TPR, CH> col(t, cols);
  float g[CH][V], b[CH][V];
  load_vector(gamma, 1.0f, col, g);
  load_vector(beta, 0.0f, col, b);
  RowRaw<T, V, TPR, CH> next;
  int64_t row = (int64_t)blockIdx.x * R + (TPR > kWave ? 0 : threadIdx.x / TPR);
  const int64_t step = (int64_t)gridDim.x * R;
  if (row < rows) next.load(x + row * cols, col);
  for (; row < rows; row += step) {
    const RowRaw<T, V, TPR, CH> cur = next;
    if (row + step < rows) next.load(x + (row + step) * cols, col);
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) s[0] += col.at[i].own(k) ? cur.get(i, k) : 0.0f;
    row_sum<TPR, 1>(s, red1);
    float mu = s[0] * inv;
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = col.at[i].own(k) ? cur.get(i, k) - mu : 0.0f;
        q[0] = fmaf(d, d, q[0]);
      }
    row_sum<TPR, 1>(q, red2);
    float var = q[0] * inv;
    if (far_from_zero(mu, var)) {
      s[0] = 0.0f;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k) s[0] += col.at[i].own(k) ? cur.get(i, k) - mu : 0.0f;
      row_sum<TPR, 1>(s, red3);
      correct_mean(mu, var, s[0] * inv);
    }
    const float r = 1.0f / sqrtf(var + eps);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = fmaf((cur.get(i, k) - mu) * r, g[i][k], b[i][k]);
      if (col.at[i].any()) store_pack(y + row * cols + col.at[i].begin, v);
    }
    if (t == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = r;
    }
  }
}

// Rows wider than registers hold, and those narrower than a pack: read three times (from L2
// after the first).
template <typename T>
__global__ __launch_bounds__(1024) void layernorm_fwd_wide_kernel(const T* x, int64_t rows, int64_t cols,
                                                                  const float* __restrict__ gamma,
                                                                  const float* __restrict__ beta, float eps, T* y,
                                                                  float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int V = kPack<T, T>, TPR = 1024;
  __shared__ float red1[TPR / kWave][1], red2[TPR / kWave][1], red3[TPR / kWave][1];
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
    float mu = s[0] * inv;
    for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
      load_row<V>(src + c, cols - c, v);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = k < cols - c ? v[k] - mu : 0.0f;
        q[0] = fmaf(d, d, q[0]);
      }
    }
    row_sum<TPR, 1>(q, red2);
    float var = q[0] * inv;
    if (far_from_zero(mu, var)) {
      s[0] = 0.0f;
      for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
        load_row<V>(src + c, cols - c, v);
#pragma unroll
        for (int k = 0; k < V; ++k) s[0] += k < cols - c ? v[k] - mu : 0.0f;
      }
      row_sum<TPR, 1>(s, red3);
      correct_mean(mu, var, s[0] * inv);
    }
    const float r = 1.0f / sqrtf(var + eps);
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
  float* dgamma;    // where a single workgroup's sums go instead; either may be null
  float* dbeta;
  __device__ __forceinline__ float* sums(int64_t group, int64_t groups, int which) const {
    return groups == 1 ? (which ? dbeta : dgamma) : partial + (2 * group + which) * cols;
  }
};

template <typename G, typename T, int TPR, int CH>
__global__ __launch_bounds__(kThreads<TPR>) void layernorm_bwd_kernel(const G* dy, const T* __restrict__ x, BwdArgs a,
                                                                      G* dx) {
  constexpr int V = kPack<G, T>, R = kRowsAtOnce<TPR>;
  __shared__ float red[2][TPR / kWave][2];
  const int t = threadIdx.x & (TPR - 1);
  const int64_t rows = a.rows, cols = a.cols;
  const float inv = 1.0f / (float)cols;
  const RowAt<V, TPR, CH> col(t, cols);
  float g[CH][V], dg[CH][V], db[CH][V];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) dg[i][k] = db[i][k] = 0.0f;
  load_vector(a.gamma, 1.0f, col, g);
  RowRaw<G, V, TPR, CH> next_dy;
  RowRaw<T, V, TPR, CH> next_x;
  float next_mu = 0.0f, next_r = 0.0f;
  auto fetch = [&](int64_t row) {
    next_dy.load(dy + row * cols, col);
    next_x.load(x + row * cols, col);
    next_mu = a.mean[row];
    next_r = a.rstd[row];
  };
  int64_t row = (int64_t)blockIdx.x * R + (TPR > kWave ? 0 : threadIdx.x / TPR);
  const int64_t step = (int64_t)gridDim.x * R;
  if (row < rows) fetch(row);
  for (int phase = 0; row < rows; row += step, phase ^= 1) {
    const RowRaw<G, V, TPR, CH> cdy = next_dy;
    const RowRaw<T, V, TPR, CH> cx = next_x;
    const float mu = next_mu, r = next_r;
    if (row + step < rows) fetch(row + step);
    float s[2] = {0.0f, 0.0f}, xh[CH][V], d[CH][V];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        xh[i][k] = (cx.get(i, k) - mu) * r;
        const float dyk = cdy.get(i, k);
        dg[i][k] = fmaf(dyk, xh[i][k], dg[i][k]);
        db[i][k] += dyk;
        d[i][k] = dyk * g[i][k];
        const float own = col.at[i].own(k) ? d[i][k] : 0.0f;
        s[0] += own;
        s[1] = col.at[i].own(k) ? fmaf(own, xh[i][k], s[1]) : s[1];
      }
    row_sum<TPR, 2>(s, red[phase]);
    const float m1 = s[0] * inv, m2 = s[1] * inv;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = r * (d[i][k] - m1 - xh[i][k] * m2);
      if (col.at[i].any()) store_pack(dx + row * cols + col.at[i].begin, v);
    }
  }
  if constexpr (TPR > kWave) {
    float* const sum_g = a.sums(blockIdx.x, gridDim.x, 0);
    float* const sum_b = a.sums(blockIdx.x, gridDim.x, 1);
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (col.at[i].any()) {
        if (sum_g) store_pack(sum_g + col.at[i].begin, dg[i]);
        if (sum_b) store_pack(sum_b + col.at[i].begin, db[i]);
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
        if (col.at[i].any()) store_pack(&part[wave][col.at[i].begin], which ? db[i] : dg[i]);
      __syncthreads();
      float* const mine = a.sums(blockIdx.x, gridDim.x, which);
      if (mine)
        for (int64_t c = threadIdx.x; c < cols; c += 256) {
          float s = 0.0f;
#pragma unroll
          for (int w = 0; w < R; ++w) s += part[w][c];
          mine[c] = s;
        }
    }
  }
}

// ---- backward of rows of fewer than kNarrow columns: a thread a row
//
// With a column a thread 128 workgroups kept 5 threads each of 200000 x 5 busy, and each added
// 1600 terms in a row (bf16 1611 us a call, 15 now; 4 x 4 fp32 4.4 and 5.0).

constexpr int kNarrow = 8, kNarrowThreads = 256;

template <typename G, typename T>
__global__ __launch_bounds__(kNarrowThreads) void layernorm_narrow_bwd_kernel(const G* dy, const T* __restrict__ x,
                                                                              BwdArgs a, G* dx) {
  constexpr int N = kNarrow - 1, W = kNarrowThreads / kWave;
  __shared__ float red[2][N][W];
  const int cols = (int)a.cols;
  const float inv = 1.0f / (float)cols;
  float g[N], sum[2][N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    g[k] = a.gamma && k < cols ? a.gamma[k] : 1.0f;
    sum[0][k] = sum[1][k] = 0.0f;
  }
  for (int64_t row = (int64_t)blockIdx.x * kNarrowThreads + threadIdx.x; row < a.rows;
       row += (int64_t)gridDim.x * kNarrowThreads) {
    const float mu = a.mean[row], r = a.rstd[row];
    float d[N], xh[N], m1 = 0.0f, m2 = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float dyk = k < cols ? to_f32(dy[row * cols + k]) : 0.0f;
      xh[k] = k < cols ? (to_f32(x[row * cols + k]) - mu) * r : 0.0f;
      sum[0][k] = fmaf(dyk, xh[k], sum[0][k]);
      sum[1][k] += dyk;
      d[k] = dyk * g[k];
      m1 += d[k];
      m2 = fmaf(d[k], xh[k], m2);
    }
    m1 *= inv;
    m2 *= inv;
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < cols) dx[row * cols + k] = from_f32<G>(r * (d[k] - m1 - xh[k] * m2));
  }
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float s = wave_sum(sum[which][k]);
      if ((threadIdx.x & (kWave - 1)) == 0) red[which][k][threadIdx.x / kWave] = s;
    }
  __syncthreads();
  const int which = threadIdx.x / kWave, k = threadIdx.x & (kWave - 1);
  if (which < 2 && k < cols) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) s += red[which][k][w];
    float* const out = a.sums(blockIdx.x, gridDim.x, which);
    if (out) out[k] = s;
  }
}

// ---- backward of wide rows: read twice

// A row's two means, by a workgroup.
template <typename G, typename T>
__global__ __launch_bounds__(1024) void layernorm_means_kernel(const G* __restrict__ dy, const T* __restrict__ x,
                                                               BwdArgs a, float2* __restrict__ means) {
  constexpr int V = kPack<G, T>, TPR = 1024;
  __shared__ float red[2][TPR / kWave][2];
  const int64_t cols = a.cols;
  int phase = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, phase ^= 1) {
    const float mu = a.mean[row], r = a.rstd[row];
    float s[2] = {0.0f, 0.0f}, v[V], w[V], g[V];
    for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += TPR * V) {
      load_row<V>(dy + row * cols + c, cols - c, v);
      load_row<V>(x + row * cols + c, cols - c, w);
      if (a.gamma) load_row<V>(a.gamma + c, cols - c, g);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = a.gamma ? v[k] * g[k] : v[k], xh = k < cols - c ? (w[k] - mu) * r : 0.0f;
        s[0] += d;
        s[1] = fmaf(d, xh, s[1]);
      }
    }
    row_sum<TPR, 2>(s, red[phase]);
    if (threadIdx.x == 0) means[row] = make_float2(s[0] / (float)cols, s[1] / (float)cols);
  }
}

// dx and the sums over rows: a thread keeps one pack of columns and walks the rows
// blockIdx.y, blockIdx.y + gridDim.y, .. with four of them in flight.  Elements that two packs share are stored by the one before only: where dx is
// dy, the other may have read them too late.
template <typename G, typename T>
__global__ __launch_bounds__(256) void layernorm_slab_kernel(const G* dy, const T* __restrict__ x, BwdArgs a,
                                                             const float2* __restrict__ means, G* dx) {
  constexpr int V = kPack<G, T>, U = 4;
  const int64_t cols = a.cols, step = gridDim.y;
  const PackAt<V> at(((int)blockIdx.x * 256 + (int)threadIdx.x) * V, (int)cols);
  if (!at.any()) return;
  float g[V], dg[V], db[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    g[k] = 1.0f;
    dg[k] = db[k] = 0.0f;
  }
  if (a.gamma) load_pack(a.gamma + at.begin, g);
  for (int64_t row0 = blockIdx.y; row0 < a.rows; row0 += U * step) {
    RowPack<G, V> pdy[U];
    RowPack<T, V> px[U];
    float mu[U], r[U];
    float2 m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = min(row0 + u * step, a.rows - 1);
      pdy[u].load(dy + row * cols + at.begin);
      px[u].load(x + row * cols + at.begin);
      mu[u] = a.mean[row];
      r[u] = a.rstd[row];
      m[u] = means[row];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = row0 + u * step;
      if (row >= a.rows) break;
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float dyk = pdy[u].get(k), xh = (px[u].get(k) - mu[u]) * r[u];
        dg[k] = fmaf(dyk, xh, dg[k]);
        db[k] += dyk;
        v[k] = r[u] * (dyk * g[k] - m[u].x - xh * m[u].y);
      }
      G* const dst = dx + row * cols + at.begin;
      if (at.shared == 0) {
        store_pack(dst, v);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (at.own(k)) dst[k] = from_f32<G>(v[k]);
      }
    }
  }
  float* const sum_g = a.sums(blockIdx.y, gridDim.y, 0);
  float* const sum_b = a.sums(blockIdx.y, gridDim.y, 1);
#pragma unroll
  for (int k = 0; k < V; ++k)
    if (at.own(k)) {
      if (sum_g) sum_g[at.begin + k] = dg[k];
      if (sum_b) sum_b[at.begin + k] = db[k];
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
// thread: a wave's where that does, then workgroups of 256 threads and more.  {0, 0}: too
// wide, or (forward) narrower than a pack.
struct RowShape {
  int tpr, packs;
};
RowShape row_shape(int64_t cols, int pack, int most, int most_threads, bool few) {
  const int64_t packs = (cols + pack - 1) / pack;
  if (cols < pack) return {0, 0};
  for (int tpr = 64; tpr <= most_threads; tpr *= tpr == 64 ? 4 : 2) {
    // few rows: one pack a thread as far as that goes
    const int cap = few && tpr < most_threads ? 1 : most;
    for (int n = 1; n <= cap; n *= 2)
      if (packs <= (int64_t)tpr * n) return {tpr, n};
  }
  return {0, 0};
}

constexpr int kCuCount = 256;

// Calls f with the shape's compile-time constants.
template <int MOST, int THREADS, typename F>
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
    default:
      if constexpr (THREADS >= 1024) packs(std::integral_constant<int, 1024>{});
  }
}

// Elements a thread holds: the forward needs the row twice and two vectors, the backward two
// rows twice, two sums and the weight: 16 are up to 190 registers, which 512 threads have
// (1024 threads spilled 18 to 220 of them: 4096 x 16384 bf16 took 134 us or more in registers, about what
// reading the rows twice takes).
constexpr int kElements = 16, kFwdThreads = 1024, kBwdThreads = 512;
constexpr int64_t kMostCols = kBwdThreads * kElements;   // of the backward in registers

// Workgroups of the backward, each of which leaves a row of sums: one a CU beyond 4096
// columns (8192 x 8192 bf16: 79 to 87 us with one, 79 to 93 with more), two below (16384 x
// 4096: 101 with one, 80 with two, 95 with four), and for rows of a wave up to four, but
// three rows a wave at least (65536 x 512: 60, 42, 40 with one, two, four; 3001 x 1024:
// 13.7, 15.6, 18.1).  A single workgroup writes the gradients itself, without the second
// launch, and takes 4 rows (2 x 8000 bf16: 12.0 to 9.1 us a call; 4 x 4096 12.5 to
// 9.5; 8 x 8192 12.0 to 14.4) or, of the form that reads twice, 8 (8 x 100000: 30 to 18).
// Many rows take more workgroups than that, so that no thread adds more than kMostRows terms
// in a row: an fp32 sum of n like terms can be off by n / 2 units of its last place.
constexpr int64_t kMostRows = 4096;
int64_t bwd_groups(int64_t rows, int64_t cols) {
  auto groups = [&](int64_t few, int64_t at_once, int64_t need, int64_t most) {
    if (rows > 0 && rows <= few) return (int64_t)1;
    const int64_t least = (rows + kMostRows * at_once - 1) / (kMostRows * at_once);
    if (most < least) most = least;
    return need < most ? need : most;
  };
  if (cols < kNarrow)
    return groups(kNarrowThreads, kNarrowThreads, (rows + kNarrowThreads - 1) / kNarrowThreads, 4 * kCuCount);
  if (cols > kMostCols) return groups(8, 1, rows, 128);
  if (cols <= 64 * kElements) return groups(4, 4, (rows + 11) / 12, 4 * kCuCount);
  return groups(4, 1, rows, cols > 4096 ? kCuCount : 2 * kCuCount);
}

// Rows' means of the form that reads rows twice, after the sums of the groups.
size_t bwd_sums_bytes(int64_t rows, int64_t cols) {
  return (size_t)bwd_groups(rows, cols) * 2 * (size_t)cols * sizeof(float);
}

}  // namespace

hipError_t launch_layernorm_fwd(const void* x, int bf16, int64_t rows, int64_t cols, const float* gamma,
                                const float* beta, float eps, void* y, float* mean, float* rstd, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  auto launch = [&](auto elem) {
    using T = decltype(elem);
    constexpr int V = kPack<T, T>;
    const RowShape s = row_shape(cols, V, kElements / V, kFwdThreads, rows < 2 * kCuCount);
    auto go = [&](auto kernel, int threads, int64_t at_once) {
      const int64_t need = (rows + at_once - 1) / at_once, most = 8 * kCuCount;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(need < most ? need : most)), dim3(threads), 0, st,
                         static_cast<const T*>(x), rows, cols, gamma, beta, eps, static_cast<T*>(y), mean, rstd);
    };
    if (s.tpr == 0) go(layernorm_fwd_wide_kernel<T>, 1024, 1);
    else
      with_shape<kElements / V, kFwdThreads>(s, [&](auto tpr, auto packs) {
        constexpr int TPR = decltype(tpr)::value;
        go(layernorm_fwd_kernel<T, TPR, decltype(packs)::value>, kThreads<TPR>, kRowsAtOnce<TPR>);
      });
  };
  bf16 ? launch(uint16_t{}) : launch(float{});
  return hipGetLastError();
}

size_t layernorm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  return bwd_sums_bytes(rows, cols) + (cols > kMostCols ? (size_t)rows * sizeof(float2) : 0);
}

hipError_t launch_layernorm_bwd(const void* dy, int g_bf16, const void* x, int bf16, const float* mean,
                                const float* rstd, const float* gamma, int64_t rows, int64_t cols, void* dx,
                                float* dgamma, float* dbeta, void* ws, hipStream_t st) {
  const BwdArgs a{mean, rstd, gamma, rows, cols, static_cast<float*>(ws), dgamma, dbeta};
  const int64_t groups = bwd_groups(rows, cols);
  auto launch = [&](auto grad, auto elem) {
    using G = decltype(grad);
    using T = decltype(elem);
    constexpr int V = kPack<G, T>;
    const RowShape s = row_shape(cols, V, kElements / V, kBwdThreads, false);
    auto go = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), 0, st, static_cast<const G*>(dy),
                         static_cast<const T*>(x), a, static_cast<G*>(dx));
    };
    if (cols < kNarrow) {
      go(layernorm_narrow_bwd_kernel<G, T>, kNarrowThreads);
    } else if (s.tpr == 0) {
      float2* const means = reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + bwd_sums_bytes(rows, cols));
      const int64_t most = 4 * kCuCount;
      hipLaunchKernelGGL((layernorm_means_kernel<G, T>), dim3((unsigned)(rows < most ? rows : most)), dim3(1024), 0, st,
                         static_cast<const G*>(dy), static_cast<const T*>(x), a, means);
      hipLaunchKernelGGL((layernorm_slab_kernel<G, T>), dim3((unsigned)((cols + 256 * V - 1) / (256 * V)), (unsigned)groups),
                         dim3(256), 0, st, static_cast<const G*>(dy), static_cast<const T*>(x), a, means,
                         static_cast<G*>(dx));
    } else
      with_shape<kElements / V, kBwdThreads>(s, [&](auto tpr, auto packs) {
        constexpr int TPR = decltype(tpr)::value;
        go(layernorm_bwd_kernel<G, T, TPR, decltype(packs)::value>, kThreads<TPR>);
      });
  };
  if (rows > 0) {
    if (g_bf16) bf16 ? launch(uint16_t{}, uint16_t{}) : launch(uint16_t{}, float{});
    else bf16 ? launch(float{}, uint16_t{}) : launch(float{}, float{});
  }
  if ((dgamma || dbeta) && groups != 1)
    hipLaunchKernelGGL(layernorm_weight_kernel, dim3((unsigned)((cols + kWave - 1) / kWave), 2), dim3(1024), 0, st,
                       a.partial, groups, cols, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace luq
