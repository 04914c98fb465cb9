// Internal launchers behind the C ABI (host side).  Arguments are already
// validated by the ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace luq {

// Sample-count argument meaning two SMP samples stored as one int8 sum per
// element (LUQ_SMP_SUM | 2 in the C ABI).
constexpr int kSmpSum = 0x12;

// ceil(n/2) rounded up to 256 bytes: the distance between SMP planes.
inline size_t plane_bytes(int64_t n) {
  const size_t b = (size_t)((n + 1) / 2);
  return (b + 255) & ~(size_t)255;
}

size_t quant_workspace_bytes(int64_t n);
// Byte offset, in a quantizer's workspace, of the status word of its last
// call: kStatusTag | luq_status, so that a word no quantizer wrote is told
// apart.
size_t quant_status_offset();
constexpr uint32_t kStatusTag = 0x4C510000u;
constexpr uint32_t kStatusTagMask = 0xFFFF0000u;

hipError_t launch_luq_quantize(const void* g, int bf16, int64_t rows, int64_t cols, int R, int pw2,
                               uint64_t seed, uint32_t counter, int ns, uint8_t* codes,
                               uint8_t* codes_t, float* alpha, float* maxabs, void* ws,
                               hipStream_t st);

// luq_quantize_grad with its workspace in the library's per-device static
// scratch array (no allocation); noalloc_scratch_bytes() is that array's size.
size_t noalloc_scratch_bytes();
hipError_t launch_luq_quantize_noalloc(const void* g, int bf16, int64_t rows, int64_t cols, int R, int pw2,
                                       uint64_t seed, uint32_t counter, int ns, uint8_t* codes, uint8_t* codes_t,
                                       float* alpha, float* maxabs, hipStream_t st);

hipError_t launch_luq_quantize_hindsight(const void* g, int bf16, int64_t rows, int64_t cols, int R, int pw2,
                                         uint64_t seed, uint32_t counter, int ns, float eta, uint8_t* codes,
                                         uint8_t* codes_t, float* state, float* alpha, float* maxabs, void* ws,
                                         hipStream_t st);

hipError_t launch_int4_quantize(const void* x, int bf16, int64_t rows, int64_t cols, int is_signed,
                                float clip, uint8_t* codes, uint8_t* codes_t, float* scale,
                                void* ws, hipStream_t st);

// C[m][n] = (alpha / ns) * bscale * sum_k A[m][k] * B[n][k] with A LUQ codes
// (ns planes, plane stride a_plane) and B INT4 codes, both K-major.
size_t gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int ns);
hipError_t launch_gemm_luq_int4(const uint8_t* A, int64_t a_plane, int ns, const float* alpha,
                                const uint8_t* B, const float* bscale, int b_signed, int64_t M,
                                int64_t N, int64_t K, float* C, void* ws, size_t ws_bytes,
                                hipStream_t st);

// The same product on the FP6 carrier (one sample): the codes are converted
// once into fragment-major FP6 blocks in the workspace, then multiplied with
// the scaled f8f6f4 MFMA; bit-identical to launch_gemm_luq_int4.
constexpr int kCarrierFp6 = 0x40;
size_t gemm_fp6_workspace_bytes(int64_t M, int64_t N, int64_t K);
bool gemm_fp6_fits(int64_t M, int64_t N, int64_t K);
hipError_t launch_gemm_luq_int4_fp6(const uint8_t* A, const float* alpha, const uint8_t* B, const float* bscale,
                                    int b_signed, int64_t M, int64_t N, int64_t K, float* C, void* ws,
                                    hipStream_t st);

// y[m][n] = x_scale * w_scale * sum_k X[m][k] * W[n][k], INT4 codes, K-major.
size_t gemm_fwd_workspace_bytes(int64_t M, int64_t N, int64_t K);
hipError_t launch_gemm_int4_fwd(const uint8_t* X, const float* x_scale, int x_signed, const uint8_t* W,
                                const float* w_scale, int w_signed, int64_t M, int64_t N, int64_t K, float* Y,
                                void* ws, hipStream_t st);

// dact[t][c] of a 3x3 / stride 1 / pad 1 convolution from LUQ codes of g
// [T][Cout] (ns planes) and INT4 codes of W transposed [9*C][Cout].
int conv3x3_max_width();
hipError_t launch_conv3x3_dgrad(const uint8_t* g, int64_t g_plane, int ns, const float* alpha, const uint8_t* w,
                                const float* wscale, int w_signed, int64_t B, int64_t H, int64_t W, int64_t C,
                                int64_t Cout, float* dact, hipStream_t st);

// dW [Cout][9*C] of the same convolution from LUQ codes of g transposed
// [Cout][T] (ns planes) and INT4 codes of the activations transposed [C][T].
size_t conv3x3_wgrad_workspace_bytes(int64_t T, int64_t C, int64_t Cout);
int64_t conv3x3_wgrad_blocks(int64_t T, int64_t C, int64_t Cout);
hipError_t launch_conv3x3_wgrad(const uint8_t* g, int64_t g_plane, int ns, const float* alpha, const uint8_t* act,
                                const float* ascale, int a_signed, int64_t B, int64_t H, int64_t W, int64_t C,
                                int64_t Cout, float* dw, void* ws, hipStream_t st);

// Operators of luq_lm.h.
size_t group_ids_workspace_bytes(int64_t n, int64_t groups);
hipError_t launch_group_ids(const void* ids, int i64, int64_t n, int64_t groups, int32_t* order, int32_t* offsets,
                            void* ws, hipStream_t st);

hipError_t launch_embedding_fwd(const void* ids, int i64, int64_t n, const void* table, int t_bf16, int64_t vocab,
                                int64_t dim, float scale, void* out, int o_bf16, hipStream_t st);
size_t embedding_grad_workspace_bytes(int64_t n, int64_t dim);
hipError_t launch_embedding_grad(const void* dout, int g_bf16, const void* ids, int i64, const int32_t* order,
                                 const int32_t* offsets, int64_t n, int64_t vocab, int64_t dim, float scale,
                                 int accumulate, float* dtable, void* ws, hipStream_t st);

hipError_t launch_layernorm_fwd(const void* x, int bf16, int64_t rows, int64_t cols, const float* gamma,
                                const float* beta, float eps, void* y, float* mean, float* rstd, hipStream_t st);
size_t layernorm_bwd_workspace_bytes(int64_t rows, int64_t cols);
hipError_t launch_layernorm_bwd(const void* dy, int g_bf16, const void* x, int bf16, const float* mean,
                                const float* rstd, const float* gamma, int64_t rows, int64_t cols, void* dx,
                                float* dgamma, float* dbeta, void* ws, hipStream_t st);

// Products grouped by expert; the A operand's codes.
enum class GroupedA { kLuq, kSums, kInt4S, kInt4U };
// Sizes whose outputs and grid are not too large.
bool grouped_rows_fit(int64_t T, int64_t N, int64_t experts);
// C [T][N], the rows grouped; w_row and w_expert in codes.
hipError_t launch_grouped_rows(GroupedA kind, const uint8_t* A, const float* alpha, const uint8_t* B, int64_t w_row,
                               int64_t w_expert, const float* bscale, int64_t scales, int b_signed,
                               const int32_t* offsets, int64_t experts, int64_t T, int64_t N, int64_t K, float* C,
                               hipStream_t st);
// C [experts][M][N], the reduction over T grouped.  Beyond the int32-exact length the
// reduction is split, and whole stages are asked for.
bool grouped_depth_fits(int64_t T, int64_t M, int64_t N, int64_t experts);
size_t grouped_depth_workspace_bytes(int64_t T, int64_t M, int64_t N, int64_t experts);
hipError_t launch_grouped_depth(GroupedA kind, const uint8_t* A, const float* alpha, const uint8_t* B,
                                const float* bscale, int b_signed, const int32_t* offsets, int64_t experts, int64_t T,
                                int64_t M, int64_t N, float* C, void* ws, hipStream_t st);

// Choice of experts.
struct RouteArgs {
  const void* logits;
  const float* bias;
  int64_t T;
  int E, K, groups, top_groups, best, renorm, sigmoid;
  float scale;
};
hipError_t launch_route_fwd(const RouteArgs& a, int bf16, int32_t* chosen, float* weights, hipStream_t st);
hipError_t launch_route_bwd(const RouteArgs& a, int bf16, const float* dweights, const int32_t* chosen, void* dlogits,
                            hipStream_t st);

// Cross entropy of the last layer.
struct CrossEntropyArgs {
  const void* x;
  const void* table;
  const void* targets;
  int x_bf16, t_bf16, i64;
  int64_t T, V, D;
  float scale, smoothing;
};
// Bytes of the workspace; backward: with a gradient of the table in bf16 (g_bf16) or fp32.
size_t cross_entropy_fwd_workspace_bytes(int64_t T, int64_t V, int64_t D, int x_bf16, int t_bf16);
size_t cross_entropy_bwd_workspace_bytes(int64_t T, int64_t V, int64_t D, int x_bf16, int t_bf16, int g_bf16);
hipError_t launch_cross_entropy_fwd(const CrossEntropyArgs& a, float* loss, float* lse, void* ws, hipStream_t st);
hipError_t launch_cross_entropy_bwd(const CrossEntropyArgs& a, const float* dloss, const float* lse, int accumulate,
                                    void* dx, void* dtable, int g_bf16, void* ws, hipStream_t st);

// A plan of AdamW: an entry for each tensor, then its chunks of elements.
constexpr int kAdamwChunk = 4096;
struct AdamwEntry {
  float* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  uint16_t* copy;
  int64_t n;
  float weight_decay, lr_scale;
  int g_bf16, state_bits;
};
struct AdamwChunk {
  uint32_t tensor, index;
};
hipError_t launch_adamw(const void* plan, int64_t count, int64_t chunks, const float* lr, const int64_t* step,
                        double beta1, double beta2, float eps, const float* grad_scale, uint64_t seed, hipStream_t st);

hipError_t launch_im2col3x3_t(const uint8_t* act, int64_t B, int64_t H, int64_t W, int64_t C,
                              uint8_t* col_t, hipStream_t st);

}  // namespace luq
