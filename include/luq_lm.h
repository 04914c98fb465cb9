/*
 * luq_lm.h -- C ABI of libluq: the operators of a Transformer's training and
 * serving steps around the 4-bit products of luq.h.
 *
 * The paper keeps the first layer and the normalisations in high precision
 * (Appendix A.4); these are the embedding lookup and layer
 * norm below.  Layers of experts take the 4-bit products of Eqs. forward,
 * backward and update on rows grouped by expert, in groups of any sizes.
 * A step of training takes three things more: the choice of experts for
 * every token, the loss of the last layer (kept in high precision as the
 * first), whose table is the embedding's or its own, and the update of the
 * weights.
 *
 * Conventions are those of luq.h (device pointers owned by the caller, work
 * enqueued on `stream`, no synchronisation, argument errors found on the host
 * before anything is enqueued), but for alignment: rows of any width are
 * taken, so tensors only need the alignment of their elements (code operands
 * and workspaces 16 bytes, as there).  Inputs and outputs must not overlap
 * unless stated.  No tensor holds more than 2^38 elements.
 */
#ifndef LUQ_LM_H
#define LUQ_LM_H

#include "luq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of a tensor of ids. */
typedef enum { LUQ_I32 = 0, LUQ_I64 = 1 } luq_index;

/*
 * luq_group_ids -- positions grouped by id, in order: a stable sort.
 *
 *  ids      [n] ids.  Ids outside [0, groups) belong to no group.
 *  order    out: [n] int32, the positions 0..n-1 sorted by id, equal ids in
 *           order of position; positions without a group come last, in order.
 *  offsets  out: [groups + 1] int32; group v is order[offsets[v]] ..
 *           order[offsets[v + 1] - 1].  offsets[0] = 0; offsets[groups] is the
 *           number of positions in a group.
 *  n        0 <= n <= 2^28;  groups  1 <= groups <= 2^28.
 *  ws       workspace of luq_workspace_size(LUQ_OP_GROUP_IDS, n, groups).
 *
 * The same result on every call, for any n (no atomics decide an order).  With the
 * ids of a batch and the vocabulary's size it is the order in which
 * luq_embedding_grad reads the gradient; with the expert of every routed row and
 * the number of experts, offsets are what the grouped products take, and order is
 * the ids with which luq_embedding_fwd gathers the rows.
 * Errors: LUQ_ERR_SHAPE, LUQ_ERR_DTYPE, LUQ_ERR_NULL, LUQ_ERR_WORKSPACE,
 * LUQ_ERR_ALIGN, LUQ_ERR_HIP.
 */
luq_status luq_group_ids(const void* ids, luq_index it, int64_t n, int64_t groups, int32_t* order,
                         int32_t* offsets, void* ws, size_t ws_bytes, void* stream);

/*
 * luq_embedding_fwd -- out[i][:] = scale * table[ids[i]][:]
 *
 *  ids    [n]; an id below 0 is padding and gives a row of zeros, one at or above
 *         vocab is a data error and gives a row of NaN.
 *  table  [vocab][dim], type tt;  out  [n][dim], type ot.  The product is rounded
 *         to fp32, and once more to a bf16 out.
 *  n and vocab in [0, 2^28], dim in [1, 2^23].  No workspace.
 */
luq_status luq_embedding_fwd(const void* ids, luq_index it, int64_t n, const void* table, luq_dtype tt,
                             int64_t vocab, int64_t dim, float scale, void* out, luq_dtype ot, void* stream);

/*
 * luq_embedding_grad -- gradient of luq_embedding_fwd's table:
 *   dtable[v][:] = scale * sum over i with ids[i] = v of dout[i][:]
 * The rows of dout are added in fp32 in the order of their positions, in pieces of a
 * length that depends on n and dim alone: the same result on every call.
 *
 *  dout    [n][dim], type gt.
 *  ids     [n], as in the forward call; ids outside [0, vocab) give no gradient.
 *  order, offsets  of luq_group_ids(ids, n, vocab).
 *  dtable  [vocab][dim] fp32.  accumulate = 0: written whole, zeros in rows that no
 *          id names; 1: the sums are added to the rows that ids name, and no other row
 *          is touched (further batches of one step, a table shared with another layer).
 *  n in [0, 2^28], vocab in [1, 2^28], dim in [1, 2^23].
 *  ws      workspace of luq_workspace_size(LUQ_OP_EMBEDDING_GRAD, n, dim).
 */
luq_status luq_embedding_grad(const void* dout, luq_dtype gt, const void* ids, luq_index it, const int32_t* order,
                              const int32_t* offsets, int64_t n, int64_t vocab, int64_t dim, float scale,
                              int accumulate, float* dtable, void* ws, size_t ws_bytes, void* stream);

/*
 * luq_layernorm_fwd -- layer norm of every row:
 *   mean = sum_j x_j / cols,  var = sum_j (x_j - mean)^2 / cols,
 *   rstd = 1 / sqrt(var + eps),  y_j = (x_j - mean) * rstd * gamma_j + beta_j
 *
 *  x, y         [rows][cols], type dt.  gamma, beta  [cols] fp32, or NULL for 1
 *               and 0.  mean, rstd  out: [rows] fp32, or NULL (serving).
 *  rows in [0, 2^30], cols in [1, 2^23]; eps >= 0 and finite.  Statistics are held in fp32, the
 *  variance from the differences to the mean, and a mean far from zero corrected by their
 *  sum: a row of equal elements gives beta.  y may be x.  No workspace.
 */
luq_status luq_layernorm_fwd(const void* x, luq_dtype dt, int64_t rows, int64_t cols, const float* gamma,
                             const float* beta, float eps, void* y, float* mean, float* rstd, void* stream);

/*
 * luq_layernorm_bwd -- gradients of luq_layernorm_fwd.  With xh = (x - mean) * rstd
 * and a = dy * gamma:
 *   dx = rstd * (a - sum_j a_j / cols - xh * sum_j (a_j xh_j) / cols)
 *   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
 *
 *  dy, dx       [rows][cols], type gt (fp32 gradients of the products, or bf16).
 *  x            [rows][cols], type dt.  mean, rstd  [rows] of the forward call.
 *  gamma        [cols] fp32 or NULL.  dgamma, dbeta  out: [cols] fp32, each may be
 *               NULL; zeros when rows = 0.  dx may be dy.
 *  ws           workspace of luq_workspace_size(LUQ_OP_LAYERNORM_BWD, rows, cols).
 *  Sums over rows are taken in fp32 in a fixed order.
 */
luq_status luq_layernorm_bwd(const void* dy, luq_dtype gt, const void* x, luq_dtype dt, const float* mean,
                             const float* rstd, const float* gamma, int64_t rows, int64_t cols, void* dx,
                             float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream);

/*
 * Products grouped by expert.  Expert e has the rows offsets[e] .. offsets[e + 1] - 1
 * of a batch of T rows (offsets: [experts + 1] int32 on the device, not decreasing,
 * offsets[0] = 0, as luq_group_ids writes them; values beyond T are taken as T).
 * Groups may be empty.  The host needs no group's size: nothing is copied back.
 * 1 <= experts <= 4096.
 *
 * Weights are read in place: w_row codes from one row of an expert's matrix to the
 * next and w_expert codes from one expert to the next, both multiples of 32.  With
 * one int4_quantize call per expert these are K and N*K.  One call on the stacked
 * weights [experts * Nout][Kin] gives the forward operand (w_row = Kin, w_expert =
 * Nout * Kin) and, as codes_t [Kin][experts * Nout], the transposed one (w_row =
 * experts * Nout, w_expert = Nout).  w_scale holds one scale per expert
 * (w_scales = experts) or one for all (w_scales = 1).
 */

/*
 * int4_gemm_fwd_grouped -- int4_gemm_fwd (Eq. forward) with each row's expert:
 *   y[m][n] = x_scale * w_scale[e] * sum_k cx[m][k] * cw[e][n][k]
 * for the expert e that row m belongs to; rows at or after offsets[experts] get 0.
 *
 *  x_codes [T][K] INT4 codes, w_codes per expert [N][K]; y [T][N] fp32.
 *  T >= 0, T <= 2^30; 1 <= N <= 2^30; T * N <= 2^36 (256 GiB of outputs), and below 2^23
 *  tiles of 256 x 256.  K a multiple of 32 in [32, 2^17] (the int32-exact length).
 *  w_row >= K, w_row <= 2^22.  No workspace.
 */
luq_status int4_gemm_fwd_grouped(const uint8_t* x_codes, const float* x_scale, int x_signed,
                                 const uint8_t* w_codes, int64_t w_row, int64_t w_expert, const float* w_scale,
                                 int64_t w_scales, int w_signed, const int32_t* offsets, int64_t experts,
                                 int64_t T, int64_t N, int64_t K, float* y, void* stream);

/*
 * luq_gemm_dgrad_grouped -- luq_gemm_dgrad (Eq. backward) with each row's expert:
 *   dx[m][n] = (alpha / n_samples) * w_scale[e] * sum_k (sum_s cg_s[m][k]) * cw[e][n][k]
 *
 *  g_codes  [T][K] LUQ codes (n_samples = 1) or the int8 sums of two samples
 *           (LUQ_SMP_SUM | 2); w_codes_t per expert [N][K], K the layer's outputs
 *           and N its inputs; dx [T][N] fp32.  Rows of no expert get 0.
 *  K a multiple of 32 in [32, 2^18]; otherwise as int4_gemm_fwd_grouped.
 */
luq_status luq_gemm_dgrad_grouped(const uint8_t* g_codes, const float* alpha, int n_samples,
                                  const uint8_t* w_codes_t, int64_t w_row, int64_t w_expert, const float* w_scale,
                                  int64_t w_scales, int w_signed, const int32_t* offsets, int64_t experts,
                                  int64_t T, int64_t N, int64_t K, float* dx, void* stream);

/* Bytes of luq_gemm_wgrad_grouped's workspace; 0 if none. */
size_t luq_grouped_wgrad_workspace(int64_t T, int64_t Nout, int64_t Kin, int64_t experts);

/*
 * luq_gemm_wgrad_grouped -- luq_gemm_wgrad (Eq. update) over each expert's rows:
 *   dw[e][o][i] = (alpha / n_samples) * a_scale * sum over t of expert e of
 *                 (sum_s cg_s[t][o]) * ca[t][i]
 * An expert without rows gets zeros.  Group bounds need no alignment.
 *
 *  g_codes_t  [Nout][T] LUQ codes, or int8 sums with LUQ_SMP_SUM | 2;
 *  a_codes_t  [Kin][T] INT4 codes; dw [experts][Nout][Kin] fp32.
 *  T a multiple of 32 in [32, 2^18], or of 128 up to 2^22 (longer reductions are split,
 *  their int32 sums added in 64 bits): rows are padded at the end of the batch, after
 *  offsets[experts]; what the padding holds does not matter.  Nout, Kin in [1, 2^30], at
 *  most 2^36 outputs in below 2^23 tiles of 256 x 256 (2^34 beyond 2^18 rows, 2^32 if they
 *  are no multiple of 4).
 *  ws         workspace of luq_grouped_wgrad_workspace(T, Nout, Kin, experts).
 */
luq_status luq_gemm_wgrad_grouped(const uint8_t* g_codes_t, const float* alpha, int n_samples,
                                  const uint8_t* a_codes_t, const float* a_scale, int a_signed,
                                  const int32_t* offsets, int64_t experts, int64_t T, int64_t Nout, int64_t Kin,
                                  float* dw, void* ws, size_t ws_bytes, void* stream);

/*
 * Choice of experts.  A row of logits l gives scores s: their softmax, or each one's
 * sigmoid.  The choice goes by c = s + bias: with groups > 1 the experts are `groups`
 * runs of equal length, a run's rank is its largest c (group_best = 1) or the sum of its
 * two largest (2; of those there are), and the experts of the top_groups first runs
 * remain; of these the top_k largest c are taken, the largest first.  Equal values:
 * the lower index first.  c is compared as if exact (in 64 bits where it is a sum), so
 * that a choice does not hang on the rounding of an exponential: without a bias experts have
 * the order of their logits, and only the ranks of groups by two are sums.
 *   w_k = scale * s_k, or with renorm scale * s_k / (sum of the row's chosen s)
 *
 * A logit or a bias of -inf bars an expert.  Where fewer than top_k remain, the places
 * left hold expert -1 and weight 0 (no group of luq_group_ids, padding of
 * luq_embedding_fwd): a row of -inf, such as a padded position's, has none.  A row with
 * a logit or c that is NaN or +inf is a data error: experts -1, weights NaN.
 */
typedef enum { LUQ_SOFTMAX = 0, LUQ_SIGMOID = 1 } luq_score;

/*
 * luq_route_fwd -- the experts of every token, and their weights.
 *
 *  logits   [T][experts], type dt.  bias  [experts] fp32, or NULL.
 *  chosen   out: [T][top_k] int32;  weights  out: [T][top_k] fp32.
 *  T in [0, 2^25], experts in [1, 4096], top_k in [1, 64]; groups in [1, 64] divides
 *  experts; top_groups in [1, groups]; top_k is at most the experts of top_groups groups.
 *  scale is finite.  No workspace.
 */
luq_status luq_route_fwd(const void* logits, luq_dtype dt, int64_t T, int64_t experts, int64_t top_k, luq_score score,
                         const float* bias, int64_t groups, int64_t top_groups, int group_best, int renorm,
                         float scale, int32_t* chosen, float* weights, void* stream);

/*
 * luq_route_bwd -- gradient of luq_route_fwd's logits from that of its weights; the choice
 * itself has none.  With d_k = scale * dweights_k, or with renorm scale / S * (dweights_k -
 * sum_j dweights_j s_j / S), S the sum of the chosen s, and e_i the sum of the d_k of expert i:
 *   softmax: dl_i = s_i * (e_i - sum_j e_j s_j),   sigmoid: dl_i = s_i * (1 - s_i) * e_i
 *
 *  dweights [T][top_k] fp32; chosen as the forward call wrote it (an expert outside
 *  [0, experts) has no weight and gives nothing; a row without any gets zeros).
 *  dlogits  out: [T][experts], type dt; it may be logits.
 */
luq_status luq_route_bwd(const float* dweights, const void* logits, luq_dtype dt, const int32_t* chosen, int64_t T,
                         int64_t experts, int64_t top_k, luq_score score, int renorm, float scale, void* dlogits,
                         void* stream);

/*
 * Softmax cross entropy of the last layer, z[t][v] = scale * sum_d x[t][d] table[v][d],
 * whose logits are not kept: the forward call leaves the logarithm of each row's sum of
 * exponentials, and the backward call forms the products again, a piece of the
 * vocabulary at a time.
 *   lse_t = log sum_v exp z_tv
 *   loss_t = lse_t - (1 - smoothing) * z_t,target - smoothing / V * sum_v z_tv
 *
 *  x        [T][D], type xt.  table  [V][D], type tt.  Both 16-byte aligned.
 *  targets  [T]; one below 0 is padding: loss 0, no gradient, whatever its row of x holds.
 *           One at or above V is a data error: loss NaN, no gradient.
 *  T in [0, 2^21], V in [1, 2^28], D in [1, 2^17]; T * V at most 2^37, T * D and V * D at most
 *  2^36; scale finite and not 0, smoothing in [0, 1].
 *
 * Products are those of bf16 matrix instructions with fp32 sums.  An fp32 tensor is taken
 * as three bf16 terms (24 bits, fewer below 2^-110: a term is a multiple of 2^-133), of
 * whose products those above 2^-24 are formed.
 * In the backward call's products with the logits' gradient, an fp32 output is formed from three
 * terms of it (24 bits) and as many of an fp32 tensor; a bf16 output from one term of it (8 bits: the
 * output is off by 1.4 times its own rounding, in the norm) and two of an fp32 tensor (16 bits).
 */

/* Bytes of the workspace of the forward call (gt = -1) or of the backward call (gt: type
 * of dtable); 0 if the sizes are refused. */
size_t luq_cross_entropy_workspace(int64_t T, int64_t V, int64_t D, luq_dtype xt, luq_dtype tt, int gt);

/*
 * luq_cross_entropy_fwd -- the loss of every token.
 *  loss, lse  out: [T] fp32; lse is 0 where the target is no row of the table.  The loss is summed from
 *             differences to the row's largest logit: without smoothing it is not below 0.
 */
luq_status luq_cross_entropy_fwd(const void* x, luq_dtype xt, const void* table, luq_dtype tt, const void* targets,
                                 luq_index it, int64_t T, int64_t V, int64_t D, float scale, float smoothing,
                                 float* loss, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * luq_cross_entropy_bwd -- gradients of luq_cross_entropy_fwd: with
 *   g_tv = dloss_t * scale * (exp(z_tv - lse_t) - (1 - smoothing) [v = target_t] - smoothing / V)
 *   dx = g table,  dtable = g^T x
 *
 *  dloss    [T] fp32.  lse  [T] of the forward call, which had the same scale and smoothing.
 *  dx       out: [T][D], type xt.
 *  dtable   out: [V][D], type gt: fp32, or bf16 where the table is.  accumulate = 0: written
 *           whole; 1: added to (a table shared with the embedding, whose lookup's gradient
 *           is there already).
 *  Sums are taken in a fixed order: the same result on every call.
 */
luq_status luq_cross_entropy_bwd(const float* dloss, const void* x, luq_dtype xt, const void* table, luq_dtype tt,
                                 const void* targets, luq_index it, const float* lse, int64_t T, int64_t V, int64_t D,
                                 float scale, float smoothing, int accumulate, void* dx, void* dtable, luq_dtype gt,
                                 void* ws, size_t ws_bytes, void* stream);

/*
 * AdamW over many tensors in one launch.  With g' = grad_scale * g, t the step and
 * r = lr * lr_scale:
 *   m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
 *   p = p - r * weight_decay * p - r * (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 *
 * States are fp32, or 8 bits: m and the root of v as e4m3 codes (OCP), of which 32
 * consecutive elements share a power of two 2^(scale - 127) that leaves the largest
 * magnitude in [128, 256).  They are rounded stochastically, to the code above with the
 * probability of the fraction (in 2^-16), as LUQ rounds gradients: to the nearest code, a
 * v that changes by a thousandth a step would never leave its own.  A root above 0 does
 * not become 0; what is not finite becomes NaN, and is left out of its block's scale.
 * The random words are Philox4x32-10 of the key seed and the counter (i >> 2 in two words,
 * the tensor's place in the plan, t): element i takes word i & 3, its low half for m and
 * its high half for v.  States begin as zeros (codes and scales 0).
 */
typedef struct {
  float* p;             /* [n] weights, updated                                    */
  const void* g;        /* [n] gradient, type gt                                   */
  void* m;              /* [n] fp32, or codes                                      */
  void* v;              /* [n] fp32 (v), or codes (its root)                       */
  uint8_t* m_scale;     /* [ceil(n / 32)] with codes, else not looked at           */
  uint8_t* v_scale;
  void* copy;           /* out: [n] bf16 copy of the new weights, or NULL          */
  int64_t n;            /* 0 <= n <= 2^35                                          */
  float weight_decay;   /* finite                                                  */
  float lr_scale;       /* finite                                                  */
  int gt;               /* luq_dtype of g                                          */
  int state_bits;       /* 32 or 8                                                 */
} luq_adamw_tensor;

/* Bytes of the plan for count tensors (at most 2^20) of n[0] .. n[count - 1] elements, at
 * most 2^35 together; 0 if refused, or if there is nothing to do. */
size_t luq_adamw_plan_bytes(const int64_t* n, int64_t count);

/*
 * luq_adamw_plan -- the work of a step, laid out once for tensors that keep their places.
 * `tensors` and `plan` are HOST memory; the caller copies the plan to the device.  None that
 * a step writes overlaps another (LUQ_ERR_PARAM; gradients may be shared); each is aligned to
 * its elements.
 * Errors: LUQ_ERR_NULL, LUQ_ERR_SHAPE, LUQ_ERR_DTYPE, LUQ_ERR_PARAM, LUQ_ERR_ALIGN,
 * LUQ_ERR_WORKSPACE (plan_bytes is not luq_adamw_plan_bytes).
 */
luq_status luq_adamw_plan(const luq_adamw_tensor* tensors, int64_t count, void* plan, size_t plan_bytes);

/*
 * luq_adamw_step -- one step of the tensors of a plan.
 *
 *  plan        device memory, 16-byte aligned, as luq_adamw_plan wrote it for `count` tensors.
 *  lr          [1] fp32 on the device;  step  [1] int64 on the device, t >= 1 (less counts
 *              as 1): a captured graph takes new ones at every replay.
 *  beta1, beta2 in [0, 1);  eps >= 0, finite.
 *  grad_scale  [1] fp32 on the device, or NULL for 1.  One that is NaN or infinite (an
 *              overflowed norm) skips the step: nothing is written.
 */
luq_status luq_adamw_step(const void* plan, size_t plan_bytes, int64_t count, const float* lr, const int64_t* step,
                          double beta1, double beta2, float eps, const float* grad_scale, uint64_t seed, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LUQ_LM_H */
