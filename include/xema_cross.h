/*
 * xema_cross.h -- the operators of a cross-attention sub-block (gfx950):
 * layer norm with the residual's addition, attention to an encoder's states
 * of another length, and the linear layer with bias, activation and residual,
 * each with its gradient.
 *
 * The block of xema.h meets the text by joint attention.  Denoisers of the
 * same family meet it in a sub-block of its own, between self-attention and
 * the feed-forward layer, and decoders of single tokens meet an encoder the
 * same way:
 *   xema_op_layernorm     h = LayerNorm(x)
 *   xema_op_linear        q = h W_q^T + b_q,  [k v] = e W_kv^T + b_kv
 *   xema_op_cross_attn    a = softmax(scale q k^T) v
 *   xema_op_linear        x <- x + a W_o^T + b_o
 * and the entry points ending in _bwd are their gradients.
 *
 * Conventions are those of xema_ffn.h: status return, host-side validation
 * before any launch, caller-owned device buffers, no allocation, no state
 * between calls, asynchronous on `stream` (a hipStream_t of the current device,
 * NULL or hipStreamLegacy = default stream, hipStreamPerThread;
 * XEMA_ERR_INVALID_ARG for a stream of another device), 16-byte aligned
 * pointers unless stated.  Every entry point can be captured into a graph;
 * workspaces are scratch memory whose contents on entry are ignored, and calls
 * that may overlap need one each.  Matrices are row-major with a leading
 * dimension ("ld", in elements) of at least their width, below 2^21, whose
 * bytes are a multiple of 16; widths are multiples of 8 and at most 131072; row
 * counts are any from 0 to 2^24 - 1.  Outputs must not overlap inputs,
 * workspaces or each other, except where an entry point allows it
 * (XEMA_ERR_INVALID_ARG); column ranges of one buffer do not overlap.  A call
 * of no rows checks its arguments like any other.
 *
 * Sums and statistics are fp32, each in one fixed order, with no atomics: the
 * same call gives the same bytes.
 */
#ifndef XEMA_CROSS_H_
#define XEMA_CROSS_H_

#include <stdint.h>

#include "xema.h"
#include "xema_ffn.h"
#include "xema_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Layer norm of x, or of the sum of x and the residual stream:
 *   s[r] = x[r] + resid[r]                       (resid NULL: s = x)
 *   m = mean_j s[r][j],  v = mean_j (s[r][j] - m)^2
 *   y[r][i] = (s[r][i] - m) / sqrt(v + eps) * gamma[i] + beta[i]
 * s is the fp32 sum: `sum` (may be NULL) receives it in sum_dtype, and y
 * comes from the fp32 value, not from the stored one.
 * x, resid, sum and y are each XEMA_BF16, XEMA_F16 or XEMA_F32 [rows, dim];
 * gamma and beta are bf16 [dim] (NULL: ones, zeros).  `sum` may be x or resid
 * itself (the same pointer, type and ld).  dim is at most 16384.  The variance
 * is taken about the mean (two passes over the registers).                  */
typedef struct {
  int64_t rows; int32_t dim;
  const void* x; int32_t x_dtype; int64_t ldx;
  const void* resid; int32_t resid_dtype; int64_t ld_resid;
  void* sum; int32_t sum_dtype; int64_t ld_sum;
  const void *gamma, *beta;
  float eps;
  void* y; int32_t y_dtype; int64_t ldy;
} xema_layernorm_args;

XEMA_API int xema_op_layernorm(const xema_layernorm_args* args, void* stream);

/* Gradient of xema_op_layernorm, for s the norm's input (x, or the stored sum)
 * and dy the gradient that reaches y, with n = (s - m) / sqrt(v + eps):
 *   g = dy * gamma
 *   dx[r][i] = (g_i - mean_j g_j - n_i mean_j(g_j n_j)) / sqrt(v + eps) + dsum[r][i]
 *   dgamma[i] = sum over rows of dy[r][i] n[r][i],  dbeta[i] = sum over rows of dy[r][i]
 * dsum (may be NULL) is the gradient that reaches s by itself, through the
 * residual stream; dx is then the gradient of both x and resid.
 * s, dy, dsum and dx are each XEMA_BF16, XEMA_F16 or XEMA_F32 [rows, dim];
 * dgamma and dbeta fp32 [dim] (each may be NULL), zeros where rows is 0; gamma
 * as above.  dx may be dy, dsum or s itself (the same pointer, type and ld).
 * The workspace (16-byte aligned) has at least
 * xema_layernorm_bwd_workspace_bytes(rows, dim) bytes; without dgamma and
 * dbeta it may be NULL.                                                     */
typedef struct {
  int64_t rows; int32_t dim;
  const void* s; int32_t s_dtype; int64_t ld_s;
  const void* dy; int32_t dy_dtype; int64_t ld_dy;
  const void* dsum; int32_t dsum_dtype; int64_t ld_dsum;
  const void* gamma;
  float eps;
  void* dx; int32_t dx_dtype; int64_t ld_dx;
  float *dgamma, *dbeta;
  void* workspace; int64_t workspace_bytes;
} xema_layernorm_bwd_args;

XEMA_API int xema_layernorm_bwd_workspace_bytes(int64_t rows, int32_t dim, int64_t* bytes);
XEMA_API int xema_op_layernorm_bwd(const xema_layernorm_bwd_args* args, void* stream);

/* Linear layer with its epilogue:
 *   z = x w^T + bias,  y = act(z) + resid
 * act: XEMA_ACT_SILU, XEMA_ACT_GELU_TANH (xema_ffn.h) or XEMA_ACT_NONE.
 * x [rows, dim] and w [out_dim, dim] (contiguous) have type `dtype` (XEMA_BF16
 * or XEMA_F16); bias bf16 [out_dim] and resid [rows, out_dim] (XEMA_BF16,
 * XEMA_F16 or XEMA_F32) may be NULL; y [rows, out_dim] is XEMA_BF16, XEMA_F16
 * or XEMA_F32 and may be resid itself (the same pointer, type and ld).  The
 * products are summed in fp32 and nothing is rounded before y.  pre (may be
 * NULL; 16-byte aligned) receives what the gradient of an activation needs, z
 * in 24 bits (the upper 24 of fp32) in xema_linear_pre_bytes(rows, out_dim)
 * bytes: per row and four columns 12 bytes, the upper halves (four uint16), then
 * the third bytes.  (16-bit values there would add a rounding of their own to
 * every gradient.)                                                          */
typedef struct {
  int32_t dtype, act;
  int64_t rows; int32_t dim, out_dim;
  const void* x; int64_t ldx;
  const void* w; const void* bias;
  const void* resid; int32_t resid_dtype; int64_t ld_resid;
  void* y; int32_t y_dtype; int64_t ldy;
  void* pre;
} xema_linear_args;

XEMA_API int xema_linear_pre_bytes(int64_t rows, int32_t out_dim, int64_t* bytes);
XEMA_API int xema_op_linear(const xema_linear_args* args, void* stream);

/* Gradient of xema_op_linear for dy, the gradient that reaches y (which is
 * resid's gradient as it stands):
 *   dz = dy act'(z)                                 (z from pre)
 *   dx = dz w  [rows, dim],  dw = dz^T x  [out_dim, dim] contiguous,
 *   dbias = column sums of dz                       bf16 [out_dim]
 * x, w, dx and dw have type `dtype`; dy is of type `dtype` or XEMA_F32.  pre is
 * xema_op_linear's of the same sizes (not read, and may be NULL, with
 * XEMA_ACT_NONE).  Each of dx, dw and dbias may be NULL (not all).  dz is formed
 * in fp32 and rounded to `dtype` once, for the products; the column sums take
 * the fp32 values.  Where rows is 0 the gradients of weights and bias are
 * zeros.  The workspace (256-byte aligned) has at least
 * xema_linear_bwd_workspace_bytes(rows, dim, out_dim) bytes.                */
typedef struct {
  int32_t dtype, act;
  int64_t rows; int32_t dim, out_dim;
  const void* x; int64_t ldx;
  const void* w;
  const void* pre;
  const void* dy; int32_t dy_dtype; int64_t ld_dy;
  void* dx; int64_t ld_dx;
  void *dw, *dbias;
  void* workspace; int64_t workspace_bytes;
} xema_linear_bwd_args;

XEMA_API int xema_linear_bwd_workspace_bytes(int64_t rows, int32_t dim, int32_t out_dim, int64_t* bytes);
XEMA_API int xema_op_linear_bwd(const xema_linear_bwd_args* args, void* stream);

/* Attention of `batch` sequences of q_len tokens to kv_len encoder states each,
 * of which the first n_b = kv_lens[b] are there:
 *   s[i][j] = scale q_i . k_j,  p[i] = softmax over j < n_b of s[i],
 *   o_i = sum_j p[i][j] v_j,  lse_i = ln sum_{j < n_b} e^s[i][j]
 * for every head h of `heads`, with head h / (heads / kv_heads) of the kv_heads
 * (heads is a multiple of kv_heads; its quotient's heads share a state's).
 * q and o [batch * q_len, heads * head_dim], k and v [batch * kv_len, kv_heads *
 * head_dim] have type `dtype` (XEMA_BF16 or XEMA_F16); row b q_len + i is token
 * i of sequence b, and head h is columns h head_dim ... .  q_len and kv_len may
 * be 0, as may batch; head_dim is a multiple of 8 up to 128; scale is finite
 * and above 0.
 * kv_lens int32 [batch] (4-byte aligned), on the device, NULL: kv_len for all;
 * values are taken between 0 and kv_len.  Rows of k and v behind a sequence's
 * last state are not read for their values: NaN there does not reach o.  A
 * sequence of no states gives o = 0 and lse = -infinity, and so do tokens whose
 * scores all are -infinity; such scores weigh nothing beside others.  Scores are
 * fp32 and so is scale log2(e) q_i . k_j: past 2^128 they are infinite.
 * lse fp32 [batch, heads, q_len] (may be NULL; 4-byte aligned) is for the
 * gradient.  p is rounded to `dtype` for its product with v; scores, sums and o
 * are fp32 until the rounding of o (weights below 2^-126 are zeros).
 * The workspace (256-byte aligned, at least xema_cross_attn_workspace_bytes
 * bytes) holds the parts of calls whose states are split over workgroups; it
 * may be NULL where that is 0.  q_len heads / kv_heads is at most 2^30, and
 * batch heads ceil(q_len / 32) and batch kv_heads ceil(kv_len / 32) at most 2^22
 * (XEMA_ERR_UNSUPPORTED).                                                    */
typedef struct {
  int32_t dtype;
  int32_t batch, heads, kv_heads, head_dim, q_len, kv_len;
  const void* q; int64_t ldq;
  const void* k; int64_t ldk;
  const void* v; int64_t ldv;
  const int32_t* kv_lens;
  float scale;
  void* o; int64_t ldo;
  float* lse;
  void* workspace; int64_t workspace_bytes;
} xema_cross_attn_args;

XEMA_API int xema_cross_attn_workspace_bytes(int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t q_len,
                                             int32_t kv_len, int64_t* bytes);
XEMA_API int xema_op_cross_attn(const xema_cross_attn_args* args, void* stream);

/* Gradient of xema_op_cross_attn for dout, the gradient that reaches o (of o's
 * type and shape, ld_do):
 *   D_i = dout_i . o_i,  dp[i][j] = dout_i . v_j,  ds[i][j] = p[i][j] (dp[i][j] - D_i)
 *   dq_i = scale sum_j ds[i][j] k_j,  dk_j = scale sum_i ds[i][j] q_i,  dv_j = sum_i p[i][j] dout_i
 * the sums over i taking the tokens of all heads that share j's head.  q, k, v,
 * o, lse, kv_lens and scale are those of the forward call; dq is laid out as q
 * (ld_dq), dk and dv as k and v (ld_dk, ld_dv).  dq may be NULL, and so may dk
 * and dv together (not all three).  Gradients of states behind a sequence's
 * last one are zeros, those of tokens with no states too.  p and ds are formed
 * in fp32 and rounded to `dtype` once, for the products; in fp16 p is carried as
 * 2^14 p (16 bits down to p = 2^-28), and ds below 2^-14 loses bits (off by up to
 * 2^-25): scale the loss as fp16 training does.  D comes from the rounded o.
 * p comes from lse, whose rounding takes it off by a factor of up to e^(|lse| / 2^22)
 * (2^-8, bf16's half step, at |lse| = 2^14); a token whose |lse| is 2^22 or more has
 * no gradient: its lse tells no weights, and p = 0.
 * The workspace (256-byte aligned) has at least
 * xema_cross_attn_bwd_workspace_bytes bytes.  Limits as above.              */
typedef struct {
  int32_t dtype;
  int32_t batch, heads, kv_heads, head_dim, q_len, kv_len;
  const void* q; int64_t ldq;
  const void* k; int64_t ldk;
  const void* v; int64_t ldv;
  const int32_t* kv_lens;
  float scale;
  const void* o; int64_t ldo;
  const float* lse;
  const void* dout; int64_t ld_do;
  void* dq; int64_t ld_dq;
  void* dk; int64_t ld_dk;
  void* dv; int64_t ld_dv;
  void* workspace; int64_t workspace_bytes;
} xema_cross_attn_bwd_args;

XEMA_API int xema_cross_attn_bwd_workspace_bytes(int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t q_len,
                                                 int32_t kv_len, int64_t* bytes);
XEMA_API int xema_op_cross_attn_bwd(const xema_cross_attn_bwd_args* args, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* XEMA_CROSS_H_ */
