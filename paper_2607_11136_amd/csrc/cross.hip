// Host entry points of the cross-attention sub-block's operators
// (xema_cross.h): argument validation, then the launches of k_layernorm.hip,
// k_linear.hip, k_cross.hip and k_cross_bwd.hip.
#include <cmath>

#include "cross.h"
#include "op_checks.h"
#include "xema_internal.h"

using namespace xema;

namespace {

bool is_act(int act) { return act == XEMA_ACT_NONE || act == XEMA_ACT_SILU || act == XEMA_ACT_GELU_TANH; }

int check_layernorm(const xema_layernorm_args* a) {
  if (!a || !a->x || !a->y || !(a->eps > 0.f)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  if (!is_norm_type(a->x_dtype) || (a->resid && !is_norm_type(a->resid_dtype)) || (a->sum && !is_norm_type(a->sum_dtype)) || !is_norm_type(a->y_dtype))
    return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_width(a->dim, XEMA_BF16));
  if (a->dim > 16384) return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_matrix(a->x, a->x_dtype, a->dim, a->ldx));
  XEMA_CHECK(check_matrix(a->resid, a->resid_dtype, a->dim, a->ld_resid, true));
  XEMA_CHECK(check_matrix(a->sum, a->sum_dtype, a->dim, a->ld_sum, true));
  XEMA_CHECK(check_matrix(a->y, a->y_dtype, a->dim, a->ldy));
  if (!aligned(a->gamma, 16) || !aligned(a->beta, 16)) return XEMA_ERR_MISALIGNED;
  const Span x = matrix(a->x, a->x_dtype, a->rows, a->dim, a->ldx), res = matrix(a->resid, a->resid_dtype, a->rows, a->dim, a->ld_resid);
  const Span sum = matrix(a->sum, a->sum_dtype, a->rows, a->dim, a->ld_sum), y = matrix(a->y, a->y_dtype, a->rows, a->dim, a->ldy);
  const Span gamma{a->gamma, 2 * (int64_t)a->dim}, beta{a->beta, 2 * (int64_t)a->dim};
  if (any_overlap(y, {x, res, sum, gamma, beta}) || any_overlap(sum, {gamma, beta})) return XEMA_ERR_INVALID_ARG;
  if (overlaps(sum, x) && !same(a->sum, a->sum_dtype, a->ld_sum, a->x, a->x_dtype, a->ldx)) return XEMA_ERR_INVALID_ARG;
  if (overlaps(sum, res) && !same(a->sum, a->sum_dtype, a->ld_sum, a->resid, a->resid_dtype, a->ld_resid)) return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_layernorm_bwd(const xema_layernorm_bwd_args* a) {
  if (!a || !a->s || !a->dy || !a->dx || !(a->eps > 0.f)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  if (!is_norm_type(a->s_dtype) || !is_norm_type(a->dy_dtype) || (a->dsum && !is_norm_type(a->dsum_dtype)) || !is_norm_type(a->dx_dtype))
    return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_width(a->dim, XEMA_BF16));
  if (a->dim > 16384) return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_matrix(a->s, a->s_dtype, a->dim, a->ld_s));
  XEMA_CHECK(check_matrix(a->dy, a->dy_dtype, a->dim, a->ld_dy));
  XEMA_CHECK(check_matrix(a->dsum, a->dsum_dtype, a->dim, a->ld_dsum, true));
  XEMA_CHECK(check_matrix(a->dx, a->dx_dtype, a->dim, a->ld_dx));
  if (!aligned(a->gamma, 16) || !aligned(a->dgamma, 16) || !aligned(a->dbeta, 16) || !aligned(a->workspace, 16)) return XEMA_ERR_MISALIGNED;
  int64_t need = 0;
  XEMA_CHECK(xema_layernorm_bwd_workspace_bytes(a->rows, a->dim, &need));
  const bool sums = a->dgamma || a->dbeta;
  if (sums) {
    if (!a->workspace) return XEMA_ERR_INVALID_ARG;
    if (a->workspace_bytes < need) return XEMA_ERR_WORKSPACE_TOO_SMALL;
  }
  const Span s = matrix(a->s, a->s_dtype, a->rows, a->dim, a->ld_s), dy = matrix(a->dy, a->dy_dtype, a->rows, a->dim, a->ld_dy);
  const Span dsum = matrix(a->dsum, a->dsum_dtype, a->rows, a->dim, a->ld_dsum), dx = matrix(a->dx, a->dx_dtype, a->rows, a->dim, a->ld_dx);
  const Span gamma{a->gamma, 2 * (int64_t)a->dim}, dgamma{a->dgamma, 4 * (int64_t)a->dim}, dbeta{a->dbeta, 4 * (int64_t)a->dim};
  const Span ws{sums ? a->workspace : nullptr, need};
  if (any_overlap(dgamma, {s, dy, dsum, dx, gamma, dbeta, ws}) || any_overlap(dbeta, {s, dy, dsum, dx, gamma, ws}) ||
      any_overlap(ws, {s, dy, dsum, dx, gamma}) || overlaps(dx, gamma))
    return XEMA_ERR_INVALID_ARG;
  if ((overlaps(dx, s) && !same(a->dx, a->dx_dtype, a->ld_dx, a->s, a->s_dtype, a->ld_s)) ||
      (overlaps(dx, dy) && !same(a->dx, a->dx_dtype, a->ld_dx, a->dy, a->dy_dtype, a->ld_dy)) ||
      (overlaps(dx, dsum) && !same(a->dx, a->dx_dtype, a->ld_dx, a->dsum, a->dsum_dtype, a->ld_dsum)))
    return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_linear(const xema_linear_args* a) {
  if (!a || !a->x || !a->w || !a->y || !is_act(a->act)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  if (!is16(a->dtype) || (a->resid && !is_norm_type(a->resid_dtype)) || !is_norm_type(a->y_dtype)) return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_width(a->dim, a->dtype));
  XEMA_CHECK(check_width(a->out_dim, a->dtype));
  XEMA_CHECK(check_matrix(a->x, a->dtype, a->dim, a->ldx));
  XEMA_CHECK(check_matrix(a->w, a->dtype, a->dim, a->dim));
  XEMA_CHECK(check_matrix(a->resid, a->resid_dtype, a->out_dim, a->ld_resid, true));
  XEMA_CHECK(check_matrix(a->y, a->y_dtype, a->out_dim, a->ldy));
  if (!aligned(a->bias, 16) || !aligned(a->pre, 16)) return XEMA_ERR_MISALIGNED;
  const int64_t N = a->out_dim;
  const Span x = matrix(a->x, a->dtype, a->rows, a->dim, a->ldx), w{a->w, 2 * N * a->dim}, bias{a->bias, 2 * N};
  const Span res = matrix(a->resid, a->resid_dtype, a->rows, N, a->ld_resid), y = matrix(a->y, a->y_dtype, a->rows, N, a->ldy);
  const Span pre{a->pre, 3 * a->rows * N};
  if (any_overlap(y, {x, w, bias, pre}) || any_overlap(pre, {x, w, bias, res})) return XEMA_ERR_INVALID_ARG;
  if (overlaps(y, res) && !same(a->y, a->y_dtype, a->ldy, a->resid, a->resid_dtype, a->ld_resid)) return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_linear_bwd(const xema_linear_bwd_args* a) {
  if (!a || !a->x || !a->w || !a->dy || !a->workspace || !is_act(a->act) || (!a->dx && !a->dw && !a->dbias)) return XEMA_ERR_INVALID_ARG;
  if (a->act != XEMA_ACT_NONE && !a->pre) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  if (!is16(a->dtype) || (a->dy_dtype != a->dtype && a->dy_dtype != XEMA_F32)) return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_width(a->dim, a->dtype));
  XEMA_CHECK(check_width(a->out_dim, a->dtype));
  XEMA_CHECK(check_matrix(a->x, a->dtype, a->dim, a->ldx));
  XEMA_CHECK(check_matrix(a->w, a->dtype, a->dim, a->dim));
  XEMA_CHECK(check_matrix(a->dy, a->dy_dtype, a->out_dim, a->ld_dy));
  XEMA_CHECK(check_matrix(a->dx, a->dtype, a->dim, a->ld_dx, true));
  XEMA_CHECK(check_matrix(a->dw, a->dtype, a->dim, a->dim, true));
  if (!aligned(a->pre, 16) || !aligned(a->dbias, 16) || !aligned(a->workspace, 256)) return XEMA_ERR_MISALIGNED;
  int64_t need = 0;
  XEMA_CHECK(xema_linear_bwd_workspace_bytes(a->rows, a->dim, a->out_dim, &need));
  if (a->workspace_bytes < need) return XEMA_ERR_WORKSPACE_TOO_SMALL;
  const int64_t N = a->out_dim, D = a->dim;
  const Span x = matrix(a->x, a->dtype, a->rows, D, a->ldx), w{a->w, 2 * N * D}, dy = matrix(a->dy, a->dy_dtype, a->rows, N, a->ld_dy);
  const Span pre{a->act == XEMA_ACT_NONE ? nullptr : a->pre, 3 * a->rows * N}, dx = matrix(a->dx, a->dtype, a->rows, D, a->ld_dx);
  const Span dw{a->dw, 2 * N * D}, db{a->dbias, 2 * N}, ws{a->workspace, need};
  if (any_overlap(ws, {x, w, dy, pre, dx, dw, db}) || any_overlap(dx, {x, w, dy, pre, dw, db}) || any_overlap(dw, {x, w, dy, pre, db}) ||
      any_overlap(db, {x, w, dy, pre}))
    return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

// The sizes of an attention call.
int check_cross_shape(int64_t batch, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t q_len, int64_t kv_len) {
  if (batch < 0 || q_len < 0 || kv_len < 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || head_dim <= 0) return XEMA_ERR_INVALID_ARG;
  if (head_dim % 8 || head_dim > 128) return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_width(heads * head_dim, XEMA_BF16));
  XEMA_CHECK(check_rows(batch * q_len));
  XEMA_CHECK(check_rows(batch * kv_len));
  // (no empty tensor asks for a launch past its limits either)
  if (batch > MAX_ROWS || q_len > MAX_ROWS || kv_len > MAX_ROWS) return XEMA_ERR_UNSUPPORTED;
  constexpr int64_t MOST = (int64_t)1 << 22;
  if (q_len * (heads / kv_heads) > (int64_t)1 << 30 || batch * heads * ((q_len + 31) / 32) > MOST || batch * kv_heads * ((kv_len + 31) / 32) > MOST)
    return XEMA_ERR_UNSUPPORTED;
  return XEMA_OK;
}

template <typename A>
CrossShape shape_of(const A* a) {
  return {a->batch, a->heads, a->kv_heads, a->head_dim, a->q_len, a->kv_len};
}

bool is_scale(float s) { return std::isfinite(s) && s > 0.f; }

int check_cross_attn(const xema_cross_attn_args* a) {
  if (!a || !a->q || !a->k || !a->v || !a->o || !is_scale(a->scale)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_cross_shape(a->batch, a->heads, a->kv_heads, a->head_dim, a->q_len, a->kv_len));
  if (!is16(a->dtype)) return XEMA_ERR_UNSUPPORTED;
  const int64_t q_rows = (int64_t)a->batch * a->q_len, kv_rows = (int64_t)a->batch * a->kv_len;
  const int64_t qw = (int64_t)a->heads * a->head_dim, kvw = (int64_t)a->kv_heads * a->head_dim;
  XEMA_CHECK(check_matrix(a->q, a->dtype, qw, a->ldq));
  XEMA_CHECK(check_matrix(a->k, a->dtype, kvw, a->ldk));
  XEMA_CHECK(check_matrix(a->v, a->dtype, kvw, a->ldv));
  XEMA_CHECK(check_matrix(a->o, a->dtype, qw, a->ldo));
  if (!aligned(a->kv_lens, 4) || !aligned(a->lse, 4) || !aligned(a->workspace, 256)) return XEMA_ERR_MISALIGNED;
  const int64_t need = cross_attn_workspace(shape_of(a));
  if (need) {
    if (!a->workspace) return XEMA_ERR_INVALID_ARG;
    if (a->workspace_bytes < need) return XEMA_ERR_WORKSPACE_TOO_SMALL;
  }
  const Span q = matrix(a->q, a->dtype, q_rows, qw, a->ldq), k = matrix(a->k, a->dtype, kv_rows, kvw, a->ldk);
  const Span v = matrix(a->v, a->dtype, kv_rows, kvw, a->ldv), o = matrix(a->o, a->dtype, q_rows, qw, a->ldo);
  const Span lens{a->kv_lens, 4 * (int64_t)a->batch}, lse{a->lse, 4 * q_rows * a->heads}, ws{need ? a->workspace : nullptr, need};
  if (any_overlap(o, {q, k, v, lens, lse, ws}) || any_overlap(lse, {q, k, v, lens, ws}) || any_overlap(ws, {q, k, v, lens})) return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_cross_attn_bwd(const xema_cross_attn_bwd_args* a) {
  if (!a || !a->q || !a->k || !a->v || !a->o || !a->lse || !a->dout || !a->workspace || !is_scale(a->scale)) return XEMA_ERR_INVALID_ARG;
  if (!a->dk != !a->dv || (!a->dq && !a->dk)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_cross_shape(a->batch, a->heads, a->kv_heads, a->head_dim, a->q_len, a->kv_len));
  if (!is16(a->dtype)) return XEMA_ERR_UNSUPPORTED;
  const int64_t q_rows = (int64_t)a->batch * a->q_len, kv_rows = (int64_t)a->batch * a->kv_len;
  const int64_t qw = (int64_t)a->heads * a->head_dim, kvw = (int64_t)a->kv_heads * a->head_dim;
  XEMA_CHECK(check_matrix(a->q, a->dtype, qw, a->ldq));
  XEMA_CHECK(check_matrix(a->k, a->dtype, kvw, a->ldk));
  XEMA_CHECK(check_matrix(a->v, a->dtype, kvw, a->ldv));
  XEMA_CHECK(check_matrix(a->o, a->dtype, qw, a->ldo));
  XEMA_CHECK(check_matrix(a->dout, a->dtype, qw, a->ld_do));
  XEMA_CHECK(check_matrix(a->dq, a->dtype, qw, a->ld_dq, true));
  XEMA_CHECK(check_matrix(a->dk, a->dtype, kvw, a->ld_dk, true));
  XEMA_CHECK(check_matrix(a->dv, a->dtype, kvw, a->ld_dv, true));
  if (!aligned(a->kv_lens, 4) || !aligned(a->lse, 4) || !aligned(a->workspace, 256)) return XEMA_ERR_MISALIGNED;
  const int64_t need = cross_attn_bwd_workspace(shape_of(a));
  if (a->workspace_bytes < need) return XEMA_ERR_WORKSPACE_TOO_SMALL;
  const Span q = matrix(a->q, a->dtype, q_rows, qw, a->ldq), k = matrix(a->k, a->dtype, kv_rows, kvw, a->ldk);
  const Span v = matrix(a->v, a->dtype, kv_rows, kvw, a->ldv), o = matrix(a->o, a->dtype, q_rows, qw, a->ldo);
  const Span dout = matrix(a->dout, a->dtype, q_rows, qw, a->ld_do), dq = matrix(a->dq, a->dtype, q_rows, qw, a->ld_dq);
  const Span dk = matrix(a->dk, a->dtype, kv_rows, kvw, a->ld_dk), dv = matrix(a->dv, a->dtype, kv_rows, kvw, a->ld_dv);
  const Span lens{a->kv_lens, 4 * (int64_t)a->batch}, lse{a->lse, 4 * q_rows * a->heads}, ws{a->workspace, need};
  if (any_overlap(ws, {q, k, v, o, dout, dq, dk, dv, lens, lse}) || any_overlap(dq, {q, k, v, o, dout, dk, dv, lens, lse}) ||
      any_overlap(dk, {q, k, v, o, dout, dv, lens, lse}) || any_overlap(dv, {q, k, v, o, dout, lens, lse}))
    return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

}  // namespace

extern "C" int xema_op_layernorm(const xema_layernorm_args* args, void* stream) {
  XEMA_CHECK(check_layernorm(args));
  if (args->rows == 0) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_layernorm(*args, s));
}

extern "C" int xema_layernorm_bwd_workspace_bytes(int64_t rows, int32_t dim, int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(rows));
  XEMA_CHECK(check_width(dim, XEMA_BF16));
  if (dim > 16384) return XEMA_ERR_UNSUPPORTED;
  *bytes = layernorm_bwd_partials(rows) * 2 * dim * 4;
  return XEMA_OK;
}

extern "C" int xema_op_layernorm_bwd(const xema_layernorm_bwd_args* args, void* stream) {
  XEMA_CHECK(check_layernorm_bwd(args));
  if (args->rows == 0 && !args->dgamma && !args->dbeta) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_layernorm_bwd(*args, s));
}

extern "C" int xema_linear_pre_bytes(int64_t rows, int32_t out_dim, int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(rows));
  XEMA_CHECK(check_width(out_dim, XEMA_BF16));
  *bytes = 3 * rows * out_dim;
  return XEMA_OK;
}

extern "C" int xema_op_linear(const xema_linear_args* args, void* stream) {
  XEMA_CHECK(check_linear(args));
  if (args->rows == 0) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_linear(*args, s));
}

extern "C" int xema_linear_bwd_workspace_bytes(int64_t rows, int32_t dim, int32_t out_dim, int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(rows));
  XEMA_CHECK(check_width(dim, XEMA_BF16));
  XEMA_CHECK(check_width(out_dim, XEMA_BF16));
  // dz in 16 bits, its partial column sums, and the partial sums of dx and dw
  *bytes = round_up(rows * out_dim * 2, kAlign) + linear_bwd_row_chunks(rows) * out_dim * 4 +
           (linear_bwd_dx_parts(rows, dim, out_dim) + linear_bwd_dw_parts(rows, dim, out_dim)) * 4;
  return XEMA_OK;
}

extern "C" int xema_op_linear_bwd(const xema_linear_bwd_args* args, void* stream) {
  XEMA_CHECK(check_linear_bwd(args));
  if (args->rows == 0 && !args->dw && !args->dbias) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_linear_bwd(*args, s));
}

extern "C" int xema_cross_attn_workspace_bytes(int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t q_len, int32_t kv_len,
                                               int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_cross_shape(batch, heads, kv_heads, head_dim, q_len, kv_len));
  *bytes = cross_attn_workspace({batch, heads, kv_heads, head_dim, q_len, kv_len});
  return XEMA_OK;
}

extern "C" int xema_op_cross_attn(const xema_cross_attn_args* args, void* stream) {
  XEMA_CHECK(check_cross_attn(args));
  if (args->batch == 0 || args->q_len == 0) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_cross_attn(*args, s));
}

extern "C" int xema_cross_attn_bwd_workspace_bytes(int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t q_len, int32_t kv_len,
                                                   int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_cross_shape(batch, heads, kv_heads, head_dim, q_len, kv_len));
  *bytes = cross_attn_bwd_workspace({batch, heads, kv_heads, head_dim, q_len, kv_len});
  return XEMA_OK;
}

extern "C" int xema_op_cross_attn_bwd(const xema_cross_attn_bwd_args* args, void* stream) {
  XEMA_CHECK(check_cross_attn_bwd(args));
  if (args->batch == 0 || (args->q_len == 0 && (!args->dk || args->kv_len == 0))) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_cross_attn_bwd(*args, s));
}
