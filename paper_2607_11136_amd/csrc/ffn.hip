// Host entry points of the feed-forward sub-block's operators (xema_ffn.h):
// argument validation, then the launches of k_norm.hip, k_ffn.hip and
// k_lora.hip.
#include "ffn.h"
#include "spans.h"
#include "xema_internal.h"

using namespace xema;

namespace {

// (a launch has fewer than 2^32 threads, and a row up to 256)
constexpr int64_t MAX_ROWS = ((int64_t)1 << 24) - 1, MAX_LD = (int64_t)1 << 21, MAX_WIDTH = 131072;

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int hip_status(hipError_t e) { return e == hipSuccess ? XEMA_OK : XEMA_ERR_HIP; }

int64_t elem(int dtype) { return dtype == XEMA_F32 ? 4 : dtype == XEMA_E4M3 ? 1 : 2; }
bool is16(int d) { return d == XEMA_BF16 || d == XEMA_F16; }
bool is_norm_type(int d) { return is16(d) || d == XEMA_F32; }

Span matrix(const void* p, int dtype, int64_t rows, int64_t width, int64_t ld) {
  return span_rows(p, width * elem(dtype), rows, ld * elem(dtype));
}

int check_rows(int64_t rows) {
  if (rows < 0) return XEMA_ERR_INVALID_ARG;
  return rows > MAX_ROWS ? XEMA_ERR_UNSUPPORTED : XEMA_OK;
}
int check_width(int64_t w, int dtype) {
  if (w <= 0) return XEMA_ERR_INVALID_ARG;
  return w % (dtype == XEMA_E4M3 ? 16 : 8) || w > MAX_WIDTH ? XEMA_ERR_UNSUPPORTED : XEMA_OK;
}
// The leading dimension and address of a matrix (p may be null if `optional`).
int check_matrix(const void* p, int dtype, int64_t width, int64_t ld, bool optional = false) {
  if (!p) return optional ? XEMA_OK : XEMA_ERR_INVALID_ARG;
  if (ld < width) return XEMA_ERR_INVALID_ARG;
  if (ld >= MAX_LD) return XEMA_ERR_UNSUPPORTED;
  return !aligned(p, 16) || ld * elem(dtype) % 16 ? XEMA_ERR_MISALIGNED : XEMA_OK;
}

// The stream of a call, which must belong to the current device, where the
// launches go.  The two handles that are no streams of their own, the default
// stream's and the calling thread's, do by their meaning, and are not asked about
// (hipStreamGetDevice follows the former as an address).
int take_stream(void* stream, hipStream_t* s) {
  *s = (hipStream_t)stream;
  if (*s == hipStreamLegacy) *s = nullptr;
  if (!*s || *s == hipStreamPerThread) return XEMA_OK;
  int device = 0;
  hipDevice_t of = 0;
  if (hipGetDevice(&device) != hipSuccess || hipStreamGetDevice(*s, &of) != hipSuccess) return XEMA_ERR_HIP;
  return of == device ? XEMA_OK : XEMA_ERR_INVALID_ARG;
}

#define XEMA_CHECK(call)               \
  do {                                 \
    const int st_ = (call);            \
    if (st_ != XEMA_OK) return st_;    \
  } while (0)

// In place: `out` may be this input, element for element.
bool same(const void* out, int dtype, int64_t ld, const void* in, int in_dtype, int64_t in_ld) {
  return out == in && dtype == in_dtype && ld == in_ld;
}

int check_rmsnorm(const xema_rmsnorm_args* a) {
  if (!a || !a->x || !a->y || !(a->eps > 0.f)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  if (!is_norm_type(a->x_dtype) || (a->resid && !is_norm_type(a->resid_dtype)) || (a->sum && !is_norm_type(a->sum_dtype)) ||
      !(is16(a->y_dtype) || a->y_dtype == XEMA_E4M3))
    return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_width(a->dim, a->y_dtype));
  if (a->dim > 16384) return XEMA_ERR_UNSUPPORTED;
  if (a->y_dtype == XEMA_E4M3 && !a->y_scale) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_matrix(a->x, a->x_dtype, a->dim, a->ldx));
  XEMA_CHECK(check_matrix(a->resid, a->resid_dtype, a->dim, a->ld_resid, true));
  XEMA_CHECK(check_matrix(a->sum, a->sum_dtype, a->dim, a->ld_sum, true));
  XEMA_CHECK(check_matrix(a->y, a->y_dtype, a->dim, a->ldy));
  if (!aligned(a->gamma, 16) || !aligned(a->y_scale, 4)) return XEMA_ERR_MISALIGNED;
  const Span x = matrix(a->x, a->x_dtype, a->rows, a->dim, a->ldx), res = matrix(a->resid, a->resid_dtype, a->rows, a->dim, a->ld_resid);
  const Span sum = matrix(a->sum, a->sum_dtype, a->rows, a->dim, a->ld_sum), y = matrix(a->y, a->y_dtype, a->rows, a->dim, a->ldy);
  const Span gamma{a->gamma, 2 * (int64_t)a->dim}, scale{a->y_dtype == XEMA_E4M3 ? a->y_scale : nullptr, 4 * a->rows};
  if (any_overlap(y, {x, res, sum, gamma, scale}) || any_overlap(scale, {x, res, sum, gamma}) || overlaps(sum, gamma))
    return XEMA_ERR_INVALID_ARG;
  if (overlaps(sum, x) && !same(a->sum, a->sum_dtype, a->ld_sum, a->x, a->x_dtype, a->ldx)) return XEMA_ERR_INVALID_ARG;
  if (overlaps(sum, res) && !same(a->sum, a->sum_dtype, a->ld_sum, a->resid, a->resid_dtype, a->ld_resid)) return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_rmsnorm_bwd(const xema_rmsnorm_bwd_args* a) {
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
  if (!aligned(a->gamma, 16) || !aligned(a->dgamma, 16) || !aligned(a->workspace, 16)) return XEMA_ERR_MISALIGNED;
  int64_t need = 0;
  XEMA_CHECK(xema_rmsnorm_bwd_workspace_bytes(a->rows, a->dim, &need));
  if (a->dgamma) {
    if (!a->workspace) return XEMA_ERR_INVALID_ARG;
    if (a->workspace_bytes < need) return XEMA_ERR_WORKSPACE_TOO_SMALL;
  }
  const Span s = matrix(a->s, a->s_dtype, a->rows, a->dim, a->ld_s), dy = matrix(a->dy, a->dy_dtype, a->rows, a->dim, a->ld_dy);
  const Span dsum = matrix(a->dsum, a->dsum_dtype, a->rows, a->dim, a->ld_dsum), dx = matrix(a->dx, a->dx_dtype, a->rows, a->dim, a->ld_dx);
  const Span gamma{a->gamma, 2 * (int64_t)a->dim}, dgamma{a->dgamma, 4 * (int64_t)a->dim}, ws{a->dgamma ? a->workspace : nullptr, need};
  if (any_overlap(dgamma, {s, dy, dsum, dx, gamma, ws}) || any_overlap(ws, {s, dy, dsum, dx, gamma}) || overlaps(dx, gamma))
    return XEMA_ERR_INVALID_ARG;
  if ((overlaps(dx, s) && !same(a->dx, a->dx_dtype, a->ld_dx, a->s, a->s_dtype, a->ld_s)) ||
      (overlaps(dx, dy) && !same(a->dx, a->dx_dtype, a->ld_dx, a->dy, a->dy_dtype, a->ld_dy)) ||
      (overlaps(dx, dsum) && !same(a->dx, a->dx_dtype, a->ld_dx, a->dsum, a->dsum_dtype, a->ld_dsum)))
    return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_gated(const xema_gated_ffn_args* a) {
  if (!a || !a->x || !a->gate_w || !a->up_w || !a->y) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  const bool f8 = a->dtype == XEMA_E4M3;
  if (!is16(a->dtype) && !f8) return XEMA_ERR_UNSUPPORTED;
  if (a->act != XEMA_ACT_SILU && a->act != XEMA_ACT_GELU_TANH) return XEMA_ERR_INVALID_ARG;
  if (!is16(a->y_dtype) || (!f8 && a->y_dtype != a->dtype) || (f8 && a->pre)) return XEMA_ERR_UNSUPPORTED;
  if (f8 && (!a->x_scale || !a->gate_scale || !a->up_scale)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_width(a->dim, a->dtype));
  XEMA_CHECK(check_width(a->hidden, XEMA_BF16));
  XEMA_CHECK(check_matrix(a->x, a->dtype, a->dim, a->ldx));
  XEMA_CHECK(check_matrix(a->gate_w, a->dtype, a->dim, a->dim));
  XEMA_CHECK(check_matrix(a->up_w, a->dtype, a->dim, a->dim));
  XEMA_CHECK(check_matrix(a->y, a->y_dtype, a->hidden, a->ldy));
  if (!aligned(a->pre, 16) || !aligned(a->gate_b, 16) || !aligned(a->up_b, 16)) return XEMA_ERR_MISALIGNED;
  if (f8 && (!aligned(a->x_scale, 4) || !aligned(a->gate_scale, 4) || !aligned(a->up_scale, 4))) return XEMA_ERR_MISALIGNED;
  const int64_t F = a->hidden, wb = F * a->dim * elem(a->dtype);
  const Span x = matrix(a->x, a->dtype, a->rows, a->dim, a->ldx), gw{a->gate_w, wb}, uw{a->up_w, wb};
  const Span gb{a->gate_b, 2 * F}, ub{a->up_b, 2 * F}, y = matrix(a->y, a->y_dtype, a->rows, F, a->ldy);
  const Span pre{a->pre, 6 * a->rows * F};
  const Span xs{f8 ? a->x_scale : nullptr, 4 * a->rows}, gs{f8 ? a->gate_scale : nullptr, 4 * F}, us{f8 ? a->up_scale : nullptr, 4 * F};
  if (any_overlap(y, {x, gw, uw, gb, ub, pre, xs, gs, us}) || any_overlap(pre, {x, gw, uw, gb, ub})) return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_gated_bwd(const xema_gated_ffn_bwd_args* a) {
  if (!a || !a->x || !a->gate_w || !a->up_w || !a->pre || !a->dy || !a->workspace) return XEMA_ERR_INVALID_ARG;
  if (!a->dgate_w != !a->dup_w || !a->dgate_b != !a->dup_b || (!a->dx && !a->dgate_w && !a->dgate_b)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  if (!is16(a->dtype)) return XEMA_ERR_UNSUPPORTED;
  if (a->act != XEMA_ACT_SILU && a->act != XEMA_ACT_GELU_TANH) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_width(a->dim, a->dtype));
  XEMA_CHECK(check_width(a->hidden, a->dtype));
  const int64_t F = a->hidden, D = a->dim;
  XEMA_CHECK(check_matrix(a->x, a->dtype, D, a->ldx));
  XEMA_CHECK(check_matrix(a->dy, a->dtype, F, a->ld_dy));
  XEMA_CHECK(check_matrix(a->dx, a->dtype, D, a->ld_dx, true));
  for (const void* p : {a->gate_w, a->up_w, a->pre, (const void*)a->dgate_w, (const void*)a->dup_w, (const void*)a->dgate_b,
                        (const void*)a->dup_b})
    if (!aligned(p, 16)) return XEMA_ERR_MISALIGNED;
  if (!aligned(a->workspace, 256)) return XEMA_ERR_MISALIGNED;
  int64_t need = 0;
  XEMA_CHECK(xema_gated_ffn_bwd_workspace_bytes(a->rows, a->dim, a->hidden, &need));
  if (a->workspace_bytes < need) return XEMA_ERR_WORKSPACE_TOO_SMALL;
  const Span x = matrix(a->x, a->dtype, a->rows, D, a->ldx), gw{a->gate_w, F * D * 2}, uw{a->up_w, F * D * 2};
  const Span pre{a->pre, 6 * a->rows * F}, dy = matrix(a->dy, a->dtype, a->rows, F, a->ld_dy);
  const Span dx = matrix(a->dx, a->dtype, a->rows, D, a->ld_dx), dgw{a->dgate_w, F * D * 2}, duw{a->dup_w, F * D * 2};
  const Span dgb{a->dgate_b, 2 * F}, dub{a->dup_b, 2 * F}, ws{a->workspace, need};
  if (any_overlap(ws, {x, gw, uw, pre, dy, dx, dgw, duw, dgb, dub}) || any_overlap(dx, {x, gw, uw, pre, dy, dgw, duw, dgb, dub}) ||
      any_overlap(dgw, {x, gw, uw, pre, dy, duw, dgb, dub}) || any_overlap(duw, {x, gw, uw, pre, dy, dgb, dub}) ||
      any_overlap(dgb, {x, gw, uw, pre, dy, dub}) || any_overlap(dub, {x, gw, uw, pre, dy}))
    return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

int check_lora(const xema_lora_args* a) {
  if (!a || !a->x || !a->w || !a->row_adapter || !a->y || !a->workspace || a->n_adapters < 0 || a->rank <= 0) return XEMA_ERR_INVALID_ARG;
  if (a->n_adapters && (!a->a || !a->b || !a->scale)) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(a->rows));
  if (!is16(a->dtype) || !is16(a->y_dtype) || a->rank % 8 || a->rank > 128) return XEMA_ERR_UNSUPPORTED;
  XEMA_CHECK(check_width(a->dim, a->dtype));
  XEMA_CHECK(check_width(a->out_dim, a->dtype));
  XEMA_CHECK(check_matrix(a->x, a->dtype, a->dim, a->ldx));
  XEMA_CHECK(check_matrix(a->w, a->dtype, a->dim, a->dim));
  XEMA_CHECK(check_matrix(a->y, a->y_dtype, a->out_dim, a->ldy));
  if (!aligned(a->bias, 16) || !aligned(a->a, 16) || !aligned(a->b, 16) || !aligned(a->scale, 4) || !aligned(a->row_adapter, 4) ||
      !aligned(a->workspace, 256))
    return XEMA_ERR_MISALIGNED;
  int64_t need = 0;
  XEMA_CHECK(xema_lora_workspace_bytes(a->rows, a->rank, &need));
  if (a->workspace_bytes < need) return XEMA_ERR_WORKSPACE_TOO_SMALL;
  const int64_t n = a->n_adapters;
  const Span x = matrix(a->x, a->dtype, a->rows, a->dim, a->ldx), w{a->w, 2 * (int64_t)a->out_dim * a->dim};
  const Span bias{a->bias, 2 * (int64_t)a->out_dim}, aa{n ? a->a : nullptr, 2 * n * a->rank * a->dim};
  const Span bb{n ? a->b : nullptr, 2 * n * a->rank * a->out_dim}, sc{n ? a->scale : nullptr, 4 * n}, ids{a->row_adapter, 4 * a->rows};
  const Span y = matrix(a->y, a->y_dtype, a->rows, a->out_dim, a->ldy), ws{a->workspace, need};
  if (any_overlap(y, {x, w, bias, aa, bb, sc, ids, ws}) || any_overlap(ws, {x, w, bias, aa, bb, sc, ids})) return XEMA_ERR_INVALID_ARG;
  return XEMA_OK;
}

}  // namespace

extern "C" int xema_op_rmsnorm(const xema_rmsnorm_args* args, void* stream) {
  XEMA_CHECK(check_rmsnorm(args));
  if (args->rows == 0) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_rmsnorm(*args, s));
}

extern "C" int xema_rmsnorm_bwd_workspace_bytes(int64_t rows, int32_t dim, int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(rows));
  XEMA_CHECK(check_width(dim, XEMA_BF16));
  if (dim > 16384) return XEMA_ERR_UNSUPPORTED;
  *bytes = rmsnorm_bwd_partials(rows) * dim * 4;
  return XEMA_OK;
}

extern "C" int xema_op_rmsnorm_bwd(const xema_rmsnorm_bwd_args* args, void* stream) {
  XEMA_CHECK(check_rmsnorm_bwd(args));
  if (args->rows == 0 && !args->dgamma) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_rmsnorm_bwd(*args, s));
}

extern "C" int xema_op_gated_ffn(const xema_gated_ffn_args* args, void* stream) {
  XEMA_CHECK(check_gated(args));
  if (args->rows == 0) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_gated_ffn(*args, s));
}

extern "C" int xema_gated_ffn_pre_bytes(int64_t rows, int32_t hidden, int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(rows));
  XEMA_CHECK(check_width(hidden, XEMA_BF16));
  *bytes = 6 * rows * hidden;
  return XEMA_OK;
}

extern "C" int xema_gated_ffn_bwd_workspace_bytes(int64_t rows, int32_t dim, int32_t hidden, int64_t* bytes) {
  if (!bytes) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(rows));
  XEMA_CHECK(check_width(dim, XEMA_BF16));
  XEMA_CHECK(check_width(hidden, XEMA_BF16));
  // dg, du in 16 bits, the partial column sums of both, and the partial sums of dx and of the weights' gradients
  *bytes = 2 * round_up(rows * hidden * 2, kAlign) + gated_bwd_row_chunks(rows) * 2 * hidden * 4 +
           (gated_bwd_dx_parts(rows, dim, hidden) + gated_bwd_dw_parts(rows, dim, hidden)) * 4;
  return XEMA_OK;
}

extern "C" int xema_op_gated_ffn_bwd(const xema_gated_ffn_bwd_args* args, void* stream) {
  XEMA_CHECK(check_gated_bwd(args));
  if (args->rows == 0 && !args->dgate_w && !args->dgate_b) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_gated_ffn_bwd(*args, s));
}

extern "C" int xema_lora_workspace_bytes(int64_t rows, int32_t rank, int64_t* bytes) {
  if (!bytes || rank <= 0) return XEMA_ERR_INVALID_ARG;
  XEMA_CHECK(check_rows(rows));
  if (rank % 8 || rank > 128) return XEMA_ERR_UNSUPPORTED;
  *bytes = round_up(rows > 0 ? rows * 2 * rank * 2 : 1, kAlign);
  return XEMA_OK;
}

extern "C" int xema_op_lora_linear(const xema_lora_args* args, void* stream) {
  XEMA_CHECK(check_lora(args));
  if (args->rows == 0) return XEMA_OK;
  hipStream_t s;
  XEMA_CHECK(take_stream(stream, &s));
  return hip_status(launch_lora_linear(*args, s));
}
