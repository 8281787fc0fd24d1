// Checks that the host entry points of the operators share: types, widths,
// leading dimensions and alignment of matrices, and the stream of a call.
#pragma once

#include <hip/hip_runtime.h>

#include "spans.h"
#include "xema_ops.h"

namespace xema {

// (a launch has fewer than 2^32 threads, and a row up to 256)
constexpr int64_t MAX_ROWS = ((int64_t)1 << 24) - 1, MAX_LD = (int64_t)1 << 21, MAX_WIDTH = 131072;

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline int hip_status(hipError_t e) { return e == hipSuccess ? XEMA_OK : XEMA_ERR_HIP; }

inline int64_t elem(int dtype) { return dtype == XEMA_F32 ? 4 : dtype == XEMA_E4M3 ? 1 : 2; }
inline bool is16(int d) { return d == XEMA_BF16 || d == XEMA_F16; }
inline bool is_norm_type(int d) { return is16(d) || d == XEMA_F32; }

inline Span matrix(const void* p, int dtype, int64_t rows, int64_t width, int64_t ld) {
  return span_rows(p, width * elem(dtype), rows, ld * elem(dtype));
}

inline int check_rows(int64_t rows) {
  if (rows < 0) return XEMA_ERR_INVALID_ARG;
  return rows > MAX_ROWS ? XEMA_ERR_UNSUPPORTED : XEMA_OK;
}
inline int check_width(int64_t w, int dtype) {
  if (w <= 0) return XEMA_ERR_INVALID_ARG;
  return w % (dtype == XEMA_E4M3 ? 16 : 8) || w > MAX_WIDTH ? XEMA_ERR_UNSUPPORTED : XEMA_OK;
}
// The leading dimension and address of a matrix (p may be null if `optional`).
inline int check_matrix(const void* p, int dtype, int64_t width, int64_t ld, bool optional = false) {
  if (!p) return optional ? XEMA_OK : XEMA_ERR_INVALID_ARG;
  if (ld < width) return XEMA_ERR_INVALID_ARG;
  if (ld >= MAX_LD) return XEMA_ERR_UNSUPPORTED;
  return !aligned(p, 16) || ld * elem(dtype) % 16 ? XEMA_ERR_MISALIGNED : XEMA_OK;
}

// The stream of a call, which must belong to the current device, where the
// launches go.  The two handles that are no streams of their own, the default
// stream's and the calling thread's, do by their meaning, and are not asked about
// (hipStreamGetDevice follows the former as an address).
inline int take_stream(void* stream, hipStream_t* s) {
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
inline bool same(const void* out, int dtype, int64_t ld, const void* in, int in_dtype, int64_t in_ld) {
  return out == in && dtype == in_dtype && ld == in_ld;
}

}  // namespace xema
