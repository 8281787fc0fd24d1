// Launch functions of the cross-attention sub-block's kernels (xema_cross.h).
#pragma once

#include <hip/hip_runtime.h>

#include "xema_cross.h"

namespace xema {

hipError_t launch_layernorm(const xema_layernorm_args& a, hipStream_t s);
int64_t layernorm_bwd_partials(int64_t rows);     // partial sums, each fp32 [2][dim]
hipError_t launch_layernorm_bwd(const xema_layernorm_bwd_args& a, hipStream_t s);

hipError_t launch_linear(const xema_linear_args& a, hipStream_t s);
int64_t linear_bwd_row_chunks(int64_t rows);      // partial column sums of dz, each fp32 [out_dim]
int64_t linear_bwd_dx_parts(int64_t rows, int dim, int out_dim);   // floats, where dx's k is split
int64_t linear_bwd_dw_parts(int64_t rows, int dim, int out_dim);   // and where the weight's gradient's is
hipError_t launch_linear_bwd(const xema_linear_bwd_args& a, hipStream_t s);

// Sizes of an attention call, whatever its pointers.
struct CrossShape {
  int batch, heads, kv_heads, head_dim, q_len, kv_len;
};
int64_t cross_attn_workspace(const CrossShape& c);
hipError_t launch_cross_attn(const xema_cross_attn_args& a, hipStream_t s);
int64_t cross_attn_bwd_workspace(const CrossShape& c);
hipError_t launch_cross_attn_bwd(const xema_cross_attn_bwd_args& a, hipStream_t s);

}  // namespace xema
