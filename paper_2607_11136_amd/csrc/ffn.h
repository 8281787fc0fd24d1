// Launch functions of the feed-forward sub-block's kernels (xema_ffn.h).
#pragma once

#include <hip/hip_runtime.h>

#include "xema_ffn.h"

namespace xema {

hipError_t launch_rmsnorm(const xema_rmsnorm_args& a, hipStream_t s);
int64_t rmsnorm_bwd_partials(int64_t rows);       // partial sums of dgamma, each fp32 [dim]
hipError_t launch_rmsnorm_bwd(const xema_rmsnorm_bwd_args& a, hipStream_t s);

hipError_t launch_gated_ffn(const xema_gated_ffn_args& a, hipStream_t s);
int64_t gated_bwd_row_chunks(int64_t rows);       // partial column sums of dg and du
int64_t gated_bwd_dx_parts(int64_t rows, int dim, int hidden);   // floats, where dx's k is split
int64_t gated_bwd_dw_parts(int64_t rows, int dim, int hidden);   // and where the weights' gradients' is
hipError_t launch_gated_ffn_bwd(const xema_gated_ffn_bwd_args& a, hipStream_t s);

hipError_t launch_lora_linear(const xema_lora_args& a, hipStream_t s);

}  // namespace xema
