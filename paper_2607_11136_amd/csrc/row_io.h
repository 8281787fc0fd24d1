// Rows of the norms: eight elements at a time between memory and fp32
// registers, and sums over the waves of a row.
#pragma once

#include "device_common.h"
#include "xema_ops.h"

namespace xema {

// Eight consecutive elements as fp32, from 16-byte loads.
template <typename T>
struct Raw8 {
  u32x4 v[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = reinterpret_cast<const u32x4*>(p)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float f[8]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  const t8 t = __builtin_bit_cast(t8, r);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (float)t[e];
}

template <typename T>
__device__ __forceinline__ void store8_as(void* p, int64_t at, const float f[8]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  t8 t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = (T)f[e];
  *reinterpret_cast<t8*>((T*)p + at) = t;
}
__device__ __forceinline__ void store8(void* p, int dtype, int64_t at, const float f[8]) {
  if (dtype == XEMA_BF16) store8_as<bf16>(p, at, f);
  else if (dtype == XEMA_F16) store8_as<f16>(p, at, f);
  else store8_as<float>(p, at, f);
}
// Sum over the WPR waves of a row (fixed order: within each wave, then over
// the waves); `red` holds WPR floats per use.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* red, int wave) {
  v = wave_sum(v);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < WPR; ++w) v += red[w];
  }
  return v;
}

}  // namespace xema
