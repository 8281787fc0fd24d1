// What the products of the feed-forward and linear layers share around their
// tiles: activations, values kept in 24 bits for the gradient, stores of a
// tile, and the sum of a product's parts.
#pragma once

#include "device_common.h"
#include "mma_tile.h"
#include "xema_ffn.h"

namespace xema {

namespace {      // (kernels of each source that includes this)

// act(g), and act'(g) where asked.  GELU's tanh form is g p with
// p = 1 / (1 + e^(-2z)), z = sqrt(2/pi) (g + 0.044715 g^3), so its slope is
// p + g p (1 - p) 2 z'; past |g| = 30 p is 0 or 1 in fp32 and the second term 0.
template <bool SLOPE>
__device__ __forceinline__ float activate(float g, int act, float* slope) {
  constexpr float LOG2E = 1.4426950408889634f;
  if (act == XEMA_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * g));
    if (SLOPE) *slope = s * fmaf(g, 1.0f - s, 1.0f);
    return g * s;
  }
  constexpr float A2 = 2.0f * 0.7978845608028654f;
  const float p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-A2 * LOG2E * fmaf(0.044715f * g, g * g, g)));
  if (SLOPE) {
    const float c = fminf(fmaxf(g, -30.0f), 30.0f);
    *slope = fmaf(c * p * (1.0f - p), A2 * fmaf(3.0f * 0.044715f * c, c, 1.0f), p);
  }
  return g * p;
}

// The upper 24 bits of fp32, rounded to nearest even (infinities and NaN keep
// their upper bits, and a NaN stays one).
__device__ __forceinline__ uint32_t round24(float v) {
  const uint32_t b = __float_as_uint(v);
  if ((b & 0x7f800000u) == 0x7f800000u) return b | (b & 0x7fffffu ? 0x400000u : 0u);
  return b + 0x7fu + (b >> 8 & 1u);
}
// Element e of one of the two, from its upper halves and third bytes.
__device__ __forceinline__ float load24(const uint32_t* upper, uint32_t low, int e) {
  const uint32_t hi = e & 1 ? upper[e >> 1] & 0xffff0000u : upper[e >> 1] << 16;
  return __uint_as_float(hi | (low >> (8 * e) & 0xffu) << 8);
}

// The tile's accumulators as rows row0 + ... of a [rows, cols] matrix.
template <typename T, typename S>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[S::MI][S::NJ], T* out, int64_t ld, int64_t row0, int64_t rows, int col0, int cols,
                                           int lane) {
  const int l16 = lane & 15, l4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const int64_t m = row0 + 16 * i + l16;
    const bool valid = m < rows;
    float v[S::NJ][4];
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j][e] = acc[i][j][e];
    store_row<T, S::NJ>(out + (valid ? m : 0) * ld, col0, cols, v, l4, valid);
  }
}

// The same in fp32.
template <typename S>
__device__ __forceinline__ void store_sums(const f32x4 (&acc)[S::MI][S::NJ], float* out, int64_t ld, int64_t row0, int64_t rows, int col0, int cols,
                                           int lane) {
  const int l16 = lane & 15, l4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const int64_t m = row0 + 16 * i + l16;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int c = col0 + 16 * j + 4 * l4;
      if (m < rows && c < cols) *reinterpret_cast<f32x4*>(out + m * ld + c) = acc[i][j];
    }
  }
}

// Outputs from their parts, in order: n elements in rows of `width`, those from
// `half` on belonging to out1.
template <typename T>
__global__ __launch_bounds__(256) void k_gated_sum(const float* __restrict__ sums, int parts, int64_t n, int width, T* __restrict__ out0,
                                                   T* __restrict__ out1, int64_t half, int64_t ld) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= n) return;
  f32x4 s = *reinterpret_cast<const f32x4*>(sums + at);
#pragma unroll 4
  for (int i = 1; i < parts; ++i) s += *reinterpret_cast<const f32x4*>(sums + i * n + at);
  t4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (T)s[e];
  const int64_t in = at < half ? at : at - half, r = in / width;
  *reinterpret_cast<t4*>((at < half ? out0 : out1) + r * ld + (in - r * width)) = o;
}

template <typename T>
hipError_t run_sum(const float* sums, int parts, int64_t n, int width, T* out0, T* out1, int64_t half, int64_t ld, hipStream_t s) {
  hipLaunchKernelGGL((k_gated_sum<T>), dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, s, sums, parts, n, width, out0, out1, half, ld);
  return hipGetLastError();
}

template <typename S>
__host__ __device__ constexpr int tiles_of(int64_t rows, int cols) {
  return (int)((rows + S::BM - 1) / S::BM) * ((cols + S::BN - 1) / S::BN);
}

// Where a tile goes: rows row0 + ... of [rows, cols], to `out`, or its sums to
// `sums` where it has a part of k alone.
template <typename T>
struct TileOut {
  T* out;
  float* sums;
  int64_t ld, row0, rows;
  int col0, cols;
};

}  // namespace

}  // namespace xema
