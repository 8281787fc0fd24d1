// What the matrix kernels share: the MFMAs, loads straight into LDS, the
// swizzle of 128-byte LDS rows, and small loads and stores of epilogues.
#pragma once

#include "device_common.h"

namespace xema {

template <typename T>
struct Mfma;
template <>
struct Mfma<bf16> {
  typedef bf16x8 frag;
  static __device__ __forceinline__ f32x16 run(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 run16(frag a, frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<f16> {
  typedef f16x8 frag;
  static __device__ __forceinline__ f32x16 run(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 run16(frag a, frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

// slot swizzle of a 128-byte row (two rows share a 256-byte bank line)
__host__ __device__ constexpr int row_swz(int r) { return (r >> 1) & 7; }
constexpr int BUF_FLAGS = 0x00020000;      // raw buffer, 32-bit dwords

// 16 bytes per lane from buffer offset voff + soff straight into LDS (one
// 1 KiB wave row at dst).  The host pass cannot check this builtin with a
// run-time scalar offset, so it sees an empty body.
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t r, uint8_t* dst, uint32_t voff,
                                           uint32_t soff) {
#if __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)dst, 16, voff, soff, 0, 0);
#endif
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes,
                                           BUF_FLAGS);
}

template <typename RT>
__device__ __forceinline__ void load4f(const RT* p, float v[4]);
template <>
__device__ __forceinline__ void load4f<float>(const float* p, float v[4]) {
  const f32x4 u = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = u[e];
}
template <>
__device__ __forceinline__ void load4f<uint16_t>(const uint16_t* p, float v[4]) {
  const u32x2 u = *reinterpret_cast<const u32x2*>(p);
  v[0] = __uint_as_float(u[0] << 16);
  v[1] = __uint_as_float(u[0] & 0xffff0000u);
  v[2] = __uint_as_float(u[1] << 16);
  v[3] = __uint_as_float(u[1] & 0xffff0000u);
}

// s_waitcnt immediate: vmcnt[3:0] in bits 3:0 and vmcnt[5:4] in bits 15:14,
// expcnt in bits 6:4 (7 = no wait), lgkmcnt in bits 11:8 (0 = wait for all).
constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4); }

// Two 16-column blocks of one row, of which a lane of 16-lane row l4 holds
// columns 4 l4 .. 4 l4 + 3 each (a, b): rows 2m and 2m + 1 swap halves, then
// the first stores 8 columns of block a and the second of block b, 16 bytes
// apiece.  `base` points at block a.
template <typename CT>
__device__ __forceinline__ void store_block_pair(CT* base, const CT __attribute__((ext_vector_type(4))) a,
                                                 const CT __attribute__((ext_vector_type(4))) b, int l4, bool valid) {
  typedef CT c4 __attribute__((ext_vector_type(4)));
  static_assert(sizeof(c4) == 8, "16-bit elements");
  const u32x2 ua = __builtin_bit_cast(u32x2, a), ub = __builtin_bit_cast(u32x2, b);
  const auto r0 = __builtin_amdgcn_permlane16_swap(ua[0], ub[0], false, false);
  const auto r1 = __builtin_amdgcn_permlane16_swap(ua[1], ub[1], false, false);
  const u32x4 o = {r0[0], r1[0], r0[1], r1[1]};
  if (valid) *reinterpret_cast<u32x4*>(base + 16 * (l4 & 1) + 8 * (l4 >> 1)) = o;
}

}  // namespace xema
