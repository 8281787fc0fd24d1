// RMS norm with the residual's addition and 16- or 8-bit output, and its
// gradient (xema_ffn.h).  Bound by HBM: a row is read once, held in registers
// as fp32 and written once.  A wave takes a row of up to 2048 elements (no
// barrier), a workgroup a wider one.  57224 x 4096 (bf16 and an fp32 residual, 8-bit
// output, 2.58 GB) 446 us, 5.8 TB/s; 1539 x 2568 9 us; the gradient of 16384 x 4096
// (0.54 GB) 107 us and 5 us for dgamma, whose parts (a row of sums for each of up
// to 1024 workgroups) are 3% of the traffic.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "ffn.h"
#include "row_io.h"

namespace xema {

namespace {

template <int WPR>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* red, int wave) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < WPR; ++w) v = max(v, red[w]);
  }
  return v;
}

// 2^k, the smallest with |v| <= 448 * 2^k and k >= -126, for the magnitude
// bits of |v|; NaN for infinity and NaN.  448 is 1.75 * 2^8, so k is v's
// exponent less 8, and one more where its significand is above 1.75.
__device__ __forceinline__ float e4m3_scale(uint32_t bits) {
  if (bits >= 0x7f800000u) return __builtin_nanf("");
  const int k = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(k, -126) + 127) << 23);
}

// Eight e4m3 codes of f / scale, 1 / scale = inv exactly.
__device__ __forceinline__ u32x2 e4m3_codes(const float f[8], float inv) {
  u32x2 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h] * inv, f[4 * h + 1] * inv, 0, false);
    o[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2] * inv, f[4 * h + 3] * inv, w, true);
  }
  return o;
}

constexpr int NORM_WAVES = 4;     // per workgroup

// A row is held by WPR waves (1, or all 4 of the workgroup) in NV vectors of
// eight a lane: vector v of a lane starts at (v * 64 * WPR + lane) * 8, so a
// wave's loads are contiguous.  RT void: no residual.
template <typename XT, typename RT, int NV, int WPR>
__global__ __launch_bounds__(NORM_WAVES * 64) void k_rmsnorm(xema_rmsnorm_args a) {
  constexpr bool RESID = !std::is_void_v<RT>;
  typedef std::conditional_t<RESID, RT, bf16> R;
  __shared__ float red[NORM_WAVES];
  __shared__ uint32_t red_max[NORM_WAVES];
  const int wave = threadIdx.x >> 6, in_row = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t r = WPR == 1 ? (int64_t)blockIdx.x * NORM_WAVES + wave : (int64_t)blockIdx.x;
  if (r >= a.rows) return;
  const XT* x = (const XT*)a.x + r * a.ldx;
  const R* res = (const R*)a.resid + r * a.ld_resid;
  Raw8<XT> rx[NV];
  Raw8<R> rr[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * 64 * WPR + in_row) * 8;
    if (c < a.dim) {
      rx[v] = load_raw8(x + c);
      if (RESID) rr[v] = load_raw8(res + c);
    }
  }
  float s[NV][8];
  float ss = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * 64 * WPR + in_row) * 8;
    if (c < a.dim) {
      unpack8(rx[v], s[v]);
      if constexpr (RESID) {
        float f[8];
        unpack8(rr[v], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[v][e] += f[e];
      }
      if (a.sum) store8(a.sum, a.sum_dtype, r * a.ld_sum + c, s[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(s[v][e], s[v][e], ss);
    }
  }
  ss = row_sum<WPR>(ss, red, wave);
  const float q = 1.0f / sqrtf(ss / (float)a.dim + a.eps);
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * 64 * WPR + in_row) * 8;
    if (c < a.dim) {
      float g[8];
      if (a.gamma) unpack8(load_raw8((const bf16*)a.gamma + c), g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[v][e] *= q;
        if (a.gamma) s[v][e] *= g[e];
        top = max(top, __float_as_uint(s[v][e]) & 0x7fffffffu);
      }
      if (a.y_dtype != XEMA_E4M3) store8(a.y, a.y_dtype, r * a.ldy + c, s[v]);
    }
  }
  if (a.y_dtype != XEMA_E4M3) return;
  // (an infinity in s gives NaN and zeros: the largest magnitude is NaN too)
  const float scale = e4m3_scale(row_max<WPR>(top, red_max, wave));
  if (in_row == 0) a.y_scale[r] = scale;
  // 2^-k: exact, and a normal number for every k from -126 to 120
  const float inv = 1.0f / scale;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * 64 * WPR + in_row) * 8;
    if (c < a.dim) *reinterpret_cast<u32x2*>((uint8_t*)a.y + r * a.ldy + c) = e4m3_codes(s[v], inv);
  }
}

template <typename XT, typename RT, int WPR>
hipError_t rmsnorm_nv(const xema_rmsnorm_args& a, hipStream_t s) {
  const dim3 grid((unsigned)(WPR == 1 ? (a.rows + NORM_WAVES - 1) / NORM_WAVES : a.rows)), block(NORM_WAVES * 64);
  const int nv = (a.dim + 512 * WPR - 1) / (512 * WPR);
  if (nv <= 1) hipLaunchKernelGGL((k_rmsnorm<XT, RT, 1, WPR>), grid, block, 0, s, a);
  else if (nv <= 2) hipLaunchKernelGGL((k_rmsnorm<XT, RT, 2, WPR>), grid, block, 0, s, a);
  else if (nv <= 4) hipLaunchKernelGGL((k_rmsnorm<XT, RT, 4, WPR>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_rmsnorm<XT, RT, 8, WPR>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename XT, typename RT>
hipError_t rmsnorm_t(const xema_rmsnorm_args& a, hipStream_t s) {
  return a.dim <= 2048 ? rmsnorm_nv<XT, RT, 1>(a, s) : rmsnorm_nv<XT, RT, NORM_WAVES>(a, s);
}
template <typename XT>
hipError_t rmsnorm_x(const xema_rmsnorm_args& a, hipStream_t s) {
  if (!a.resid) return rmsnorm_t<XT, void>(a, s);
  switch (a.resid_dtype) {
    case XEMA_BF16: return rmsnorm_t<XT, bf16>(a, s);
    case XEMA_F16: return rmsnorm_t<XT, f16>(a, s);
    default: return rmsnorm_t<XT, float>(a, s);
  }
}

// The gradient.  Workgroup b takes the rows b, b + grid, ... (WPR = 4) or the
// groups of four rows b, b + grid, ... (WPR = 1), holds its part of dgamma in
// registers over them and writes it once.  A row's s, dy and dsum are loaded
// while the row before is computed.  ST void: no dsum.
template <typename XT, typename DT, typename ST, int NV>
struct BwdRow {
  typedef std::conditional_t<std::is_void_v<ST>, bf16, ST> S;
  Raw8<XT> x[NV];
  Raw8<DT> d[NV];
  Raw8<S> ds[std::is_void_v<ST> ? 1 : NV];
  template <int STRIDE>
  __device__ __forceinline__ void load(const xema_rmsnorm_bwd_args& a, int64_t r, int in_row) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) {
        x[v] = load_raw8((const XT*)a.s + r * a.ld_s + c);
        d[v] = load_raw8((const DT*)a.dy + r * a.ld_dy + c);
        if constexpr (!std::is_void_v<ST>) ds[v] = load_raw8((const ST*)a.dsum + r * a.ld_dsum + c);
      }
    }
  }
};

template <typename XT, typename DT, typename ST, int NV, int WPR>
__global__ __launch_bounds__(NORM_WAVES * 64) void k_rmsnorm_bwd(xema_rmsnorm_bwd_args a, float* __restrict__ partial) {
  constexpr int STRIDE = 512 * WPR;
  __shared__ float red[2][2][NORM_WAVES];
  __shared__ float fold[WPR == 1 ? NORM_WAVES : 1][WPR == 1 ? NV * 512 : 1];
  const int wave = threadIdx.x >> 6, in_row = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  float dg[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[v][e] = 0.f;
  const int64_t first = WPR == 1 ? (int64_t)blockIdx.x * NORM_WAVES + wave : (int64_t)blockIdx.x;
  const int64_t step = (int64_t)gridDim.x * (WPR == 1 ? NORM_WAVES : 1);
  int turn = 0;
  BwdRow<XT, DT, ST, NV> next;
  if (first < a.rows) next.template load<STRIDE>(a, first, in_row);
  for (int64_t r = first; r < a.rows; r += step, turn ^= 1) {
    const BwdRow<XT, DT, ST, NV> row = next;
    if (r + step < a.rows) next.template load<STRIDE>(a, r + step, in_row);
    float ss = 0.f, gx = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) {
        float x[8], g[8], gam[8];
        unpack8(row.x[v], x);
        unpack8(row.d[v], g);
        if (a.gamma) unpack8(load_raw8((const bf16*)a.gamma + c), gam);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ss = fmaf(x[e], x[e], ss);
          gx = fmaf(a.gamma ? g[e] * gam[e] : g[e], x[e], gx);
        }
      }
    }
    ss = wave_sum(ss);
    gx = wave_sum(gx);
    if constexpr (WPR > 1) {
      if ((threadIdx.x & 63) == 0) {
        red[turn][0][wave] = ss;
        red[turn][1][wave] = gx;
      }
      __syncthreads();   // (the next row writes the other half)
      ss = gx = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) {
        ss += red[turn][0][w];
        gx += red[turn][1][w];
      }
    }
    const float q = 1.0f / sqrtf(ss / (float)a.dim + a.eps);
    const float along = gx * q / (float)a.dim;      // mean(g n)
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) {
        float x[8], g[8], gam[8], ds[8], o[8];
        unpack8(row.x[v], x);
        unpack8(row.d[v], g);
        if (a.gamma) unpack8(load_raw8((const bf16*)a.gamma + c), gam);
        if constexpr (!std::is_void_v<ST>) unpack8(row.ds[v], ds);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float n = x[e] * q;
          dg[v][e] = fmaf(g[e], n, dg[v][e]);
          o[e] = q * ((a.gamma ? g[e] * gam[e] : g[e]) - n * along);
          if constexpr (!std::is_void_v<ST>) o[e] += ds[e];
        }
        store8(a.dx, a.dx_dtype, r * a.ld_dx + c, o);
      }
    }
  }
  if (!partial) return;
  if constexpr (WPR == 1) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) fold[wave][v * 512 + in_row * 8 + e] = dg[v][e];
    __syncthreads();
    for (int c = threadIdx.x; c < a.dim; c += NORM_WAVES * 64) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < NORM_WAVES; ++w) s += fold[w][c];
      partial[(int64_t)blockIdx.x * a.dim + c] = s;
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) store8_as<float>(partial, (int64_t)blockIdx.x * a.dim + c, dg[v]);
    }
  }
}

// dgamma: the workgroups' parts, in order.  64 columns a workgroup, a part of
// the parts for each of its 16 waves, eight loads in flight.
__global__ __launch_bounds__(1024) void k_rmsnorm_dgamma(const float* __restrict__ partial, int parts, int dim, float* __restrict__ dgamma) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = (int)blockIdx.x * 64 + lane;
  const int p0 = parts * wave / 16, p1 = parts * (wave + 1) / 16;
  float s = 0.f;
  if (c < dim) {
#pragma unroll 8
    for (int i = p0; i < p1; ++i) s += partial[(int64_t)i * dim + c];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave || c >= dim) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += red[w][lane];
  dgamma[c] = s;
}

template <typename XT, typename DT, typename ST, int WPR>
void rmsnorm_bwd_nv(const xema_rmsnorm_bwd_args& a, float* partial, hipStream_t s) {
  const dim3 grid((unsigned)rmsnorm_bwd_partials(a.rows)), block(NORM_WAVES * 64);
  const int nv = (a.dim + 512 * WPR - 1) / (512 * WPR);
  if (nv <= 1) hipLaunchKernelGGL((k_rmsnorm_bwd<XT, DT, ST, 1, WPR>), grid, block, 0, s, a, partial);
  else if (nv <= 2) hipLaunchKernelGGL((k_rmsnorm_bwd<XT, DT, ST, 2, WPR>), grid, block, 0, s, a, partial);
  else if (nv <= 4) hipLaunchKernelGGL((k_rmsnorm_bwd<XT, DT, ST, 4, WPR>), grid, block, 0, s, a, partial);
  else if constexpr (WPR > 1) hipLaunchKernelGGL((k_rmsnorm_bwd<XT, DT, ST, 8, WPR>), grid, block, 0, s, a, partial);
}

template <typename XT, typename DT, typename ST>
void rmsnorm_bwd_t(const xema_rmsnorm_bwd_args& a, float* partial, hipStream_t s) {
  if (a.dim <= 2048) rmsnorm_bwd_nv<XT, DT, ST, 1>(a, partial, s);
  else rmsnorm_bwd_nv<XT, DT, ST, NORM_WAVES>(a, partial, s);
}
template <typename XT, typename DT>
void rmsnorm_bwd_d(const xema_rmsnorm_bwd_args& a, float* partial, hipStream_t s) {
  if (!a.dsum) return rmsnorm_bwd_t<XT, DT, void>(a, partial, s);
  switch (a.dsum_dtype) {
    case XEMA_BF16: return rmsnorm_bwd_t<XT, DT, bf16>(a, partial, s);
    case XEMA_F16: return rmsnorm_bwd_t<XT, DT, f16>(a, partial, s);
    default: return rmsnorm_bwd_t<XT, DT, float>(a, partial, s);
  }
}
template <typename XT>
void rmsnorm_bwd_x(const xema_rmsnorm_bwd_args& a, float* partial, hipStream_t s) {
  switch (a.dy_dtype) {
    case XEMA_BF16: return rmsnorm_bwd_d<XT, bf16>(a, partial, s);
    case XEMA_F16: return rmsnorm_bwd_d<XT, f16>(a, partial, s);
    default: return rmsnorm_bwd_d<XT, float>(a, partial, s);
  }
}

}  // namespace

hipError_t launch_rmsnorm(const xema_rmsnorm_args& a, hipStream_t s) {
  switch (a.x_dtype) {
    case XEMA_BF16: return rmsnorm_x<bf16>(a, s);
    case XEMA_F16: return rmsnorm_x<f16>(a, s);
    default: return rmsnorm_x<float>(a, s);
  }
}

int64_t rmsnorm_bwd_partials(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(1024, (rows + 3) / 4)); }

hipError_t launch_rmsnorm_bwd(const xema_rmsnorm_bwd_args& a, hipStream_t s) {
  float* partial = a.dgamma ? (float*)a.workspace : nullptr;
  int parts = 0;
  if (a.rows > 0) {
    parts = (int)rmsnorm_bwd_partials(a.rows);
    switch (a.s_dtype) {
      case XEMA_BF16: rmsnorm_bwd_x<bf16>(a, partial, s); break;
      case XEMA_F16: rmsnorm_bwd_x<f16>(a, partial, s); break;
      default: rmsnorm_bwd_x<float>(a, partial, s); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.dgamma) return hipSuccess;
  hipLaunchKernelGGL(k_rmsnorm_dgamma, dim3((a.dim + 63) / 64), dim3(1024), 0, s, partial, parts, a.dim, a.dgamma);
  return hipGetLastError();
}

}  // namespace xema
