// Layer norm with the residual's addition, and its gradient (xema_cross.h).
// Bound by HBM: a row is read once, held in registers as fp32 and written
// once; the variance is taken about the mean, from the registers.  A wave takes
// a row of up to 2048 elements (no barrier), a workgroup a wider one.
#include <algorithm>
#include <type_traits>

#include "cross.h"
#include "device_common.h"
#include "row_io.h"

namespace xema {

namespace {

constexpr int LN_WAVES = 4;       // per workgroup

// A row is held by WPR waves (1, or all 4 of the workgroup) in NV vectors of
// eight a lane: vector v of a lane starts at (v * 64 * WPR + lane) * 8, so a
// wave's loads are contiguous.  RT void: no residual.
template <typename XT, typename RT, int NV, int WPR>
__global__ __launch_bounds__(LN_WAVES * 64) void k_layernorm(xema_layernorm_args a) {
  constexpr bool RESID = !std::is_void_v<RT>;
  typedef std::conditional_t<RESID, RT, bf16> R;
  __shared__ float red[2][LN_WAVES];
  const int wave = threadIdx.x >> 6, in_row = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t r = WPR == 1 ? (int64_t)blockIdx.x * LN_WAVES + wave : (int64_t)blockIdx.x;
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
  float total = 0.f;
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
      for (int e = 0; e < 8; ++e) total += s[v][e];
    }
  }
  const float mean = row_sum<WPR>(total, red[0], wave) / (float)a.dim;
  float ss = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * 64 * WPR + in_row) * 8;
    if (c < a.dim) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[v][e] -= mean;
        ss = fmaf(s[v][e], s[v][e], ss);
      }
    }
  }
  const float q = 1.0f / sqrtf(row_sum<WPR>(ss, red[1], wave) / (float)a.dim + a.eps);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * 64 * WPR + in_row) * 8;
    if (c < a.dim) {
      float g[8], b[8];
      if (a.gamma) unpack8(load_raw8((const bf16*)a.gamma + c), g);
      if (a.beta) unpack8(load_raw8((const bf16*)a.beta + c), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[v][e] *= q;
        if (a.gamma) s[v][e] *= g[e];
        if (a.beta) s[v][e] += b[e];
      }
      store8(a.y, a.y_dtype, r * a.ldy + c, s[v]);
    }
  }
}

template <typename XT, typename RT, int WPR>
void layernorm_nv(const xema_layernorm_args& a, hipStream_t s) {
  const dim3 grid((unsigned)(WPR == 1 ? (a.rows + LN_WAVES - 1) / LN_WAVES : a.rows)), block(LN_WAVES * 64);
  const int nv = (a.dim + 512 * WPR - 1) / (512 * WPR);
  if (nv <= 1) hipLaunchKernelGGL((k_layernorm<XT, RT, 1, WPR>), grid, block, 0, s, a);
  else if (nv <= 2) hipLaunchKernelGGL((k_layernorm<XT, RT, 2, WPR>), grid, block, 0, s, a);
  else if (nv <= 4) hipLaunchKernelGGL((k_layernorm<XT, RT, 4, WPR>), grid, block, 0, s, a);
  else if constexpr (WPR > 1) hipLaunchKernelGGL((k_layernorm<XT, RT, 8, WPR>), grid, block, 0, s, a);
}

template <typename XT, typename RT>
void layernorm_t(const xema_layernorm_args& a, hipStream_t s) {
  if (a.dim <= 2048) layernorm_nv<XT, RT, 1>(a, s);
  else layernorm_nv<XT, RT, LN_WAVES>(a, s);
}
template <typename XT>
void layernorm_x(const xema_layernorm_args& a, hipStream_t s) {
  if (!a.resid) return layernorm_t<XT, void>(a, s);
  switch (a.resid_dtype) {
    case XEMA_BF16: return layernorm_t<XT, bf16>(a, s);
    case XEMA_F16: return layernorm_t<XT, f16>(a, s);
    default: return layernorm_t<XT, float>(a, s);
  }
}

// Eight elements of a type known at run time (the same for a whole launch).
struct AnyRaw8 {
  u32x4 v[2];
  __device__ __forceinline__ void load(const void* p, int dtype, int64_t at) {
    if (dtype == XEMA_F32) {
      v[0] = reinterpret_cast<const u32x4*>((const float*)p + at)[0];
      v[1] = reinterpret_cast<const u32x4*>((const float*)p + at)[1];
    } else {
      v[0] = *reinterpret_cast<const u32x4*>((const uint16_t*)p + at);
    }
  }
  __device__ __forceinline__ void add_to(int dtype, float f[8]) const {
    float d[8];
    if (dtype == XEMA_F32) unpack8(Raw8<float>{{v[0], v[1]}}, d);
    else if (dtype == XEMA_BF16) unpack8(Raw8<bf16>{{v[0]}}, d);
    else unpack8(Raw8<f16>{{v[0]}}, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += d[e];
  }
};

// The gradient.  Workgroup b takes the rows b, b + grid, ... (WPR = 4) or the
// groups of four rows b, b + grid, ... (WPR = 1), holds its part of dgamma and
// dbeta in registers over them and writes it once.  A row's s, dy and dsum are
// loaded while the row before is computed.
template <typename XT, typename DT, int NV>
struct LnBwdRow {
  Raw8<XT> x[NV];
  Raw8<DT> d[NV];
  AnyRaw8 ds[NV];
  template <int STRIDE>
  __device__ __forceinline__ void load(const xema_layernorm_bwd_args& a, int64_t r, int in_row) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) {
        x[v] = load_raw8((const XT*)a.s + r * a.ld_s + c);
        d[v] = load_raw8((const DT*)a.dy + r * a.ld_dy + c);
        if (a.dsum) ds[v].load(a.dsum, a.dsum_dtype, r * a.ld_dsum + c);
      }
    }
  }
};

template <typename XT, typename DT, int NV, int WPR>
__global__ __launch_bounds__(LN_WAVES * 64) void k_layernorm_bwd(xema_layernorm_bwd_args a, float* __restrict__ partial) {
  constexpr int STRIDE = 512 * WPR;
  __shared__ float red[4][LN_WAVES];
  __shared__ float fold[WPR == 1 ? LN_WAVES : 1][WPR == 1 ? NV * 512 : 1];
  const int wave = threadIdx.x >> 6, in_row = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  const float n = (float)a.dim;
  float dg[NV][8], db[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[v][e] = db[v][e] = 0.f;
  const int64_t first = WPR == 1 ? (int64_t)blockIdx.x * LN_WAVES + wave : (int64_t)blockIdx.x;
  const int64_t step = (int64_t)gridDim.x * (WPR == 1 ? LN_WAVES : 1);
  LnBwdRow<XT, DT, NV> next;
  if (first < a.rows) next.template load<STRIDE>(a, first, in_row);
  for (int64_t r = first; r < a.rows; r += step) {
    const LnBwdRow<XT, DT, NV> row = next;
    if (r + step < a.rows) next.template load<STRIDE>(a, r + step, in_row);
    float total = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v * STRIDE + in_row * 8 < a.dim) {
        float x[8];
        unpack8(row.x[v], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) total += x[e];
      }
    }
    // (a row's second use of `red` is apart from its first, and the next row's
    // first comes after every wave has read this one's)
    const float mean = row_sum<WPR>(total, red[0], wave) / n;
    float ss = 0.f, sg = 0.f, sgx = 0.f;
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
          const float d = x[e] - mean, w = a.gamma ? g[e] * gam[e] : g[e];
          ss = fmaf(d, d, ss);
          sg += w;
          sgx = fmaf(w, d, sgx);
        }
      }
    }
    ss = wave_sum(ss);
    sg = wave_sum(sg);
    sgx = wave_sum(sgx);
    if constexpr (WPR > 1) {
      if ((threadIdx.x & 63) == 0) {
        red[1][wave] = ss;
        red[2][wave] = sg;
        red[3][wave] = sgx;
      }
      __syncthreads();
      ss = sg = sgx = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) {
        ss += red[1][w];
        sg += red[2][w];
        sgx += red[3][w];
      }
    }
    const float q = 1.0f / sqrtf(ss / n + a.eps);
    const float along = sgx * q / n, level = sg / n;      // mean(g n), mean(g)
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) {
        float x[8], g[8], gam[8], o[8];
        unpack8(row.x[v], x);
        unpack8(row.d[v], g);
        if (a.gamma) unpack8(load_raw8((const bf16*)a.gamma + c), gam);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float norm = (x[e] - mean) * q;
          dg[v][e] = fmaf(g[e], norm, dg[v][e]);
          db[v][e] += g[e];
          o[e] = q * ((a.gamma ? g[e] * gam[e] : g[e]) - level - norm * along);
        }
        if (a.dsum) row.ds[v].add_to(a.dsum_dtype, o);
        store8(a.dx, a.dx_dtype, r * a.ld_dx + c, o);
      }
    }
  }
  if (!partial) return;
  float* const out = partial + (int64_t)blockIdx.x * 2 * a.dim;
  if constexpr (WPR == 1) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h) __syncthreads();
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) fold[wave][v * 512 + in_row * 8 + e] = h ? db[v][e] : dg[v][e];
      __syncthreads();
      for (int c = threadIdx.x; c < a.dim; c += LN_WAVES * 64) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < LN_WAVES; ++w) s += fold[w][c];
        out[(int64_t)h * a.dim + c] = s;
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) {
        store8_as<float>(out, c, dg[v]);
        store8_as<float>(out, (int64_t)a.dim + c, db[v]);
      }
    }
  }
}

// dgamma and dbeta: the workgroups' parts, in order.  64 columns a workgroup, a
// part of the parts for each of its 16 waves, eight loads in flight.
__global__ __launch_bounds__(1024) void k_layernorm_sums(const float* __restrict__ partial, int parts, int dim, float* __restrict__ dgamma,
                                                         float* __restrict__ dbeta) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = (int)blockIdx.x * 64 + lane;
  const int p0 = parts * wave / 16, p1 = parts * (wave + 1) / 16;
  float s = 0.f;
  if (c < 2 * dim) {
#pragma unroll 8
    for (int i = p0; i < p1; ++i) s += partial[(int64_t)i * 2 * dim + c];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave || c >= 2 * dim) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += red[w][lane];
  float* const out = c < dim ? dgamma : dbeta;
  if (out) out[c < dim ? c : c - dim] = s;
}

template <typename XT, typename DT, int WPR>
void layernorm_bwd_nv(const xema_layernorm_bwd_args& a, float* partial, hipStream_t s) {
  const dim3 grid((unsigned)layernorm_bwd_partials(a.rows)), block(LN_WAVES * 64);
  const int nv = (a.dim + 512 * WPR - 1) / (512 * WPR);
  if (nv <= 1) hipLaunchKernelGGL((k_layernorm_bwd<XT, DT, 1, WPR>), grid, block, 0, s, a, partial);
  else if (nv <= 2) hipLaunchKernelGGL((k_layernorm_bwd<XT, DT, 2, WPR>), grid, block, 0, s, a, partial);
  else if (nv <= 4) hipLaunchKernelGGL((k_layernorm_bwd<XT, DT, 4, WPR>), grid, block, 0, s, a, partial);
  else if constexpr (WPR > 1) hipLaunchKernelGGL((k_layernorm_bwd<XT, DT, 8, WPR>), grid, block, 0, s, a, partial);
}
template <typename XT, typename DT>
void layernorm_bwd_t(const xema_layernorm_bwd_args& a, float* partial, hipStream_t s) {
  if (a.dim <= 2048) layernorm_bwd_nv<XT, DT, 1>(a, partial, s);
  else layernorm_bwd_nv<XT, DT, LN_WAVES>(a, partial, s);
}
template <typename XT>
void layernorm_bwd_x(const xema_layernorm_bwd_args& a, float* partial, hipStream_t s) {
  switch (a.dy_dtype) {
    case XEMA_BF16: return layernorm_bwd_t<XT, bf16>(a, partial, s);
    case XEMA_F16: return layernorm_bwd_t<XT, f16>(a, partial, s);
    default: return layernorm_bwd_t<XT, float>(a, partial, s);
  }
}

}  // namespace

hipError_t launch_layernorm(const xema_layernorm_args& a, hipStream_t s) {
  switch (a.x_dtype) {
    case XEMA_BF16: layernorm_x<bf16>(a, s); break;
    case XEMA_F16: layernorm_x<f16>(a, s); break;
    default: layernorm_x<float>(a, s); break;
  }
  return hipGetLastError();
}

int64_t layernorm_bwd_partials(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(1024, (rows + 3) / 4)); }

hipError_t launch_layernorm_bwd(const xema_layernorm_bwd_args& a, hipStream_t s) {
  const bool sums = a.dgamma || a.dbeta;
  float* partial = sums ? (float*)a.workspace : nullptr;
  int parts = 0;
  if (a.rows > 0) {
    parts = (int)layernorm_bwd_partials(a.rows);
    switch (a.s_dtype) {
      case XEMA_BF16: layernorm_bwd_x<bf16>(a, partial, s); break;
      case XEMA_F16: layernorm_bwd_x<f16>(a, partial, s); break;
      default: layernorm_bwd_x<float>(a, partial, s); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  hipLaunchKernelGGL(k_layernorm_sums, dim3((2 * a.dim + 63) / 64), dim3(1024), 0, s, partial, parts, a.dim, a.dgamma, a.dbeta);
  return hipGetLastError();
}

}  // namespace xema
