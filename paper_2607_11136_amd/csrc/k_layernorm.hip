// Layer norm with the residual's addition, and its gradient (xema_cross.h).
// Bound by HBM: a row is read once, held in registers as fp32 and written
// once; the variance is taken about the mean, from the registers.  A wave takes
// a row of up to 2048 elements (no barrier), a workgroup a wider one.  57224 x 4096,
// bf16 and an fp32 residual stream: 512 us, 5.5 TB/s (a copy of 1 GiB: 5.0); its
// gradient, 16384 x 4096 in bf16: 112 us, 4.8 TB/s, and 5 for the sums of dgamma's
// and dbeta's parts; 4 x 4096: 6.4 us, as long as any call.
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
  if constexpr (WPR == 1) {      // (rows of four waves have more than 2048 elements)
    if (nv <= 1) {
      hipLaunchKernelGGL((k_layernorm<XT, RT, 1, WPR>), grid, block, 0, s, a);
      return;
    }
  }
  if (nv <= 2) hipLaunchKernelGGL((k_layernorm<XT, RT, 2, WPR>), grid, block, 0, s, a);
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

// store8 with one branch, the 16-bit types by a choice of values.  With the three-way
// switch that store8 becomes, hipcc of ROCm 7.2 makes wrong code here: the IR joins the
// running sums from all three stores, the machine code enters the fp32 store from the
// tests of the other types with its copies of four of them undefined (16-bit s and dy,
// fp32 dx, narrow rows: dbeta wrong in up to half of the columns).
__device__ __forceinline__ void put8(void* p, int dtype, int64_t at, const float f[8]) {
  typedef bf16 b8 __attribute__((ext_vector_type(8)));
  if (dtype == XEMA_F32) {
    store8_as<float>(p, at, f);
  } else {
    b8 b;
    f16x8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      b[e] = (bf16)f[e];
      h[e] = (f16)f[e];
    }
    const u32x4 vb = __builtin_bit_cast(u32x4, b), vh = __builtin_bit_cast(u32x4, h);
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = dtype == XEMA_BF16 ? vb[e] : vh[e];
    *reinterpret_cast<u32x4*>((uint16_t*)p + at) = v;
  }
}

// Sum over each 16 lanes, by rotations, and over all 64 (the same in all, in a fixed order).
__device__ __forceinline__ float lane_sum16(float v) {
  auto turned = [](float x, auto ror) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x120 + decltype(ror)::value, 0xf, 0xf, false));
  };
  v += turned(v, std::integral_constant<int, 8>());
  v += turned(v, std::integral_constant<int, 4>());
  v += turned(v, std::integral_constant<int, 2>());
  return v + turned(v, std::integral_constant<int, 1>());
}
__device__ __forceinline__ float lane_sum(float v) {
  v = lane_sum16(v);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// The gradient.  A workgroup has G groups of WPR waves, a row each at a time;
// group i of them all takes the rows i, i + all groups, ..., holds its part of
// dgamma and dbeta in registers over them, and the groups' parts are added in the
// end and written once.  A row's s, dy and dsum are loaded while the row before is
// computed.  Each wave takes its sums about its own mean, so that one exchange
// joins them (16384 x 4096: 116 us; with an exchange for the mean, one for the
// variance and one for the rest, a row in flight and gamma read for each, 146): for
// a wave of n elements with mean m, the row's mean is the
// weighted mean M, its squares about M those about m and n (m - M)^2, and
// sum g (s - M) = sum g (s - m) + (m - M) sum g.  ST void: no dsum.
template <typename XT, typename DT, typename ST, int NV>
struct LnBwdRow {
  typedef std::conditional_t<std::is_void_v<ST>, bf16, ST> S;
  Raw8<XT> x[NV];
  Raw8<DT> d[NV];
  Raw8<S> ds[std::is_void_v<ST> ? 1 : NV];
  template <int STRIDE>
  __device__ __forceinline__ void load(const xema_layernorm_bwd_args& a, int64_t r, int in_row) {
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

template <typename XT, typename DT, typename ST, int NV, int WPR, int G>
__global__ __launch_bounds__(G * WPR * 64) void k_layernorm_bwd(xema_layernorm_bwd_args a, float* __restrict__ partial) {
  constexpr int STRIDE = 512 * WPR, WAVES = G * WPR;
  __shared__ __attribute__((aligned(16))) float red[2][WAVES][4];
  __shared__ float fold[G > 1 ? G : 1][G > 1 ? NV * STRIDE : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave / WPR, in_row = threadIdx.x - group * WPR * 64;
  const float n = (float)a.dim;
  float dg[NV][8], db[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[v][e] = db[v][e] = 0.f;
  // gamma in registers over all rows, as they allow
  constexpr bool KEEP = NV == 1;
  float kept[8];
  if constexpr (KEEP) {
#pragma unroll
    for (int e = 0; e < 8; ++e) kept[e] = 1.f;
    if (a.gamma && in_row * 8 < a.dim) unpack8(load_raw8((const bf16*)a.gamma + in_row * 8), kept);
  }
  // g = dy * gamma of a lane's vector at column c
  auto weigh = [&](int c, const float dy[8], float w[8]) {
    float gam[8];
    if (!KEEP && a.gamma) unpack8(load_raw8((const bf16*)a.gamma + c), gam);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = KEEP ? dy[e] * kept[e] : a.gamma ? dy[e] * gam[e] : dy[e];
  };
  // elements of a row that wave w of a group has
  auto share = [&](int w) {
    int k = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) k += max(0, min(512, a.dim - v * STRIDE - w * 512));
    return (float)k;
  };
  const float mine = WPR == 1 ? n : fmaxf(share(wave % WPR), 1.f), theirs = (int)(threadIdx.x & 15) < WPR ? share(threadIdx.x & 15) : 0.f;
  // (every wave meets every barrier: a group past the last row takes it again and keeps nothing)
  const int64_t step = (int64_t)gridDim.x * G, first = (int64_t)blockIdx.x * G + group, turns = (a.rows + step - 1) / step;
  // rows in flight, as the registers allow
  constexpr int AHEAD = NV == 1 && WAVES == 8 && sizeof(XT) + sizeof(DT) + sizeof(typename LnBwdRow<XT, DT, ST, NV>::S) <= 8 ? 2 : 1;
  LnBwdRow<XT, DT, ST, NV> next[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) next[i].template load<STRIDE>(a, first + i * step < a.rows ? first + i * step : a.rows - 1, in_row);
  auto take = [&](int64_t turn, auto slot) {
    LnBwdRow<XT, DT, ST, NV>& ahead = next[decltype(slot)::value];
    const int64_t r = first + turn * step;
    const LnBwdRow<XT, DT, ST, NV> row = ahead;
    if (r + AHEAD * step < a.rows) ahead.template load<STRIDE>(a, r + AHEAD * step, in_row);
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
    float mean = lane_sum(total) / mine, ss = 0.f, sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = v * STRIDE + in_row * 8;
      if (c < a.dim) {
        float x[8], g[8], w[8];
        unpack8(row.x[v], x);
        unpack8(row.d[v], g);
        weigh(c, g, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = x[e] - mean;
          ss = fmaf(d, d, ss);
          sg += w[e];
          sgx = fmaf(w[e], d, sgx);
        }
      }
    }
    ss = lane_sum(ss);
    sg = lane_sum(sg);
    sgx = lane_sum(sgx);
    if constexpr (WPR > 1) {
      float(*const at)[4] = red[turn & 1];
      if ((threadIdx.x & 63) == 0) *reinterpret_cast<f32x4*>(at[wave]) = f32x4{mean, ss, sg, sgx};
      __syncthreads();   // (the next row writes the other half)
      // (lane i of each 16 joins wave i's; one of no elements left zeros)
      const int i = threadIdx.x & 15;
      const f32x4 w = i < WPR ? *reinterpret_cast<const f32x4*>(at[group * WPR + i]) : f32x4{0.f, 0.f, 0.f, 0.f};
      mean = lane_sum16(w[0] * theirs) / n;
      const float off = theirs > 0.f ? w[0] - mean : 0.f;
      ss = lane_sum16(fmaf(theirs * off, off, w[1]));
      sg = lane_sum16(w[2]);
      sgx = lane_sum16(fmaf(w[2], off, w[3]));
    }
    const float q = 1.0f / sqrtf(ss / n + a.eps);
    const float along = sgx * q / n, level = sg / n;      // mean(g n), mean(g)
    if (r < a.rows) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = v * STRIDE + in_row * 8;
        if (c < a.dim) {
          float x[8], g[8], o[8], ds[8];
          unpack8(row.x[v], x);
          unpack8(row.d[v], g);
          weigh(c, g, o);
          if constexpr (!std::is_void_v<ST>) unpack8(row.ds[v], ds);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float norm = (x[e] - mean) * q;
            dg[v][e] = fmaf(g[e], norm, dg[v][e]);
            db[v][e] += g[e];
            const float t = fmaf(-along, norm, o[e] - level);
            o[e] = std::is_void_v<ST> ? q * t : fmaf(q, t, ds[e]);
          }
          put8(a.dx, a.dx_dtype, r * a.ld_dx + c, o);
        }
      }
    }
  };
  for (int64_t turn = 0; turn < turns; turn += AHEAD) {
    take(turn, std::integral_constant<int, 0>());
    if constexpr (AHEAD > 1) {
      if (turn + 1 < turns) take(turn + 1, std::integral_constant<int, 1>());
    }
  }
  if (!partial) return;
  float* const out = partial + (int64_t)blockIdx.x * 2 * a.dim;
  if constexpr (G > 1) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h) __syncthreads();
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) fold[group][v * STRIDE + in_row * 8 + e] = h ? db[v][e] : dg[v][e];
      __syncthreads();
      for (int c = threadIdx.x; c < a.dim; c += WAVES * 64) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < G; ++w) s += fold[w][c];
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

// Eight elements a lane, a row to as many waves as it needs, eight waves a
// workgroup to rows of 4096 elements and sixteen past that; at most two workgroups
// a CU, so that the parts of dgamma and dbeta are few.  Returns those parts.
template <typename XT, typename DT, typename ST, int NV, int WPR, int G>
int layernorm_bwd_run(const xema_layernorm_bwd_args& a, float* partial, hipStream_t s) {
  const int parts = (int)std::min<int64_t>(layernorm_bwd_partials(a.rows), (a.rows + G - 1) / G);
  hipLaunchKernelGGL((k_layernorm_bwd<XT, DT, ST, NV, WPR, G>), dim3(parts), dim3(G * WPR * 64), 0, s, a, partial);
  return parts;
}
template <typename XT, typename DT, typename ST>
int layernorm_bwd_t(const xema_layernorm_bwd_args& a, float* partial, hipStream_t s) {
  if (a.dim <= 512) return layernorm_bwd_run<XT, DT, ST, 1, 1, 8>(a, partial, s);
  if (a.dim <= 1024) return layernorm_bwd_run<XT, DT, ST, 1, 2, 4>(a, partial, s);
  if (a.dim <= 2048) return layernorm_bwd_run<XT, DT, ST, 1, 4, 2>(a, partial, s);
  if (a.dim <= 4096) return layernorm_bwd_run<XT, DT, ST, 1, 8, 1>(a, partial, s);
  if (a.dim <= 8192) return layernorm_bwd_run<XT, DT, ST, 1, 16, 1>(a, partial, s);
  // (more a lane, in eight waves: sixteen have too few registers)
  return layernorm_bwd_run<XT, DT, ST, 4, 8, 1>(a, partial, s);
}
template <typename XT, typename DT>
int layernorm_bwd_d(const xema_layernorm_bwd_args& a, float* partial, hipStream_t s) {
  if (!a.dsum) return layernorm_bwd_t<XT, DT, void>(a, partial, s);
  switch (a.dsum_dtype) {
    case XEMA_BF16: return layernorm_bwd_t<XT, DT, bf16>(a, partial, s);
    case XEMA_F16: return layernorm_bwd_t<XT, DT, f16>(a, partial, s);
    default: return layernorm_bwd_t<XT, DT, float>(a, partial, s);
  }
}
// Returns the parts of dgamma and dbeta that it leaves.
template <typename XT>
int layernorm_bwd_x(const xema_layernorm_bwd_args& a, float* partial, hipStream_t s) {
  switch (a.dy_dtype) {
    case XEMA_BF16: return layernorm_bwd_d<XT, bf16>(a, partial, s);
    case XEMA_F16: return layernorm_bwd_d<XT, f16>(a, partial, s);
    default: return layernorm_bwd_d<XT, float>(a, partial, s);
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

int64_t layernorm_bwd_partials(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(512, rows)); }

hipError_t launch_layernorm_bwd(const xema_layernorm_bwd_args& a, hipStream_t s) {
  const bool sums = a.dgamma || a.dbeta;
  float* partial = sums ? (float*)a.workspace : nullptr;
  int parts = 0;
  if (a.rows > 0) {
    switch (a.s_dtype) {
      case XEMA_BF16: parts = layernorm_bwd_x<bf16>(a, partial, s); break;
      case XEMA_F16: parts = layernorm_bwd_x<f16>(a, partial, s); break;
      default: parts = layernorm_bwd_x<float>(a, partial, s); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  hipLaunchKernelGGL(k_layernorm_sums, dim3((2 * a.dim + 63) / 64), dim3(1024), 0, s, partial, parts, a.dim, a.dgamma, a.dbeta);
  return hipGetLastError();
}

}  // namespace xema
