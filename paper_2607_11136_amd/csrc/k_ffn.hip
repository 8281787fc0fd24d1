// Gated feed-forward on gfx950 MFMA, forward and gradient (xema_ffn.h).
//
// Forward: one kernel, bound by its MFMAs (8192 x 4096 x 2 11008 in bf16 1.16 ms, 1270
// TFLOP/s with g and u kept, 720 MB of stores; 17776 x 4096 x 2 16384 in e4m3 1.73
// ms, 2750 TFLOP/s), or for few rows by reading the weights (one row of 4096 x 2
// 16384: 46 us, 5.8 TB/s; in e4m3 30 us, 4.4 TB/s).
// Gradient: dg and du first, bound by HBM (1.08 GB in 222 us), as both products
// need them in either order; then dx, the weights' and the biases' gradients in
// one launch (8192 x 4096 x 11008: 2.2 ms, 1340 TFLOP/s) where they take the same
// tile, and the sums of the parts where a product splits its k; the weights and x read
// in place through transposing LDS reads: copies in the other order would cost
// 0.9 GB of traffic a step.
#include <algorithm>

#include "device_common.h"
#include "few_rows.h"
#include "ffn.h"
#include "mma_tile.h"

namespace xema {

namespace {

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

// The stored g and u: the upper 24 bits of fp32, rounded to nearest even
// (infinities and NaN keep their upper bits, and a NaN stays one).  Four units
// take 24 bytes: upper halves of g, of u, third bytes of g, of u.
constexpr int PRE_GROUP = 24;
__device__ __forceinline__ uint32_t round24(float v) {
  const uint32_t b = __float_as_uint(v);
  if ((b & 0x7f800000u) == 0x7f800000u) return b | (b & 0x7fffffu ? 0x400000u : 0u);
  return b + 0x7fu + (b >> 8 & 1u);
}
__device__ __forceinline__ void store_pre(uint8_t* at, const float g[4], const float u[4]) {
  uint32_t r[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    r[e] = round24(g[e]);
    r[4 + e] = round24(u[e]);
  }
  u32x2 w[3];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 2; ++e) w[h][e] = __builtin_amdgcn_perm(r[4 * h + 2 * e + 1], r[4 * h + 2 * e], 0x07060302u);
    uint32_t low = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) low |= (r[4 * h + e] >> 8 & 0xffu) << (8 * e);
    w[2][h] = low;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) reinterpret_cast<u32x2*>(at)[i] = w[i];
}
// Element e of one of the two, from its upper halves and third bytes.
__device__ __forceinline__ float load24(const uint32_t* upper, uint32_t low, int e) {
  const uint32_t hi = e & 1 ? upper[e >> 1] & 0xffff0000u : upper[e >> 1] << 16;
  return __uint_as_float(hi | (low >> (8 * e) & 0xffu) << 8);
}

// Four floats from a 4-byte aligned address.
__device__ __forceinline__ void load4_at4(const float* p, float v[4]) {
  typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
  const f4 u = *reinterpret_cast<const f4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = u[e];
}

struct GatedParams {
  const void* x; const float* x_scale;
  const void *gate_w, *up_w; const float *gate_scale, *up_scale;
  const uint16_t *gate_b, *up_b;
  void* y; void* pre;
  int64_t rows, ldx, ldy;
  int dim, hidden, act;
};

// y = act(x Wg^T + bg) * (x Wu^T + bu).  A tile's columns are gate and up rows
// of the same hidden units, half and half within each wave, so that a lane
// holds both factors of its outputs and the product needs no exchange.
template <typename T, typename YT, typename S>
__global__ __launch_bounds__(S::NW * 64, 1) void k_gated(GatedParams p) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[S::LDS];
  constexpr int HN = S::BN / 2, NB = S::NJ / 2;      // hidden units per tile, blocks per wave
  const int tiles_n = (p.hidden + HN - 1) / HN, tiles_m = (int)((p.rows + S::BM - 1) / S::BM);
  int tm, tn;
  tile_of((int)blockIdx.x, tiles_m, tiles_n, 1024 / S::BM, &tm, &tn);
  const int64_t m0 = (int64_t)tm * S::BM;
  const int n0 = tn * HN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kbytes = p.dim * (int)sizeof(T);

  RowOperand<S::BM, S::NW> a;
  PairOperand<S::BN, S::NW, S::WC> b;
  a.init((const T*)p.x + m0 * p.ldx, nullptr, p.rows - m0, p.ldx * sizeof(T), kbytes, 0x7fffffff, wave, lane);
  b.init((const T*)p.gate_w + (int64_t)n0 * p.dim, (const T*)p.up_w + (int64_t)n0 * p.dim, p.hidden - n0, kbytes, kbytes, wave, lane);
  f32x4 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  tile_products<S, T, ROWS, ROWS>(a, b, (kbytes + KB - 1) / KB, smem, wave, lane, acc);

  const int l16 = lane & 15, l4 = lane >> 4;
  const int col0 = n0 + wave % S::WNW * (S::WC / 2);
  float sg[NB][4], su[NB][4], bg[NB][4] = {}, bu[NB][4] = {};
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int col = min(col0 + 16 * j + 4 * l4, p.hidden - 4);      // (units past the last are not stored)
    if (sizeof(T) == 1) {
      load4_at4(p.gate_scale + col, sg[j]);
      load4_at4(p.up_scale + col, su[j]);
    }
    if (p.gate_b) load4f<uint16_t>(p.gate_b + col, bg[j]);
    if (p.up_b) load4f<uint16_t>(p.up_b + col, bu[j]);
  }
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const int64_t m = m0 + wave / S::WNW * S::WR + 16 * i + l16;
    const bool valid = m < p.rows;
    const int64_t mv = valid ? m : p.rows - 1;
    const float sx = sizeof(T) == 1 ? p.x_scale[mv] : 1.f;
    float g[NB][4], u[NB][4], y[NB][4];
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[j][e] = acc[i][j][e];
        u[j][e] = acc[i][NB + j][e];
        if (sizeof(T) == 1) {
          g[j][e] *= sx * sg[j][e];
          u[j][e] *= sx * su[j][e];
        }
        g[j][e] += bg[j][e];
        u[j][e] += bu[j][e];
        y[j][e] = activate<false>(g[j][e], p.act, nullptr) * u[j][e];
      }
    store_row<YT, NB>((YT*)p.y + mv * p.ldy, col0, p.hidden, y, l4, valid);
    if (sizeof(T) == 2 && p.pre) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int unit = col0 + 16 * j + 4 * l4;
        if (valid && unit < p.hidden) store_pre((uint8_t*)p.pre + (m * p.hidden + unit) / 4 * PRE_GROUP, g[j], u[j]);
      }
    }
  }
}

// The same for few rows: 16 hidden units a workgroup, gate rows as block 0 and
// up rows as block 1.
constexpr int FEW_WAVES = 8;
template <typename T, typename YT, int MT, int UNROLL>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_gated_few(GatedParams p) {
  typedef FewRows<MT, 2, FEW_WAVES> S;
  __shared__ __attribute__((aligned(16))) float red[S::FLOATS];
  const int n0 = (int)blockIdx.x * 16, l16 = threadIdx.x & 15;
  const int64_t kb = (int64_t)p.dim * sizeof(T);
  const int64_t unit = min(n0 + l16, p.hidden - 1);
  const uint8_t* x[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = 16 * i + l16;
    x[i] = (const uint8_t*)p.x + (m < p.rows ? m : p.rows - 1) * p.ldx * sizeof(T);
  }
  const uint8_t* const w[2] = {(const uint8_t*)p.gate_w + unit * kb, (const uint8_t*)p.up_w + unit * kb};
  few_rows_products<T, MT, 2, FEW_WAVES, UNROLL>(x, w, (int)kb, red);
  // four units of one row per thread
  const int t = (int)threadIdx.x, m = t / 4, c = t % 4 * 4, col = n0 + c;
  if (m >= 16 * MT || m >= p.rows || col >= p.hidden) return;
  const f32x4 rg = few_rows_sum4<S>(red, m, c), ru = few_rows_sum4<S>(red, m, 16 + c);
  float g[4], u[4];
  typedef YT y4 __attribute__((ext_vector_type(4)));
  y4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    g[e] = rg[e];
    u[e] = ru[e];
    if (sizeof(T) == 1) {
      g[e] *= p.x_scale[m] * p.gate_scale[col + e];
      u[e] *= p.x_scale[m] * p.up_scale[col + e];
    }
    g[e] += p.gate_b ? bf16_bits_to_f32(p.gate_b[col + e]) : 0.f;
    u[e] += p.up_b ? bf16_bits_to_f32(p.up_b[col + e]) : 0.f;
    y[e] = (YT)(activate<false>(g[e], p.act, nullptr) * u[e]);
  }
  *reinterpret_cast<y4*>((YT*)p.y + m * p.ldy + col) = y;
  if (sizeof(T) == 2 && p.pre) store_pre((uint8_t*)p.pre + ((int64_t)m * p.hidden + col) / 4 * PRE_GROUP, g, u);
}

template <typename T, typename YT, int MT, int UNROLL>
hipError_t run_gated_few(const GatedParams& p, hipStream_t s) {
  hipLaunchKernelGGL((k_gated_few<T, YT, MT, UNROLL>), dim3((p.hidden + 15) / 16), dim3(FEW_WAVES * 64), 0, s, p);
  return hipGetLastError();
}

template <typename T, typename YT, typename S>
hipError_t run_gated(const GatedParams& p, hipStream_t s) {
  const int64_t tiles = (p.rows + S::BM - 1) / S::BM * ((p.hidden + S::BN / 2 - 1) / (S::BN / 2));
  hipLaunchKernelGGL((k_gated<T, YT, S>), dim3((unsigned)tiles), dim3(S::NW * 64), 0, s, p);
  return hipGetLastError();
}

template <typename T, typename YT>
hipError_t gated_t(const GatedParams& p, hipStream_t s) {
  const FewPick few = pick_gated_few(p.rows, p.hidden);
  if (few.rows16 == 1) return run_gated_few<T, YT, 1, 4>(p, s);
  if (few.rows16 == 2) return run_gated_few<T, YT, 2, 2>(p, s);
  return with_tile(pick_tile(p.rows, 2 * (int64_t)p.hidden, ((int64_t)p.dim * sizeof(T) + KB - 1) / KB),
                   [&](auto shape) { return run_gated<T, YT, decltype(shape)>(p, s); });
}

// dg = dy u act'(g), du = dy act(g), rounded to T, and the column sums of the
// rounded-free values over each chunk of rows.  A workgroup takes 256 columns,
// 8 a thread, of `chunk` rows, 8 rows at a time.
template <typename T>
__global__ __launch_bounds__(256) void k_gated_grad(const uint8_t* __restrict__ pre, const T* __restrict__ dy, int64_t ld_dy, int64_t rows,
                                                    int hidden, int act, int chunk, T* __restrict__ dg, T* __restrict__ du,
                                                    float* __restrict__ partial) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  __shared__ float red[8][2][256 + 8];
  const int c8 = threadIdx.x & 31, r8 = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 256 + c8 * 8;
  const bool in = col < hidden;
  const int64_t r0 = (int64_t)blockIdx.y * chunk, r1 = r0 + chunk < rows ? r0 + chunk : rows;
  float sg[8], su[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sg[e] = su[e] = 0.f;
  if (in)
    for (int64_t r = r0 + r8; r < r1; r += 8) {
      uint32_t w[12];
      const u32x4* at = reinterpret_cast<const u32x4*>(pre + (r * hidden + col) / 4 * PRE_GROUP);
#pragma unroll
      for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * i + e] = at[i][e];
      const t8 d = *reinterpret_cast<const t8*>(dy + r * ld_dy + col);
      t8 og, ou;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float slope;
        const uint32_t* four = w + e / 4 * 6;
        const float g = load24(four, four[4], e % 4), u = load24(four + 2, four[5], e % 4);
        const float a = activate<true>(g, act, &slope), df = (float)d[e];
        const float vg = df * u * slope, vu = df * a;
        sg[e] += vg;
        su[e] += vu;
        og[e] = (T)vg;
        ou[e] = (T)vu;
      }
      *reinterpret_cast<t8*>(dg + r * hidden + col) = og;
      *reinterpret_cast<t8*>(du + r * hidden + col) = ou;
    }
  if (!partial) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    red[r8][0][c8 * 8 + e] = sg[e];
    red[r8][1][c8 * 8 + e] = su[e];
  }
  __syncthreads();
  const int c = (int)blockIdx.x * 256 + threadIdx.x;
  if (c < hidden) {
    float a = 0.f, b = 0.f;
    for (int r = 0; r < 8; ++r) {
      a += red[r][0][threadIdx.x];
      b += red[r][1][threadIdx.x];
    }
    partial[(int64_t)blockIdx.y * 2 * hidden + c] = a;
    partial[(int64_t)blockIdx.y * 2 * hidden + hidden + c] = b;
  }
}

struct BwdParams {
  const void *dg, *du;          // [rows, hidden]
  const void *gate_w, *up_w;    // [hidden, dim]
  const void* x;
  void *dx, *dgate_w, *dup_w;
  float* dx_parts;              // [parts][rows][dim] where dx's k is split
  float* dw_parts;              // [w_parts][2][hidden][dim] where the weights' gradients' k (rows) is split
  const float* partial;         // [chunks][2 hidden]
  uint16_t *dgate_b, *dup_b;
  int64_t rows, ldx, ld_dx;
  int dim, hidden, chunks, parts, w_parts;
};

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

// dx = dg Wg + du Wu: the weights are read k by k (a row of W is one k).  With
// parts, workgroup wg has part wg / tiles of the steps, its sums kept in fp32.
template <typename T, typename S>
__device__ __forceinline__ TileOut<T> dx_tile(const BwdParams& p, int wg, uint8_t* smem, int wave, int lane, f32x4 (&acc)[S::MI][S::NJ]) {
  const int tiles = tiles_of<S>(p.rows, p.dim), part = __builtin_amdgcn_readfirstlane(wg / tiles);
  int tm, tn;
  tile_of(wg - part * tiles, (int)((p.rows + S::BM - 1) / S::BM), (p.dim + S::BN - 1) / S::BN, 1024 / S::BM, &tm, &tn);
  const int64_t m0 = (int64_t)tm * S::BM;
  const int n0 = tn * S::BN, steps = (p.hidden + 63) / 64, each = (2 * steps + p.parts - 1) / p.parts, first = part * each;
  RowOperand<S::BM, S::NW> a;
  ColumnOperand<S::BN, S::NW> b;
  a.init((const T*)p.dg + m0 * p.hidden, (const T*)p.du + m0 * p.hidden, p.rows - m0, (int64_t)p.hidden * 2, p.hidden * 2, steps, wave, lane, first);
  b.init((const T*)p.gate_w + n0, (const T*)p.up_w + n0, p.dim - n0, (int64_t)p.dim * 2, p.hidden, steps, wave, lane, first);
  tile_products<S, T, ROWS, COLUMNS>(a, b, min(each, 2 * steps - first), smem, wave, lane, acc);
  return {(T*)p.dx, p.parts > 1 ? p.dx_parts + part * p.rows * p.dim : nullptr, p.parts > 1 ? p.dim : p.ld_dx,
          m0 + wave / S::WNW * S::WR, p.rows, n0 + wave % S::WNW * S::WC, p.dim};
}

// dWg = dg^T x and dWu = du^T x: both operands are read k (row) by k.  With
// w_parts, workgroup wg has part wg / tiles of the rows, its sums kept in fp32.
template <typename T, typename S>
__device__ __forceinline__ TileOut<T> dw_tile(const BwdParams& p, int wg, uint8_t* smem, int wave, int lane, f32x4 (&acc)[S::MI][S::NJ]) {
  const int tiles_h = (p.hidden + S::BM - 1) / S::BM, tiles = 2 * tiles_of<S>(p.hidden, p.dim);
  const int steps = (int)((p.rows + 63) / 64);
  int part = 0, first = 0, count = steps;
  if (p.w_parts > 1) {
    const int each = (steps + p.w_parts - 1) / p.w_parts;
    part = __builtin_amdgcn_readfirstlane(wg / tiles);
    first = part * each;
    count = min(each, steps - first);
  }
  int tm, tn;
  tile_of(wg - part * tiles, 2 * tiles_h, (p.dim + S::BN - 1) / S::BN, 1024 / S::BM, &tm, &tn);
  const bool up = tm >= tiles_h;
  const int64_t r0 = (int64_t)first * 64;
  const int m0 = (up ? tm - tiles_h : tm) * S::BM, n0 = tn * S::BN;
  ColumnOperand<S::BM, S::NW> a;
  ColumnOperand<S::BN, S::NW> b;
  a.init((const T*)(up ? p.du : p.dg) + r0 * p.hidden + m0, nullptr, p.hidden - m0, (int64_t)p.hidden * 2, p.rows - r0, 0x7fffffff, wave, lane);
  b.init((const T*)p.x + r0 * p.ldx + n0, nullptr, p.dim - n0, p.ldx * 2, p.rows - r0, 0x7fffffff, wave, lane);
  tile_products<S, T, COLUMNS, COLUMNS>(a, b, count, smem, wave, lane, acc);
  return {(T*)(up ? p.dup_w : p.dgate_w), p.w_parts > 1 ? p.dw_parts + ((int64_t)part * 2 + up) * p.hidden * p.dim : nullptr, p.dim,
          m0 + wave / S::WNW * S::WR, p.hidden, n0 + wave % S::WNW * S::WC, p.dim};
}

// The products of the gradient in one launch: first dx's tiles, whose k is the
// longer where rows are few, then those of the weights' gradients, then the
// biases' (the chunks' column sums, in order), so that what each leaves idle
// the next one takes.
template <typename T, typename S>
__global__ __launch_bounds__(S::NW * 64, 1) void k_gated_products(BwdParams p, int dx_tiles, int dw_tiles) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[S::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wg = (int)blockIdx.x;
  if (wg >= dx_tiles + dw_tiles) {
    const int c = (wg - dx_tiles - dw_tiles) * S::NW * 64 + (int)threadIdx.x;
    if (c >= 2 * p.hidden) return;
    float v = 0.f;
#pragma unroll 8
    for (int i = 0; i < p.chunks; ++i) v += p.partial[(int64_t)i * 2 * p.hidden + c];
    (c < p.hidden ? p.dgate_b + c : p.dup_b + (c - p.hidden))[0] = __builtin_bit_cast(uint16_t, (bf16)v);
    return;
  }
  f32x4 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const TileOut<T> o = wg < dx_tiles ? dx_tile<T, S>(p, wg, smem, wave, lane, acc) : dw_tile<T, S>(p, wg - dx_tiles, smem, wave, lane, acc);
  if (o.sums) store_sums<S>(acc, o.sums, o.ld, o.row0, o.rows, o.col0, o.cols, lane);
  else store_tile<T, S>(acc, o.out, o.ld, o.row0, o.rows, o.col0, o.cols, lane);
}

template <typename T, typename S>
hipError_t run_products(const BwdParams& p, bool dx, bool dw, bool db, hipStream_t s) {
  const int dx_tiles = dx ? tiles_of<S>(p.rows, p.dim) * p.parts : 0, dw_tiles = dw ? 2 * tiles_of<S>(p.hidden, p.dim) * p.w_parts : 0;
  const int db_wgs = db ? (2 * p.hidden + S::NW * 64 - 1) / (S::NW * 64) : 0;
  if (!(dx_tiles + dw_tiles + db_wgs)) return hipSuccess;
  hipLaunchKernelGGL((k_gated_products<T, S>), dim3((unsigned)(dx_tiles + dw_tiles + db_wgs)), dim3(S::NW * 64), 0, s, p, dx_tiles, dw_tiles);
  return hipGetLastError();
}

template <typename T>
hipError_t bwd_t(const xema_gated_ffn_bwd_args& a, hipStream_t s) {
  const int64_t part = (a.rows * a.hidden * 2 + 255) / 256 * 256;
  uint8_t* ws = (uint8_t*)a.workspace;
  T *dg = (T*)ws, *du = (T*)(ws + part);
  float* partial = a.dgate_b ? (float*)(ws + 2 * part) : nullptr;
  const int chunks = (int)gated_bwd_row_chunks(a.rows);
  hipError_t e = hipSuccess;
  if (a.rows > 0) {
    const int chunk = (int)((a.rows + chunks - 1) / chunks);
    hipLaunchKernelGGL((k_gated_grad<T>), dim3((a.hidden + 255) / 256, chunks), dim3(256), 0, s, (const uint8_t*)a.pre, (const T*)a.dy, a.ld_dy,
                       a.rows, a.hidden, a.act, chunk, dg, du, partial);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const bool dx = a.dx && a.rows > 0, dw = a.dgate_w, db = a.dgate_b;
  const FfnSplit sx = pick_split(a.rows, a.dim, 2 * ((a.hidden + 63) / 64));
  const FfnSplit sw = pick_split(2 * (int64_t)a.hidden, a.dim, (a.rows + 63) / 64);
  float* dx_parts = (float*)(ws + 2 * part + gated_bwd_row_chunks(a.rows) * 2 * a.hidden * 4);
  float* dw_parts = dx_parts + gated_bwd_dx_parts(a.rows, a.dim, a.hidden);
  const BwdParams p{dg, du, a.gate_w, a.up_w, a.x, a.dx, a.dgate_w, a.dup_w, dx_parts, dw_parts, partial, (uint16_t*)a.dgate_b, (uint16_t*)a.dup_b,
                    a.rows, a.ldx, a.ld_dx, a.dim, a.hidden, a.rows > 0 ? chunks : 0, sx.parts, sw.parts};
  // one launch where both products take the same tile
  if (dx && dw && sx.tile != sw.tile) {
    e = with_tile(sx.tile, [&](auto shape) { return run_products<T, decltype(shape)>(p, true, false, false, s); });
    if (e == hipSuccess) e = with_tile(sw.tile, [&](auto shape) { return run_products<T, decltype(shape)>(p, false, true, db, s); });
  } else {
    e = with_tile(dx ? sx.tile : sw.tile, [&](auto shape) { return run_products<T, decltype(shape)>(p, dx, dw, db, s); });
  }
  if (e == hipSuccess && dx && sx.parts > 1)
    e = run_sum<T>(dx_parts, sx.parts, a.rows * a.dim, a.dim, (T*)a.dx, (T*)a.dx, a.rows * a.dim, a.ld_dx, s);
  if (e == hipSuccess && dw && sw.parts > 1) {
    const int64_t one = (int64_t)a.hidden * a.dim;
    e = run_sum<T>(dw_parts, sw.parts, 2 * one, a.dim, (T*)a.dgate_w, (T*)a.dup_w, one, a.dim, s);
  }
  return e;
}

}  // namespace

hipError_t launch_gated_ffn(const xema_gated_ffn_args& a, hipStream_t s) {
  const GatedParams p{a.x, a.x_scale, a.gate_w, a.up_w, a.gate_scale, a.up_scale, (const uint16_t*)a.gate_b, (const uint16_t*)a.up_b,
                      a.y, a.pre, a.rows, a.ldx, a.ldy, a.dim, a.hidden, a.act};
  if (a.dtype == XEMA_E4M3) return a.y_dtype == XEMA_BF16 ? gated_t<e4m3, bf16>(p, s) : gated_t<e4m3, f16>(p, s);
  return a.dtype == XEMA_BF16 ? gated_t<bf16, bf16>(p, s) : gated_t<f16, f16>(p, s);
}

int64_t gated_bwd_row_chunks(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(64, (rows + 7) / 8)); }

int64_t gated_bwd_dx_parts(int64_t rows, int dim, int hidden) {
  const int parts = rows > 0 ? pick_split(rows, dim, 2 * ((hidden + 63) / 64)).parts : 1;
  return parts > 1 ? parts * rows * dim : 0;
}

int64_t gated_bwd_dw_parts(int64_t rows, int dim, int hidden) {
  const int parts = pick_split(2 * (int64_t)hidden, dim, (rows + 63) / 64).parts;
  return parts > 1 ? (int64_t)parts * 2 * hidden * dim : 0;
}

hipError_t launch_gated_ffn_bwd(const xema_gated_ffn_bwd_args& a, hipStream_t s) {
  return a.dtype == XEMA_BF16 ? bwd_t<bf16>(a, s) : bwd_t<f16>(a, s);
}

}  // namespace xema
