// Linear layer with bias, activation and residual in its epilogue, and its
// gradient (xema_cross.h), on the tiles of mma_tile.h.
//
// Forward: one kernel, bound by its MFMAs, or for few rows by reading the weights;
// the last rows take a launch of their own where the rule's model has that faster
// (4608 x 4096 x 4096 with an fp32 residual 145 us, in one launch 163).  9216 x
// 4096 x 4096: in bf16 245 us, 1260 TFLOP/s; with the fp32 residual 306, as its
// 302 MB come and go while no tile multiplies (loads ahead of the epilogue gained
// nothing; the rest's tiles ahead of the others in one launch, so that half of the
// CUs end at unlike times, 5% here and nothing at other sizes). 24 x 4096 x 4096:
// 12 us, 2.8 TB/s.
//
// Gradient: dz first where there is an activation, dy in fp32 or a bias (bound by
// HBM: both products need it in either order; 8192 x 11008, gelu, 143 us, 4.4
// TB/s); then dx, dw and the bias's gradient in one launch where they take the
// same tile, w and x read in place through transposing LDS reads (8192 x 4096 x
// 11008 1100 us, 1340 TFLOP/s); and the sums of the parts where a product splits
// its k.
#include <algorithm>

#include "cross.h"
#include "device_common.h"
#include "few_rows.h"
#include "mma_tile.h"
#include "product_out.h"
#include "row_io.h"

namespace xema {

namespace {

// z, the upper 24 bits of fp32: four columns take 12 bytes, upper halves, then
// third bytes.
constexpr int Z_GROUP = 12;
typedef uint32_t u32x3_4 __attribute__((ext_vector_type(3), aligned(4)));
__device__ __forceinline__ void store_z(uint8_t* at, const float z[4]) {
  uint32_t r[4], low = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    r[e] = round24(z[e]);
    low |= (r[e] >> 8 & 0xffu) << (8 * e);
  }
  *reinterpret_cast<u32x3_4*>(at) = u32x3_4{__builtin_amdgcn_perm(r[1], r[0], 0x07060302u), __builtin_amdgcn_perm(r[3], r[2], 0x07060302u), low};
}

struct LinearParams {
  const void *x, *w;
  const uint16_t* bias;
  const void* resid;
  void *y, *pre;
  int64_t rows, ldx, ld_resid, ldy;
  int dim, out_dim, act, resid_dtype;
};

__device__ __forceinline__ void add4(const void* p, int dtype, int64_t at, float v[4]) {
  float r[4];
  if (dtype == XEMA_F32) {
    load4f<float>((const float*)p + at, r);
  } else if (dtype == XEMA_BF16) {
    load4f<uint16_t>((const uint16_t*)p + at, r);
  } else {
    const f16x4 h = *reinterpret_cast<const f16x4*>((const f16*)p + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (float)h[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] += r[e];
}

template <typename T, typename YT, typename S>
__global__ __launch_bounds__(S::NW * 64, 1) void k_linear(LinearParams p) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[S::LDS];
  const int tiles_n = (p.out_dim + S::BN - 1) / S::BN, tiles_m = (int)((p.rows + S::BM - 1) / S::BM);
  int tm, tn;
  tile_of((int)blockIdx.x, tiles_m, tiles_n, 1024 / S::BM, &tm, &tn);
  const int64_t m0 = (int64_t)tm * S::BM;
  const int n0 = tn * S::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, l4 = lane >> 4;
  const int64_t mw = m0 + wave / S::WNW * S::WR;
  const int nw = n0 + wave % S::WNW * S::WC;
  const int kbytes = p.dim * 2;

  RowOperand<S::BM, S::NW> a;
  RowOperand<S::BN, S::NW> b;
  a.init((const T*)p.x + m0 * p.ldx, nullptr, p.rows - m0, p.ldx * 2, kbytes, 0x7fffffff, wave, lane);
  b.init((const T*)p.w + (int64_t)n0 * p.dim, nullptr, p.out_dim - n0, kbytes, kbytes, 0x7fffffff, wave, lane);
  f32x4 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  tile_products<S, T, ROWS, ROWS>(a, b, (kbytes + KB - 1) / KB, smem, wave, lane, acc);

  float bv[S::NJ][4] = {};
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) load4f<uint16_t>(p.bias + min(nw + 16 * j + 4 * l4, p.out_dim - 4), bv[j]);
  }
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const int64_t m = mw + 16 * i + l16;
    const bool valid = m < p.rows;
    float v[S::NJ][4];
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int col = nw + 16 * j + 4 * l4;
      const bool in = valid && col < p.out_dim;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j][e] = acc[i][j][e] + bv[j][e];
      if (p.pre && in) store_z((uint8_t*)p.pre + (m * p.out_dim + col) / 4 * Z_GROUP, v[j]);
      if (p.act != XEMA_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[j][e] = activate<false>(v[j][e], p.act, nullptr);
      }
      if (p.resid && in) add4(p.resid, p.resid_dtype, m * p.ld_resid + col, v[j]);
    }
    if constexpr (sizeof(YT) == 4) {
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        const int col = nw + 16 * j + 4 * l4;
        if (valid && col < p.out_dim) *reinterpret_cast<f32x4*>((float*)p.y + m * p.ldy + col) = f32x4{v[j][0], v[j][1], v[j][2], v[j][3]};
      }
    } else {
      store_row<YT, S::NJ>((YT*)p.y + (valid ? m : 0) * p.ldy, nw, p.out_dim, v, l4, valid);
    }
  }
}

template <typename T, typename YT, typename S>
hipError_t run_linear(const LinearParams& p, hipStream_t s) {
  const int64_t tiles = (p.rows + S::BM - 1) / S::BM * ((p.out_dim + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((k_linear<T, YT, S>), dim3((unsigned)tiles), dim3(S::NW * 64), 0, s, p);
  return hipGetLastError();
}

// Few rows (few_rows.h), 16 NB columns a workgroup and NB outputs a thread.
template <typename T, typename YT, int MT, int NB, int UNROLL>
__global__ __launch_bounds__(16 * 64) void k_linear_few(LinearParams p) {
  constexpr int WAVES = 16;
  typedef FewRows<MT, NB, WAVES> S;
  static_assert(S::ROWS * 16 <= WAVES * 64, "NB outputs a thread");
  __shared__ __attribute__((aligned(16))) float red[S::FLOATS];
  const int n0 = (int)blockIdx.x * S::COLS, l16 = threadIdx.x & 15;
  const uint8_t *x[MT], *w[NB];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = 16 * i + l16;
    x[i] = (const uint8_t*)p.x + (m < p.rows ? m : p.rows - 1) * p.ldx * 2;
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) w[b] = (const uint8_t*)p.w + (int64_t)min(n0 + 16 * b + l16, p.out_dim - 1) * p.dim * 2;
  // (what the outputs need besides the products is loaded first)
  const int m = (int)threadIdx.x / 16, c = (int)threadIdx.x % 16 * NB, col = n0 + c;
  const bool in = m < S::ROWS && m < p.rows && col < p.out_dim;
  float v[NB], r[NB];
#pragma unroll
  for (int e = 0; e < NB; ++e) {
    v[e] = in && p.bias ? bf16_bits_to_f32(p.bias[col + e]) : 0.f;
    r[e] = 0.f;
    if (in && p.resid) {
      const int64_t at = m * p.ld_resid + col + e;
      r[e] = p.resid_dtype == XEMA_F32 ? ((const float*)p.resid)[at] : p.resid_dtype == XEMA_BF16 ? (float)((const bf16*)p.resid)[at]
                                                                                                 : (float)((const f16*)p.resid)[at];
    }
  }
  few_rows_products<T, MT, NB, WAVES, UNROLL>(x, w, p.dim * 2, red);
  if (!in) return;
#pragma unroll
  for (int e = 0; e < NB; ++e) v[e] += few_rows_sum<S>(red, m, c + e);
  if (p.pre) {      // a thread's columns lie in one group of four (NB divides 4)
    uint8_t* const at = (uint8_t*)p.pre + ((int64_t)m * p.out_dim + col) / 4 * Z_GROUP;
#pragma unroll
    for (int e = 0; e < NB; ++e) {
      const uint32_t z = round24(v[e]);
      ((uint16_t*)at)[(col + e) % 4] = (uint16_t)(z >> 16);
      at[8 + (col + e) % 4] = (uint8_t)(z >> 8);
    }
  }
  typedef YT yn __attribute__((ext_vector_type(NB)));
  yn y;
#pragma unroll
  for (int e = 0; e < NB; ++e) y[e] = (YT)((p.act == XEMA_ACT_NONE ? v[e] : activate<false>(v[e], p.act, nullptr)) + r[e]);
  *reinterpret_cast<yn*>((YT*)p.y + m * p.ldy + col) = y;
}

template <typename T, typename YT, int MT, int NB, int UNROLL>
hipError_t run_linear_few(const LinearParams& p, hipStream_t s) {
  hipLaunchKernelGGL((k_linear_few<T, YT, MT, NB, UNROLL>), dim3((p.out_dim + 16 * NB - 1) / (16 * NB)), dim3(16 * 64), 0, s, p);
  return hipGetLastError();
}

template <typename T, typename YT>
hipError_t linear_t(const LinearParams& p, hipStream_t s) {
  const FewPick few = pick_lora_few(p.rows, p.out_dim);
  if (few.cols16 == 1) {
    if (few.rows16 == 1) return run_linear_few<T, YT, 1, 1, 4>(p, s);
    if (few.rows16 == 2) return run_linear_few<T, YT, 2, 1, 4>(p, s);
    if (few.rows16 == 3) return run_linear_few<T, YT, 3, 1, 2>(p, s);
    return run_linear_few<T, YT, 4, 1, 2>(p, s);
  }
  if (few.cols16 == 2) {
    if (few.rows16 == 1) return run_linear_few<T, YT, 1, 2, 4>(p, s);
    if (few.rows16 == 2) return run_linear_few<T, YT, 2, 2, 2>(p, s);
    if (few.rows16 == 3) return run_linear_few<T, YT, 3, 2, 2>(p, s);
    return run_linear_few<T, YT, 4, 2, 1>(p, s);
  }
  if (few.cols16 == 4) return few.rows16 == 1 ? run_linear_few<T, YT, 1, 4, 1>(p, s) : run_linear_few<T, YT, 2, 4, 1>(p, s);
  const FfnRows pick = pick_rows(p.rows, p.out_dim, (p.dim * 2 + KB - 1) / KB);
  LinearParams rest = p;
  if (pick.rows) {
    LinearParams first = p;
    first.rows = pick.rows;
    const hipError_t e = run_linear<T, YT, Tile256x256>(first, s);
    if (e != hipSuccess) return e;
    rest.rows -= pick.rows;
    rest.x = (const T*)p.x + pick.rows * p.ldx;
    rest.y = (YT*)p.y + pick.rows * p.ldy;
    if (p.resid) rest.resid = (const uint8_t*)p.resid + pick.rows * p.ld_resid * (p.resid_dtype == XEMA_F32 ? 4 : 2);
    if (p.pre) rest.pre = (uint8_t*)p.pre + pick.rows * p.out_dim / 4 * Z_GROUP;
  }
  return with_tile(pick.rest, [&](auto shape) { return run_linear<T, YT, decltype(shape)>(rest, s); });
}
template <typename T>
hipError_t linear_y(const LinearParams& p, int y_dtype, hipStream_t s) {
  return y_dtype == XEMA_BF16 ? linear_t<T, bf16>(p, s) : y_dtype == XEMA_F16 ? linear_t<T, f16>(p, s) : linear_t<T, float>(p, s);
}

// dz = dy act'(z), rounded to T, the type of its products' other operands (not stored
// where dz is null), and the column sums of the values before that rounding over each
// chunk of rows.  A workgroup takes 256 columns, 8 a thread, of `chunk` rows, 8 rows
// at a time.
template <typename T, typename DT, bool ACT>
__global__ __launch_bounds__(256) void k_linear_grad(const uint8_t* __restrict__ pre, const DT* __restrict__ dy, int64_t ld_dy, int64_t rows,
                                                     int out_dim, int act, int chunk, T* __restrict__ dz, float* __restrict__ partial) {
  __shared__ float red[8][256 + 8];
  const int c8 = threadIdx.x & 31, r8 = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 256 + c8 * 8;
  const bool in = col < out_dim;
  const int64_t r0 = (int64_t)blockIdx.y * chunk, r1 = r0 + chunk < rows ? r0 + chunk : rows;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  if (in) {
#pragma unroll 2
    for (int64_t r = r0 + r8; r < r1; r += 8) {
      float d[8];
      unpack8(load_raw8(dy + r * ld_dy + col), d);
      if constexpr (ACT) {
        uint32_t w[6];
        const u32x2* at = reinterpret_cast<const u32x2*>(pre + (r * out_dim + col) / 4 * Z_GROUP);
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) w[2 * i + e] = at[i][e];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t* four = w + e / 4 * 3;
          float slope;
          activate<true>(load24(four, four[2], e % 4), act, &slope);
          d[e] *= slope;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += d[e];
      if (dz) store8_as<T>(dz, r * out_dim + col, d);
    }
  }
  if (!partial) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) red[r8][c8 * 8 + e] = sum[e];
  __syncthreads();
  const int c = (int)blockIdx.x * 256 + threadIdx.x;
  if (c < out_dim) {
    float a = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) a += red[r][threadIdx.x];
    partial[(int64_t)blockIdx.y * out_dim + c] = a;
  }
}

struct LinearBwd {
  const void *dz, *w, *x;       // dz [rows, out_dim] (dy itself where it is that already)
  void *dx, *dw;
  float* dx_parts;              // [parts][rows][dim] where dx's k is split
  float* dw_parts;              // [w_parts][out_dim][dim] where the weight's gradient's k (rows) is split
  const float* partial;         // [chunks][out_dim]
  uint16_t* dbias;
  int64_t rows, ldx, ld_dz, ld_dx;
  int dim, out_dim, chunks, parts, w_parts;
};

// dx = dz w: w is read k by k (a row of it is one k).  With parts, workgroup wg
// has part wg / tiles of the steps, its sums kept in fp32.
template <typename T, typename S>
__device__ __forceinline__ TileOut<T> linear_dx_tile(const LinearBwd& p, int wg, uint8_t* smem, int wave, int lane, f32x4 (&acc)[S::MI][S::NJ]) {
  const int tiles = tiles_of<S>(p.rows, p.dim), part = __builtin_amdgcn_readfirstlane(wg / tiles);
  int tm, tn;
  tile_of(wg - part * tiles, (int)((p.rows + S::BM - 1) / S::BM), (p.dim + S::BN - 1) / S::BN, 1024 / S::BM, &tm, &tn);
  const int64_t m0 = (int64_t)tm * S::BM;
  const int n0 = tn * S::BN, steps = (p.out_dim + 63) / 64, each = (steps + p.parts - 1) / p.parts, first = part * each;
  RowOperand<S::BM, S::NW> a;
  ColumnOperand<S::BN, S::NW> b;
  a.init((const T*)p.dz + m0 * p.ld_dz, nullptr, p.rows - m0, p.ld_dz * 2, p.out_dim * 2, 0x7fffffff, wave, lane, first);
  b.init((const T*)p.w + n0, nullptr, p.dim - n0, (int64_t)p.dim * 2, p.out_dim, 0x7fffffff, wave, lane, first);
  tile_products<S, T, ROWS, COLUMNS>(a, b, min(each, steps - first), smem, wave, lane, acc);
  return {(T*)p.dx, p.parts > 1 ? p.dx_parts + part * p.rows * p.dim : nullptr, p.parts > 1 ? p.dim : p.ld_dx,
          m0 + wave / S::WNW * S::WR, p.rows, n0 + wave % S::WNW * S::WC, p.dim};
}

// dw = dz^T x: both operands are read k (row) by k.  With w_parts, workgroup wg
// has part wg / tiles of the rows, its sums kept in fp32.
template <typename T, typename S>
__device__ __forceinline__ TileOut<T> linear_dw_tile(const LinearBwd& p, int wg, uint8_t* smem, int wave, int lane, f32x4 (&acc)[S::MI][S::NJ]) {
  const int tiles = tiles_of<S>(p.out_dim, p.dim), steps = (int)((p.rows + 63) / 64);
  const int part = __builtin_amdgcn_readfirstlane(wg / tiles), each = (steps + p.w_parts - 1) / p.w_parts, first = part * each;
  int tm, tn;
  tile_of(wg - part * tiles, (p.out_dim + S::BM - 1) / S::BM, (p.dim + S::BN - 1) / S::BN, 1024 / S::BM, &tm, &tn);
  const int64_t r0 = (int64_t)first * 64;
  const int m0 = tm * S::BM, n0 = tn * S::BN;
  ColumnOperand<S::BM, S::NW> a;
  ColumnOperand<S::BN, S::NW> b;
  a.init((const T*)p.dz + r0 * p.ld_dz + m0, nullptr, p.out_dim - m0, p.ld_dz * 2, p.rows - r0, 0x7fffffff, wave, lane);
  b.init((const T*)p.x + r0 * p.ldx + n0, nullptr, p.dim - n0, p.ldx * 2, p.rows - r0, 0x7fffffff, wave, lane);
  tile_products<S, T, COLUMNS, COLUMNS>(a, b, min(each, steps - first), smem, wave, lane, acc);
  return {(T*)p.dw, p.w_parts > 1 ? p.dw_parts + (int64_t)part * p.out_dim * p.dim : nullptr, p.dim,
          m0 + wave / S::WNW * S::WR, p.out_dim, n0 + wave % S::WNW * S::WC, p.dim};
}

// The products of the gradient in one launch: dx's tiles, those of the weight's
// gradient, then the bias's gradient (the chunks' column sums, in order).
template <typename T, typename S>
__global__ __launch_bounds__(S::NW * 64, 1) void k_linear_products(LinearBwd p, int dx_tiles, int dw_tiles) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[S::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wg = (int)blockIdx.x;
  if (wg >= dx_tiles + dw_tiles) {
    const int c = (wg - dx_tiles - dw_tiles) * S::NW * 64 + (int)threadIdx.x;
    if (c >= p.out_dim) return;
    float v = 0.f;
#pragma unroll 8
    for (int i = 0; i < p.chunks; ++i) v += p.partial[(int64_t)i * p.out_dim + c];
    // (bf16 in fp16 calls too, as the bias itself: the library's vectors of weights have one type)
    p.dbias[c] = __builtin_bit_cast(uint16_t, (bf16)v);
    return;
  }
  f32x4 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const TileOut<T> o =
      wg < dx_tiles ? linear_dx_tile<T, S>(p, wg, smem, wave, lane, acc) : linear_dw_tile<T, S>(p, wg - dx_tiles, smem, wave, lane, acc);
  if (o.sums) store_sums<S>(acc, o.sums, o.ld, o.row0, o.rows, o.col0, o.cols, lane);
  else store_tile<T, S>(acc, o.out, o.ld, o.row0, o.rows, o.col0, o.cols, lane);
}

template <typename T, typename S>
hipError_t run_linear_products(const LinearBwd& p, bool dx, bool dw, bool db, hipStream_t s) {
  const int dx_tiles = dx ? tiles_of<S>(p.rows, p.dim) * p.parts : 0, dw_tiles = dw ? tiles_of<S>(p.out_dim, p.dim) * p.w_parts : 0;
  const int db_wgs = db ? (p.out_dim + S::NW * 64 - 1) / (S::NW * 64) : 0;
  if (!(dx_tiles + dw_tiles + db_wgs)) return hipSuccess;
  hipLaunchKernelGGL((k_linear_products<T, S>), dim3((unsigned)(dx_tiles + dw_tiles + db_wgs)), dim3(S::NW * 64), 0, s, p, dx_tiles, dw_tiles);
  return hipGetLastError();
}

template <typename T, typename DT>
void run_grad(const xema_linear_bwd_args& a, int chunks, T* dz, float* partial, hipStream_t s) {
  const int chunk = (int)((a.rows + chunks - 1) / chunks);
  const dim3 grid((a.out_dim + 255) / 256, chunks);
  if (a.act == XEMA_ACT_NONE)
    hipLaunchKernelGGL((k_linear_grad<T, DT, false>), grid, dim3(256), 0, s, nullptr, (const DT*)a.dy, a.ld_dy, a.rows, a.out_dim, a.act, chunk, dz, partial);
  else
    hipLaunchKernelGGL((k_linear_grad<T, DT, true>), grid, dim3(256), 0, s, (const uint8_t*)a.pre, (const DT*)a.dy, a.ld_dy, a.rows, a.out_dim, a.act,
                       chunk, dz, partial);
}

template <typename T>
hipError_t linear_bwd_t(const xema_linear_bwd_args& a, hipStream_t s) {
  uint8_t* ws = (uint8_t*)a.workspace;
  float* sums = (float*)(ws + (a.rows * a.out_dim * 2 + 255) / 256 * 256);
  const int chunks = (int)linear_bwd_row_chunks(a.rows);
  float* partial = a.dbias ? sums : nullptr;
  const bool dx = a.dx && a.rows > 0, dw = a.dw, db = a.dbias;
  // dy as it stands, where that is dz already
  const bool ready = a.act == XEMA_ACT_NONE && a.dy_dtype == a.dtype;
  T* dz = ready || !(dx || dw) ? nullptr : (T*)ws;
  hipError_t e = hipSuccess;
  if (a.rows > 0 && (dz || db)) {
    if (a.dy_dtype == XEMA_F32) run_grad<T, float>(a, chunks, dz, partial, s);
    else run_grad<T, T>(a, chunks, dz, partial, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const FfnSplit sx = pick_split(a.rows, a.dim, (a.out_dim + 63) / 64), sw = pick_split(a.out_dim, a.dim, (a.rows + 63) / 64);
  float* dx_parts = sums + linear_bwd_row_chunks(a.rows) * a.out_dim;
  float* dw_parts = dx_parts + linear_bwd_dx_parts(a.rows, a.dim, a.out_dim);
  const LinearBwd p{ready ? a.dy : dz, a.w, a.x, a.dx, a.dw, dx_parts, dw_parts, partial, (uint16_t*)a.dbias,
                    a.rows, a.ldx, ready ? a.ld_dy : a.out_dim, a.ld_dx, a.dim, a.out_dim, a.rows > 0 ? chunks : 0, sx.parts, sw.parts};
  // one launch where both products take the same tile
  if (dx && dw && sx.tile != sw.tile) {
    e = with_tile(sx.tile, [&](auto shape) { return run_linear_products<T, decltype(shape)>(p, true, false, false, s); });
    if (e == hipSuccess) e = with_tile(sw.tile, [&](auto shape) { return run_linear_products<T, decltype(shape)>(p, false, true, db, s); });
  } else {
    e = with_tile(dx ? sx.tile : sw.tile, [&](auto shape) { return run_linear_products<T, decltype(shape)>(p, dx, dw, db, s); });
  }
  if (e == hipSuccess && dx && sx.parts > 1)
    e = run_sum<T>(dx_parts, sx.parts, a.rows * a.dim, a.dim, (T*)a.dx, (T*)a.dx, a.rows * a.dim, a.ld_dx, s);
  if (e == hipSuccess && dw && sw.parts > 1) {
    const int64_t n = (int64_t)a.out_dim * a.dim;
    e = run_sum<T>(dw_parts, sw.parts, n, a.dim, (T*)a.dw, (T*)a.dw, n, a.dim, s);
  }
  return e;
}

}  // namespace

hipError_t launch_linear(const xema_linear_args& a, hipStream_t s) {
  const LinearParams p{a.x, a.w, (const uint16_t*)a.bias, a.resid, a.y, a.pre, a.rows, a.ldx, a.ld_resid, a.ldy,
                       a.dim, a.out_dim, a.act, a.resid_dtype};
  return a.dtype == XEMA_BF16 ? linear_y<bf16>(p, a.y_dtype, s) : linear_y<f16>(p, a.y_dtype, s);
}

int64_t linear_bwd_row_chunks(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(64, (rows + 7) / 8)); }

int64_t linear_bwd_dx_parts(int64_t rows, int dim, int out_dim) {
  const int parts = rows > 0 ? pick_split(rows, dim, (out_dim + 63) / 64).parts : 1;
  return parts > 1 ? parts * rows * dim : 0;
}

int64_t linear_bwd_dw_parts(int64_t rows, int dim, int out_dim) {
  const int parts = pick_split(out_dim, dim, (rows + 63) / 64).parts;
  return parts > 1 ? (int64_t)parts * out_dim * dim : 0;
}

hipError_t launch_linear_bwd(const xema_linear_bwd_args& a, hipStream_t s) {
  return a.dtype == XEMA_BF16 ? linear_bwd_t<bf16>(a, s) : linear_bwd_t<f16>(a, s);
}

}  // namespace xema
