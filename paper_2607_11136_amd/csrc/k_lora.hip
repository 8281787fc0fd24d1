// A projection shared by requests with low-rank adapters of their own
// (xema_op_lora_linear, xema_ffn.h): a reduction t = scale x a^T, then the shared
// product with t b^T added to its accumulators.  The reduction is a launch of its
// own because every column tile of the product needs all of t.  t is kept as two
// 16-bit values, a rounding and its remainder: b's MFMA then runs over 2 rank k's,
// which for ranks to 16 is the one k-step that rank alone would take.
//
// 18432 x 4096 x 4096, rank 32, an adapter for each of four sequences: 47 us reducing
// (x once from HBM: 29 us) and 485 us (the product alone 460, 1350 TFLOP/s);
// 3204 x 1544 x 4104, rank 64, seven requests: 13 and 60 us (rows of 3088 bytes
// straddle the 128-byte lines; the adapters' loads are bound by their latency,
// 1.3 us a k-step); 48 single tokens of 4096 x 4096: 5 and 18 us (x from L2 for
// every 16 columns).
#include "device_common.h"
#include "few_rows.h"
#include "ffn.h"
#include "mma_tile.h"

namespace xema {

namespace {

struct LoraParams {
  const void *x, *w; const uint16_t* bias;
  const void *a, *b; const float* scale;
  const int32_t* ids;
  void *y, *t;                 // t: [rows, 2 rank], the scaled x a^T as rounded value and remainder
  int64_t rows, ldx, ldy;
  int dim, out_dim, rank, n_adapters;
};

__device__ __forceinline__ bool has_adapter(const LoraParams& p, int id) { return id >= 0 && id < p.n_adapters; }

constexpr int REDUCE_WAVES = 8;

// Value and remainder of s in T, eight ranks of one row.
template <typename T>
__device__ __forceinline__ void store_reduced(T* t, int rank, int q, const float s[8]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  t8 hi, lo;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // (one fp32 value for both: the product that made it, fused into the first
    // conversion, may round to the other neighbour than the remainder is of)
    const float v = as_rounded_f32(s[e]);
    hi[e] = (T)v;
    // (an infinity leaves no remainder: taken from itself it would be NaN)
    lo[e] = __builtin_isinf((float)hi[e]) ? (T)0.f : (T)(v - (float)hi[e]);
  }
  *reinterpret_cast<t8*>(t + q) = hi;
  *reinterpret_cast<t8*>(t + rank + q) = lo;
}

// t[r] = scale[i] x[r] a[i]^T as value and remainder.  A workgroup per block of
// 16 MT rows and 16 RT ranks multiplies them on MFMA with the adapter that the
// rows share, its waves a part of k each; where a block has several adapters
// (requests that meet in it, or single tokens), with one after the other, and a
// row keeps its own.  While the blocks are fewer than the CUs, what bounds it is
// how fast one CU gets its part of a and x from L2 (256 KiB in 10 us): the ranks
// are then dealt to several workgroups (pick_reduce).
template <typename T, int MT, int RT>
__global__ __launch_bounds__(REDUCE_WAVES * 64) void k_lora_reduce(LoraParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int RB = 16 * MT, RR = 16 * RT;
  __shared__ __attribute__((aligned(16))) float red[REDUCE_WAVES][RB][RR + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, l4 = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.x * RB;
  const int q0 = (int)blockIdx.y * RR, ranks = min(p.rank - q0, RR);
  const int id = lane < RB && m0 + lane < p.rows ? p.ids[m0 + lane] : -2;
  const T* xr[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + 16 * i + l16;
    xr[i] = (const T*)p.x + (m < p.rows ? m : p.rows - 1) * p.ldx;
  }
  const int span = (p.dim + REDUCE_WAVES * 64 - 1) / (REDUCE_WAVES * 64) * 64;
  const int begin = wave * span, end = min(begin + span, p.dim);
  for (uint64_t todo = __ballot(has_adapter(p, id)); todo;) {
    const int one = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
    const uint64_t rows = __ballot(id == one);
    todo &= ~rows;
    const float scale = p.scale[one];
    const T* ar[RT];
#pragma unroll
    for (int q = 0; q < RT; ++q) ar[q] = (const T*)p.a + ((int64_t)one * p.rank + min(q0 + 16 * q + l16, p.rank - 1)) * p.dim;
    f32x4 acc[MT][RT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int q = 0; q < RT; ++q) acc[i][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int UNROLL = RT + MT <= 5 ? 2 : 1;
    for (int k0 = begin; k0 < end; k0 += 64 * UNROLL) {
      frag fx[UNROLL][2][MT], fa[UNROLL][2][RT];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = k0 + u * 64 + 32 * h + 8 * l4;
          const bool in = k < end;
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            fx[u][h][i] = frag{};
            if (in) fx[u][h][i] = *reinterpret_cast<const frag*>(xr[i] + k);
          }
#pragma unroll
          for (int q = 0; q < RT; ++q) {
            fa[u][h][q] = frag{};
            if (in) fa[u][h][q] = *reinterpret_cast<const frag*>(ar[q] + k);
          }
        }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < RT; ++q) acc[i][q] = Frag<T>::run(fa[u][h][q], fx[u][h][i], acc[i][q]);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int q = 0; q < RT; ++q) *reinterpret_cast<f32x4*>(&red[wave][16 * i + l16][16 * q + 4 * l4]) = acc[i][q];
    __syncthreads();
    for (int at = threadIdx.x; at < RB * ranks / 8; at += REDUCE_WAVES * 64) {
      const int row = at / (ranks / 8), q = at % (ranks / 8) * 8;
      if (!(rows >> row & 1)) continue;
      float s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[e] = 0.f;
#pragma unroll
        for (int w = 0; w < REDUCE_WAVES; ++w) s[e] += red[w][row][q + e];
        s[e] *= scale;
      }
      store_reduced<T>((T*)p.t + (m0 + row) * 2 * p.rank, p.rank, q0 + q, s);
    }
    if (todo) __syncthreads();
  }
}

// The same for few rows: a workgroup per row and 32 ranks, four ranks a wave;
// where that leaves waves over, k in parts too.  (All ranks of a row in one
// workgroup: 64 rows of 4096, rank 128, 50 us with the product; so 40.)
constexpr int ROW_RANKS = REDUCE_WAVES * 4;
template <typename T>
__global__ __launch_bounds__(REDUCE_WAVES * 64) void k_lora_reduce_rows(LoraParams p) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  __shared__ float sums[REDUCE_WAVES * 4];                       // [parts][ranks of this workgroup]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = blockIdx.x;
  const int own = p.ids[r];
  if (!has_adapter(p, own)) return;
  const float scale = p.scale[own];
  const int q0 = (int)blockIdx.y * ROW_RANKS, ranks = min(p.rank - q0, ROW_RANKS);
  const int batches = ranks / 4, parts = REDUCE_WAVES / batches;
  const int batch = wave % batches, part = wave / batches;       // (part `parts`: waves that no batch needs)
  const T* x = (const T*)p.x + r * p.ldx;
  const T* a = (const T*)p.a + ((int64_t)own * p.rank + q0 + batch * 4) * p.dim;
  if (part < parts) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = part * 512 + lane * 8; k < p.dim; k += parts * 512) {
      const t8 u = *reinterpret_cast<const t8*>(x + k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const t8 v = *reinterpret_cast<const t8*>(a + (int64_t)i * p.dim + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i] = fmaf((float)u[e], (float)v[e], s[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = wave_sum(s[i]);
      if (lane == 0) sums[part * ranks + batch * 4 + i] = s[i];
    }
  }
  __syncthreads();
  if ((int)threadIdx.x >= ranks / 8) return;
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    s[e] = 0.f;
    for (int w = 0; w < parts; ++w) s[e] += sums[w * ranks + threadIdx.x * 8 + e];
    s[e] *= scale;
  }
  store_reduced<T>((T*)p.t + r * 2 * p.rank, p.rank, q0 + (int)threadIdx.x * 8, s);
}

// The adapters of a wave's rows: the first PASSES different ones, each met by
// all rows on MFMA, and the rows that have yet another.
constexpr int PASSES = 3;
template <int MI>
struct WaveAdapters {
  int id[MI];          // of this lane's row of each block of 16
  int one[PASSES];     // -1 for none (scalars)
  int others;          // blocks with a row of a further adapter, a bit each (scalar)
  __device__ __forceinline__ void init(const LoraParams& p, int64_t m0, int lane) {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t m = m0 + 16 * i + (lane & 15);
      id[i] = m < p.rows ? p.ids[m] : -2;
    }
#pragma unroll
    for (int n = 0; n < PASSES; ++n) {
      one[n] = -1;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const uint64_t left = __ballot(further(p, id[i], n));
        if (left && one[n] < 0) one[n] = __builtin_amdgcn_readlane(id[i], __builtin_ctzll(left));
      }
    }
    others = 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) others |= __ballot(further(p, id[i], PASSES)) ? 1 << i : 0;
  }
  // a row's adapter, if it is none of the first n
  __device__ __forceinline__ bool further(const LoraParams& p, int i, int n) const {
    bool f = has_adapter(p, i);
#pragma unroll
    for (int k = 0; k < PASSES; ++k)
      if (k < n) f = f && i != one[k];
    return f;
  }
};

// b as the remainders meet it: zeros in place of infinities and NaN (16-bit
// elements whose exponent is all ones), which the values have met with t's sign
// already: a remainder, zero or of the other sign, would make NaN of infinity.
// (A full exponent and its own lowest bit carry into the sign's place.)  us
// without and with it and the second pass of add_to_others: 1000 x 4096 x 4096,
// rank 64, mixed rows 211 and 213; 128 rows, rank 16, mixed 33 and 35; 3204 x 1544 x
// 4104, rank 64, seven requests 75 and 75.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type finite_only(typename Frag<T>::type f) {
  constexpr uint32_t EXP = std::is_same_v<T, bf16> ? 0x7f807f80u : 0x7c007c00u, LOW = std::is_same_v<T, bf16> ? 0x00800080u : 0x04000400u;
  u32x4 w = __builtin_bit_cast(u32x4, f);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const uint32_t full = ((w[d] & EXP) + LOW) >> 15 & 0x00010001u;
    w[d] &= ~((full << 16) - full);
  }
  return __builtin_bit_cast(typename Frag<T>::type, w);
}

// acc += t[r] b[i]^T for the rows with adapter `one` (-1: none): the values'
// MFMA k-range and the remainders', over the same b.  The products are formed
// for all rows, and kept for those (a product with zeros in the place of
// another row's t would not do: the adapter may hold infinities).
template <typename T, typename S>
__device__ __forceinline__ void add_adapter(const LoraParams& p, int64_t m0, int n0, int lane, const WaveAdapters<S::MI>& who, int one,
                                            f32x4 (&acc)[S::MI][S::NJ]) {
  typedef typename Frag<T>::type frag;
  const int l16 = lane & 15, l4 = lane >> 4;
  const int slots = one >= 0 ? p.rank / 4 : 0, rs = p.rank / 8;    // 16-byte slots of a row of t and of a row of b
  const T* b = (const T*)p.b + (int64_t)one * p.out_dim * p.rank;
  // k-steps loaded at once, as the registers beside acc allow (the latency is paid once for both)
  constexpr int AHEAD = S::MI == 8 ? 1 : 2;
#pragma unroll 1
  for (int k = 0; k < slots; k += 4 * AHEAD) {
    frag fb[AHEAD][S::NJ], ft[AHEAD][S::MI];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int at = k + 4 * u + l4;
      const bool in = at < slots;
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        fb[u][j] = frag{};
        if (in) fb[u][j] = *reinterpret_cast<const frag*>(b + min(n0 + 16 * j + l16, p.out_dim - 1) * p.rank + (at < rs ? at : at - rs) * 8);
      }
#pragma unroll
      for (int i = 0; i < S::MI; ++i) {
        const int64_t m = m0 + 16 * i + l16;
        ft[u][i] = frag{};
        if (in) ft[u][i] = *reinterpret_cast<const frag*>((const T*)p.t + (m < p.rows ? m : p.rows - 1) * 2 * p.rank + at * 8);
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (k + 4 * u + 3 >= rs)                 // (a step that no remainder is in is left as it is)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) fb[u][j] = k + 4 * u + l4 >= rs ? finite_only<T>(fb[u][j]) : fb[u][j];
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      const bool keep = who.id[i] == one;
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        f32x4 v = acc[i][j];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v = Frag<T>::run(fb[u][j], ft[u][i], v);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = keep ? v[e] : acc[i][j][e];
      }
    }
  }
}

// sum += t b^T for one row and C columns, eight ranks at a time.
template <typename T, int C>
__device__ __forceinline__ void add_row(const LoraParams& p, const T* t, const T* const (&b)[C], float (&sum)[C]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
#pragma unroll 4
  for (int q = 0; q < p.rank; q += 8) {
    const t8 hi = *reinterpret_cast<const t8*>(t + q), lo = *reinterpret_cast<const t8*>(t + p.rank + q);
    t8 v[C];
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = *reinterpret_cast<const t8*>(b[c] + q);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[c] = fmaf((float)hi[e] + (float)lo[e], (float)v[c][e], sum[c]);
  }
}

// acc += t[r] b[i]^T for the rows with further adapters: a block's adapters in
// turn, TOGETHER of them at once as the registers beside acc allow, each on MFMA
// over the block's 16 rows; bound by the latency of b's lines from L2.  A lane
// per row would read each line of b in eight 16-byte pieces, from L2 again each
// time.  With the reduction, that and this, us, adapters drawn per row of 24,
// rank 64: 1000 x 4096 x 4096 268 and 221, 1000 x 2048 x 8192 303 and 219.
template <typename T, typename S>
__device__ __forceinline__ void add_to_others(const LoraParams& p, int64_t m0, int n0, int lane, const WaveAdapters<S::MI>& who,
                                             f32x4 (&acc)[S::MI][S::NJ]) {
  typedef typename Frag<T>::type frag;
  constexpr int TOGETHER = S::MI == 8 ? 1 : 2;
  const int l16 = lane & 15, l4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    if (!(who.others >> i & 1)) continue;
    const int64_t m = m0 + 16 * i + l16;
    const T* t = (const T*)p.t + (m < p.rows ? m : p.rows - 1) * 2 * p.rank;
    const bool further = who.further(p, who.id[i], PASSES);
    f32x4 before[S::NJ];
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) before[j] = acc[i][j];
    // Where a sum comes out infinite or NaN all are formed again with finite_only
    // (in every pass that took 3 to 10% of the whole call, and where all is finite
    // it changes nothing).
    for (bool again = false;; again = true) {
      for (uint64_t todo = __ballot(further); todo;) {
        int one[TOGETHER];
        f32x4 v[TOGETHER][S::NJ];
#pragma unroll
        for (int u = 0; u < TOGETHER; ++u) {
          one[u] = todo ? __builtin_amdgcn_readlane(who.id[i], __builtin_ctzll(todo)) : one[0];
          todo &= ~__ballot(who.id[i] == one[u]);
#pragma unroll
          for (int j = 0; j < S::NJ; ++j) v[u][j] = acc[i][j];
        }
        for (int k0 = 0; k0 < p.rank; k0 += 32) {
          const int k = k0 + l4 * 8;
          frag fb[TOGETHER][S::NJ], hi = {}, lo = {};
#pragma unroll
          for (int u = 0; u < TOGETHER; ++u)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) fb[u][j] = frag{};
          if (k < p.rank) {
#pragma unroll
            for (int u = 0; u < TOGETHER; ++u) {
              const T* b = (const T*)p.b + (int64_t)one[u] * p.out_dim * p.rank + k;
#pragma unroll
              for (int j = 0; j < S::NJ; ++j) fb[u][j] = *reinterpret_cast<const frag*>(b + min(n0 + 16 * j + l16, p.out_dim - 1) * p.rank);
            }
            hi = *reinterpret_cast<const frag*>(t + k);
            lo = *reinterpret_cast<const frag*>(t + p.rank + k);
          }
#pragma unroll
          for (int u = 0; u < TOGETHER; ++u)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) {
              v[u][j] = Frag<T>::run(fb[u][j], hi, v[u][j]);
              if (again) fb[u][j] = finite_only<T>(fb[u][j]);
            }
#pragma unroll
          for (int u = 0; u < TOGETHER; ++u)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) v[u][j] = Frag<T>::run(fb[u][j], lo, v[u][j]);
        }
#pragma unroll
        for (int u = 0; u < TOGETHER; ++u)
#pragma unroll
          for (int j = 0; j < S::NJ; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = who.id[i] == one[u] ? v[u][j][e] : acc[i][j][e];
      }
      if (again) break;
      float zero = 0.f;                        // (an infinity or NaN makes NaN of it)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) zero = fmaf(acc[i][j][e], 0.f, zero);
      if (!__ballot(further && zero != 0.f)) break;
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) acc[i][j] = further ? before[j] : acc[i][j];
    }
  }
}

template <typename T, typename YT, typename S>
__global__ __launch_bounds__(S::NW * 64, 1) void k_lora_project(LoraParams p) {
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
  WaveAdapters<S::MI> who;
  who.init(p, mw, lane);
  f32x4 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  tile_products<S, T, ROWS, ROWS>(a, b, (kbytes + KB - 1) / KB, smem, wave, lane, acc,
                                  [&] {
#pragma unroll
                                    for (int n = 0; n < PASSES; ++n) add_adapter<T, S>(p, mw, nw, lane, who, who.one[n], acc);
                                  });
  add_to_others<T, S>(p, mw, nw, lane, who, acc);

  float bv[S::NJ][4] = {};
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) load4f<uint16_t>(p.bias + min(nw + 16 * j + 4 * l4, p.out_dim - 4), bv[j]);
  }
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const bool valid = who.id[i] >= -1;
    float v[S::NJ][4];
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j][e] = who.id[i] < p.n_adapters ? acc[i][j][e] + bv[j][e] : __builtin_nanf("");
    store_row<YT, S::NJ>((YT*)p.y + (valid ? mw + 16 * i + l16 : 0) * p.ldy, nw, p.out_dim, v, l4, valid);
  }
}

template <typename T, typename YT, typename S>
hipError_t run_project(const LoraParams& p, hipStream_t s) {
  const int64_t tiles = (p.rows + S::BM - 1) / S::BM * ((p.out_dim + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((k_lora_project<T, YT, S>), dim3((unsigned)tiles), dim3(S::NW * 64), 0, s, p);
  return hipGetLastError();
}

// Few rows (few_rows.h), 16 NB columns a workgroup.
template <typename T, typename YT, int MT, int NB, int FEW_WAVES, int UNROLL>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_lora_project_few(LoraParams p) {
  typedef FewRows<MT, NB, FEW_WAVES> S;
  static_assert(S::ROWS * 16 <= FEW_WAVES * 64, "NB outputs a thread");
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
  // NB outputs a thread (what they need of their row besides is loaded first)
  const int m = (int)threadIdx.x / 16, c = (int)threadIdx.x % 16 * NB, col = n0 + c;
  const bool in = m < S::ROWS && m < p.rows && col < p.out_dim;
  const int id = in ? p.ids[m] : -2;
  float v[NB];
#pragma unroll
  for (int e = 0; e < NB; ++e) v[e] = in && p.bias ? bf16_bits_to_f32(p.bias[col + e]) : 0.f;
  few_rows_products<T, MT, NB, FEW_WAVES, UNROLL>(x, w, p.dim * 2, red);
  if (id < -1) return;
#pragma unroll
  for (int e = 0; e < NB; ++e) v[e] += few_rows_sum<S>(red, m, c + e);
  if (id >= p.n_adapters) {
#pragma unroll
    for (int e = 0; e < NB; ++e) v[e] = __builtin_nanf("");
  } else if (id >= 0) {
    const T* b[NB];
#pragma unroll
    for (int e = 0; e < NB; ++e) b[e] = (const T*)p.b + ((int64_t)id * p.out_dim + col + e) * p.rank;
    add_row<T, NB>(p, (const T*)p.t + (int64_t)m * 2 * p.rank, b, v);
  }
  typedef YT yn __attribute__((ext_vector_type(NB)));
  yn y;
#pragma unroll
  for (int e = 0; e < NB; ++e) y[e] = (YT)v[e];
  *reinterpret_cast<yn*>((YT*)p.y + m * p.ldy + col) = y;
}

template <typename T, typename YT, int MT, int NB, int FEW_WAVES, int UNROLL>
hipError_t run_project_few(const LoraParams& p, hipStream_t s) {
  hipLaunchKernelGGL((k_lora_project_few<T, YT, MT, NB, FEW_WAVES, UNROLL>), dim3((p.out_dim + 16 * NB - 1) / (16 * NB)), dim3(FEW_WAVES * 64), 0, s, p);
  return hipGetLastError();
}

template <typename T, int MT, int RT>
hipError_t run_reduce_rt(const LoraParams& p, hipStream_t s) {
  hipLaunchKernelGGL((k_lora_reduce<T, MT, RT>), dim3((unsigned)((p.rows + 16 * MT - 1) / (16 * MT)), (p.rank + 16 * RT - 1) / (16 * RT)),
                     dim3(REDUCE_WAVES * 64), 0, s, p);
  return hipGetLastError();
}

template <typename T, int MT>
hipError_t run_reduce(const LoraParams& p, int ranks16, hipStream_t s) {
  return ranks16 == 4 ? run_reduce_rt<T, MT, 4>(p, s) : ranks16 == 2 ? run_reduce_rt<T, MT, 2>(p, s) : run_reduce_rt<T, MT, 1>(p, s);
}

template <typename T>
hipError_t reduce(const LoraParams& p, hipStream_t s) {
  const ReducePick pick = pick_reduce(p.rows, p.rank);
  switch (pick.rows16) {
    case 0:
      hipLaunchKernelGGL((k_lora_reduce_rows<T>), dim3((unsigned)p.rows, (p.rank + ROW_RANKS - 1) / ROW_RANKS), dim3(REDUCE_WAVES * 64), 0, s, p);
      return hipGetLastError();
    case 1: return run_reduce<T, 1>(p, pick.ranks16, s);
    case 2: return run_reduce<T, 2>(p, pick.ranks16, s);
    default: return run_reduce<T, 3>(p, pick.ranks16, s);
  }
}

template <typename T, typename YT>
hipError_t lora_t(const LoraParams& p, hipStream_t s) {
  if (p.n_adapters) {
    const hipError_t e = reduce<T>(p, s);
    if (e != hipSuccess) return e;
  }
  const FewPick few = pick_lora_few(p.rows, p.out_dim);
  if (few.cols16 == 1) {
    if (few.rows16 == 1) return run_project_few<T, YT, 1, 1, 16, 4>(p, s);
    if (few.rows16 == 2) return run_project_few<T, YT, 2, 1, 16, 4>(p, s);
    if (few.rows16 == 3) return run_project_few<T, YT, 3, 1, 16, 2>(p, s);
    return run_project_few<T, YT, 4, 1, 16, 2>(p, s);
  }
  if (few.cols16 == 2) {
    if (few.rows16 == 1) return run_project_few<T, YT, 1, 2, 16, 4>(p, s);
    if (few.rows16 == 2) return run_project_few<T, YT, 2, 2, 16, 2>(p, s);
    if (few.rows16 == 3) return run_project_few<T, YT, 3, 2, 16, 2>(p, s);
    return run_project_few<T, YT, 4, 2, 16, 1>(p, s);
  }
  if (few.cols16 == 4) return few.rows16 == 1 ? run_project_few<T, YT, 1, 4, 16, 1>(p, s) : run_project_few<T, YT, 2, 4, 16, 1>(p, s);
  return with_tile(pick_tile(p.rows, p.out_dim, (p.dim * 2 + KB - 1) / KB), [&](auto shape) { return run_project<T, YT, decltype(shape)>(p, s); });
}

}  // namespace

hipError_t launch_lora_linear(const xema_lora_args& a, hipStream_t s) {
  const LoraParams p{a.x, a.w, (const uint16_t*)a.bias, a.a, a.b, a.scale, a.row_adapter, a.y, a.workspace,
                     a.rows, a.ldx, a.ldy, a.dim, a.out_dim, a.rank, a.n_adapters};
  if (a.dtype == XEMA_BF16) return a.y_dtype == XEMA_BF16 ? lora_t<bf16, bf16>(p, s) : lora_t<bf16, f16>(p, s);
  return a.y_dtype == XEMA_BF16 ? lora_t<f16, bf16>(p, s) : lora_t<f16, f16>(p, s);
}

}  // namespace xema
