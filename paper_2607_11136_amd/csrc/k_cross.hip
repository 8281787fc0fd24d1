// Attention to an encoder's states (xema_cross.h), forward, on gfx950 MFMA:
// one pass over the states with a running reference maximum and sum.
//
// k_cross: a wave holds 32 queries of one head; the workgroup's four waves share
// tiles of 32 states, two stages in LDS.  S^T = K Q^T leaves a lane with one
// query's scores, whose exponentials feed O^T = V^T P^T from their registers
// (cross_tile.h).  The reference maximum moves only when a tile's sum of
// exponentials passes PMAX, so the common path takes no maximum: P stays below
// PMAX, and the largest weight is at least 1 against the sum.  Tiles of 32 states
// leave three workgroups a CU (four at head dims to 64), which hide each other's
// loads, barriers and exponentials: 2 x 28612 tokens, 32 heads of 128, 512 and 256
// states 415 to 475 us by the card, 510 with tiles of 64 and two workgroups.
// 18432 tokens, 32 heads of 128: 64 states 63 us (4.8 TB/s), 512 states 201 (770
// TFLOP/s), 2048 states 590 (1045); MFMAs are busy 13, 46 and 60% of the cycles, at
// 2.5, 1.95 and 1.7 GHz.  A workgroup's loads of q, products, exponentials and stores
// of o follow one another, which other workgroups hide in part; the more of it they
// hide, the lower the card's clock.
//
// k_cross_few: single tokens.  The tokens of all heads that share a state's head
// are one block of up to 32 queries, and the workgroup's waves take tiles of 32
// states in turn, each with stages of its own and no barrier, so that the states
// stream from HBM; the waves' sums meet in LDS at the end (4 sequences of 16384
// to 4096 states, 32 heads on 8 of 128: 39 us and 4 for the join, 3.8 TB/s).
//
// Where a call has too few workgroups for the CUs, its states are split into
// parts, each workgroup's sums kept in fp32 with their maximum, and k_cross_join
// joins them.
#include "cross.h"
#include "cross_tile.h"

namespace xema {

namespace {

constexpr int KT = 32;                 // states per tile
constexpr int CROSS_WAVES = 4;
constexpr float PMAX = 4096.f;         // (fp16 P stays finite; 2^12 beside sums in fp32 loses nothing)
constexpr float LOWEST = -0x1.fffffep127f;   // a reference that no finite score is below; -infinity less it stays one
// References from here on have steps of 2 and more: what their own rounding leaves of
// c s - m, formed in one step, would be whole factors of 2 in every weight.
constexpr float COARSE = 0x1p24f;

struct CrossParams {
  const void *q, *k, *v;
  void* o;
  float* lse;
  const int32_t* kv_lens;
  float* part_o;                       // [parts][rows][head_dim]
  float2* part_ml;                     // [parts][rows]: maximum (log2 units), sum
  int64_t ldq, ldk, ldv, ldo;
  int64_t rows;                        // batch * heads * q_len
  int batch, heads, kv_heads, head_dim, q_len, kv_len, parts, blocks;     // blocks of queries of a head
  Divisor by_blocks, by_parts, by_batch, by_kv_heads, by_group;
  float c;                             // scale * log2(e)
};

// The running softmax of a lane's column, and its sum over V.
template <int ND>
struct Column {
  float m, l;                          // reference (log2 units); this lane's share of the sum
  f32x16 o[ND];
  __device__ __forceinline__ void init() {
    m = LOWEST;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  }
  // scores (of NB blocks of 32 states) to weights 2^(c s - m).  Coarse references
  // take every tile through the branch, whose c s is rounded as the maximum's is.
  template <int NB>
  __device__ __forceinline__ void weigh(f32x16 (&s)[NB], float c, bool first) {
    f32x16 p[NB];
    float sum = first ? 0.f : exps<NB>(s, p, 1.f, c);
    const bool grow = first || !(pair_max(sum) <= PMAX) || !(fabsf(m) < COARSE);
    if (__builtin_amdgcn_ballot_w64(grow)) {
      float top = s[0][0] * c;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r] * c);
      top = fmaxf(pair_max(top), m);
      const float to = grow ? top : m, f = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= f;
      const bool fine = fabsf(m) < COARSE;
      sum = exps<NB>(s, p, fine ? 1.f : c, fine ? c : 1.f);
    }
    l += sum;
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = p[b];
  }
  // p = 2^((a s) b - m), a s rounded; returns this lane's sum
  template <int NB>
  __device__ __forceinline__ float exps(const f32x16 (&s)[NB], f32x16 (&p)[NB], float a, float b) const {
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[n][r] = __builtin_amdgcn_exp2f(fmaf(a * s[n][r], b, -m));
        part[r & 3] += p[n][r];
      }
    return (part[0] + part[1]) + (part[2] + part[3]);
  }
};

// Scores of states at or past `left` become -infinity: block b's register r is state 32 b + 8 (r / 4) + 4 hi + r % 4.
template <int NB>
__device__ __forceinline__ void mask_from(f32x16 (&s)[NB], int left, int hi) {
  const int mine = left - 4 * hi;      // (against constants, which take no registers)
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (32 * b + 8 * (r >> 2) + (r & 3) >= mine) s[b][r] = -INFINITY;
}

// ln of the sum, of which l is what 2^m leaves (v_log_f32 is log2); -infinity for none.
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f; }

template <typename T, int HDP>
__global__ __launch_bounds__(CROSS_WAVES * 64, HDP <= 64 ? 4 : 3) void k_cross(CrossParams p) {
  typedef Rows<HDP> R;
  typedef typename Mfma<T>::frag frag;
  constexpr int KK = R::KK, ND = R::ND, TILE = KT * R::RB;
  // two stages of K and V, and one tile more: the waves' rows of queries and of
  // outputs pass through that and the stage that holds no tile then
  __shared__ __attribute__((aligned(1024))) uint8_t smem[3][2 * TILE];
  static_assert(CROSS_WAVES * WaveRows<HDP>::BYTES == 4 * TILE, "rows of four waves");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  // workgroup -> (head, batch, part, block of queries): an XCD's range holds all
  // sequences of its heads, whose lengths may differ
  const int t = xcd_order((int)blockIdx.x, (int)gridDim.x);
  int block, part, b, rest;
  const int h = p.by_batch.divide(p.by_parts.divide(p.by_blocks.divide(t, &block), &part), &b), kvh = p.by_group.divide(h, &rest);
  const int n = states_of(p.kv_lens, b, p.kv_len), tiles = (n + KT - 1) / KT;
  int first, count;
  part_of(tiles, part, p.parts, &first, &count);
  auto rows_at = [&](int free) { return smem[wave < 2 ? 2 : free] + (wave & 1) * WaveRows<HDP>::BYTES; };

  // this wave's queries: q0 .. q0 + 31, of which `left_q` are there
  const int q0 = (block * CROSS_WAVES + wave) * 32, left_q = p.q_len - q0;
  const int64_t tok0 = (int64_t)b * p.q_len + q0;
  WaveRows<HDP>::load((const T*)p.q + tok0 * p.ldq + (int64_t)h * p.head_dim, (uint32_t)p.ldq * 2, p.head_dim, left_q, rows_at(1), lane);

  const int64_t kv_row = (int64_t)b * p.kv_len + (int64_t)first * KT;
  const uint8_t* kb = (const uint8_t*)((const T*)p.k + kv_row * p.ldk + kvh * p.head_dim);
  const uint8_t* vb = (const uint8_t*)((const T*)p.v + kv_row * p.ldv + kvh * p.head_dim);
  const uint32_t ldk = (uint32_t)p.ldk * 2, ldv = (uint32_t)p.ldv * 2;
  TileLoads<HDP, KT, CROSS_WAVES> lk, lv;
  lk.init(ldk, p.head_dim, wave, lane);
  lv.init(ldv, p.head_dim, wave, lane);
  int left = n - first * KT;                     // states from the next tile to load on
  auto issue = [&](int stage) {
    lk.issue(kb, ldk, left, smem[stage], wave);
    lv.issue(vb, ldv, left, smem[stage] + TILE, wave);
    kb += (int64_t)KT * ldk;
    vb += (int64_t)KT * ldv;
    left -= KT;
  };
  if (count > 0) issue(0);

  AlongRows<T, HDP> rk;
  AcrossRows<T, HDP> rv;
  rk.init(lane);
  rv.init(lane);
  frag qf[KK];
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  asm volatile("" ::: "memory");
  WaveRows<HDP>::template read<T>(rows_at(1), rk, qf);
  Column<ND> col;
  col.init();
  // (stages by name, so that a fragment's address is a register and an immediate)
  auto tile = [&](int i, auto stage) {
    constexpr int ST = decltype(stage)::value;
    // tile i has landed (this wave's part: vmcnt; the others': the barrier), and
    // every wave has read tile i - 1 (or its queries), whose stage tile i + 1 takes
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __syncthreads();
    if (i + 1 < count) issue(ST ^ 1);
    const uint8_t *ks = smem[ST], *vs = ks + TILE;
    if constexpr (ND == 4) {        // (all of a wide head's addresses beside its sums would not fit the registers)
      forget(rk.base);
      forget(rv.base);
    }
    f32x16 s[1];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) s[0] = Mfma<T>::run(rk.read(ks, 0, kk), qf[kk], kk ? s[0] : f32x16{});
    const int here = n - (first + i) * KT;
    if (here < KT) mask_from<1>(s, here, hi);
    col.template weigh<1>(s, p.c, i == 0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const frag pf = pack8<T>(s[0], u);
#pragma unroll
      for (int d = 0; d < ND; ++d) col.o[d] = Mfma<T>::run(rv.read(vs, 16 * u, d), pf, col.o[d]);
    }
  };
  for (int i = 0; i < count; i += 2) {
    tile(i, std::integral_constant<int, 0>());
    if (i + 1 < count) tile(i + 1, std::integral_constant<int, 1>());
  }
  const float l = pair_sum(col.l);
  const bool valid = c32 < left_q;
  const int64_t row = ((int64_t)b * p.heads + h) * p.q_len + q0 + (valid ? c32 : 0);
  if (p.parts > 1) {
    const int64_t at = part * p.rows + row;
    store_column_f32<ND>(p.part_o + at * p.head_dim, p.head_dim, col.o, 1.f, hi, valid);
    if (valid && !hi) p.part_ml[at] = float2{col.m, l};
    return;
  }
  // (the stage that the last tile is not in)
  WaveRows<HDP>::template store<T>((T*)p.o + tok0 * p.ldo + (int64_t)h * p.head_dim, p.ldo, p.head_dim, left_q, col.o, l == 0.f ? 0.f : 1.f / l,
                                   rows_at(count & 1), lane);
  if (p.lse && valid && !hi) p.lse[row] = lse_of(col.m, l);
}

constexpr int FT = 32;                 // states per tile of a wave of k_cross_few
constexpr int FEW_WAVES = 2;

template <typename T, int HDP>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_cross_few(CrossParams p) {
  typedef Rows<HDP> R;
  typedef typename Mfma<T>::frag frag;
  constexpr int KK = R::KK, ND = R::ND, TILE = FT * R::RB, STAGE = 2 * TILE, LOADS = 2 * TileLoads<HDP, FT, 1>::LOADS;
  constexpr int ROW = HDP + 4;                   // fp32 of a column where the waves' sums meet (padded against bank conflicts)
  constexpr int LDS = FEW_WAVES * (2 * STAGE > 32 * ROW * 4 ? 2 * STAGE : 32 * ROW * 4);
  __shared__ __attribute__((aligned(1024))) uint8_t smem[LDS];
  __shared__ float2 ml[FEW_WAVES][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  // workgroup -> (batch, state head, block of queries, part)
  const int t = (int)blockIdx.x;
  int part, block, kvh;
  const int b = p.by_kv_heads.divide(p.by_blocks.divide(p.by_parts.divide(t, &part), &block), &kvh), group = (int)p.by_group.d;
  const int n = states_of(p.kv_lens, b, p.kv_len), tiles = (n + FT - 1) / FT;
  // parts of kv_len, so that a short sequence has few: the rest leave an empty sum
  const int each = ((p.kv_len + FT - 1) / FT + p.parts - 1) / p.parts, first = part * each, count = min(each, tiles - first);
  if (count <= 0 && p.parts > 1) {
    const int r = block * 32 + (int)threadIdx.x, rows = p.q_len * group;
    if ((int)threadIdx.x < 32 && r < rows) {
      int g;
      const int token = p.by_group.divide(r, &g), h = kvh * group + g;
      p.part_ml[part * p.rows + ((int64_t)b * p.heads + h) * p.q_len + token] = float2{LOWEST, 0.f};
    }
    return;
  }
  // this wave's tiles: first + wave, first + wave + FEW_WAVES, ...
  const int mine = max(count - wave + FEW_WAVES - 1, 0) / FEW_WAVES;

  uint8_t* const stages = smem + wave * 2 * STAGE;
  const uint32_t ldk = (uint32_t)p.ldk * 2, ldv = (uint32_t)p.ldv * 2;
  const int64_t kv_row = (int64_t)b * p.kv_len;
  const T* const kh = (const T*)p.k + kv_row * p.ldk + kvh * p.head_dim;
  const T* const vh = (const T*)p.v + kv_row * p.ldv + kvh * p.head_dim;
  TileLoads<HDP, FT, 1> lk, lv;
  lk.init(ldk, p.head_dim, 0, lane);
  lv.init(ldv, p.head_dim, 0, lane);
  // (tiles past the wave's last have no states: their loads read nothing)
  auto issue = [&](int i) {
    const int64_t at = i < mine ? (int64_t)(first + wave + i * FEW_WAVES) * FT : n;
    uint8_t* const st = stages + (i & 1) * STAGE;
    lk.issue((const uint8_t*)(kh + at * p.ldk), ldk, n - (int)at, st, 0);
    lv.issue((const uint8_t*)(vh + at * p.ldv), ldv, n - (int)at, st + TILE, 0);
  };
  issue(0);
  issue(1);

  // query r of the block: token r / group of the head kvh * group + r % group
  const int r0 = block * 32 + c32, rows = p.q_len * group;
  int g;
  const int token = p.by_group.divide(min(r0, rows - 1), &g), h = kvh * group + g;
  frag qf[KK];
  load_column<T, HDP>((const T*)p.q + ((int64_t)b * p.q_len + token) * p.ldq + (int64_t)h * p.head_dim, p.head_dim, hi, qf);
  Column<ND> col;
  col.init();
  AlongRows<T, HDP> rk;
  AcrossRows<T, HDP> rv;
  rk.init(lane);
  rv.init(lane);
  for (int i = 0; i < mine; ++i) {
    // the wave's tile i has landed, tile i + 1 may be in flight
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(LOADS));
    asm volatile("" ::: "memory");
    const uint8_t *ks = stages + (i & 1) * STAGE, *vs = ks + TILE;
    f32x16 s[1];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) s[0] = Mfma<T>::run(rk.read(ks, 0, kk), qf[kk], kk ? s[0] : f32x16{});
    const int here = n - (first + wave + i * FEW_WAVES) * FT;
    if (here < FT) mask_from<1>(s, here, hi);
    col.template weigh<1>(s, p.c, i == 0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const frag pf = pack8<T>(s[0], u);
#pragma unroll
      for (int d = 0; d < ND; ++d) col.o[d] = Mfma<T>::run(rv.read(vs, 16 * u, d), pf, col.o[d]);
    }
    // its reads are done: tile i + 2 takes its stage
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);          // lgkmcnt(0)
    issue(i + 2);
  }
  // the loads that ran ahead write to LDS: let them finish, then the waves' sums meet
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  const float l = pair_sum(col.l);
  if (!hi) ml[wave][c32] = float2{col.m, l};
  __syncthreads();
  float* const sums = (float*)smem;
  float top = LOWEST;
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) top = fmaxf(top, ml[w][c32].x);
  store_column_f32<ND>(sums + (wave * 32 + c32) * ROW, HDP, col.o, __builtin_amdgcn_exp2f(col.m - top), hi, true);
  __syncthreads();
  // THREADS threads a query, four columns each at a time
  constexpr int THREADS = FEW_WAVES * 2;
  const int q = (int)threadIdx.x / THREADS, at = block * 32 + q;
  if (at >= rows) return;
  float m = LOWEST, sum = 0.f;
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) m = fmaxf(m, ml[w][q].x);
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) sum += ml[w][q].y * __builtin_amdgcn_exp2f(ml[w][q].x - m);
  const int tq = p.by_group.divide(at, &g), hq = kvh * group + g;
  const int64_t row = ((int64_t)b * p.heads + hq) * p.q_len + tq, prow = part * p.rows + row;
  T* const orow = (T*)p.o + ((int64_t)b * p.q_len + tq) * p.ldo + (int64_t)hq * p.head_dim;
  const float f = p.parts > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
  for (int e = (int)threadIdx.x % THREADS * 4; e < p.head_dim; e += 4 * THREADS) {
    f32x4 v = *reinterpret_cast<const f32x4*>(sums + q * ROW + e);
#pragma unroll
    for (int w = 1; w < FEW_WAVES; ++w) v += *reinterpret_cast<const f32x4*>(sums + (w * 32 + q) * ROW + e);
    if (p.parts > 1) {
      *reinterpret_cast<f32x4*>(p.part_o + prow * p.head_dim + e) = v;
    } else {
      typedef T t4 __attribute__((ext_vector_type(4)));
      t4 o;
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x] = (T)(v[x] * f);
      *reinterpret_cast<t4*>(orow + e) = o;
    }
  }
  if (threadIdx.x % THREADS) return;
  if (p.parts > 1) p.part_ml[prow] = float2{m, sum};
  else if (p.lse) p.lse[row] = lse_of(m, sum);
}

// The parts of a (batch, head, token)'s sums (up to 64), joined in a fixed order: a
// workgroup a row, a lane a part's maximum and sum, then sixteen threads a part,
// eight columns each, sixteen parts at a time.
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
template <typename T>
__global__ __launch_bounds__(256) void k_cross_join(CrossParams p) {
  __shared__ __attribute__((aligned(16))) float sums[16][128];
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, e = ((int)threadIdx.x & 15) * 8, first = (int)threadIdx.x / 16;
  const float2 ml = lane < p.parts ? p.part_ml[lane * p.rows + row] : float2{LOWEST, 0.f};
  const float m = wave_max(ml.x), w = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - m), sum = wave_sum(ml.y * w);
  // (a part of no sum may not have been written; one whose sum weighs nothing here may hold a NaN)
  const uint64_t written = __builtin_amdgcn_ballot_w64(ml.y != 0.f);
  f32x4 v[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  for (int i0 = 0; i0 < p.parts; i0 += 16) {
    const int i = i0 + first;
    const float f = __shfl(w, i & 63, 64);
    if (i < p.parts && (written >> i & 1) && e < p.head_dim) {
      const f32x4* const at = reinterpret_cast<const f32x4*>(p.part_o + (i * p.rows + row) * p.head_dim + e);
#pragma unroll
      for (int x = 0; x < 2; ++x) v[x] += at[x] * f;
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) *reinterpret_cast<f32x4*>(&sums[first][e + 4 * x]) = v[x];
  __syncthreads();
  if (threadIdx.x == 0 && p.lse) p.lse[row] = lse_of(m, sum);
  const int c = (int)threadIdx.x * 2;
  if (c >= p.head_dim) return;
  float o[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int x = 0; x < 2; ++x) o[x] += sums[i][c + x];
  const int64_t bh = row / p.q_len, token = row - bh * p.q_len, b = bh / p.heads, h = bh - b * p.heads;
  typedef T t2 __attribute__((ext_vector_type(2)));
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<t2*>((T*)p.o + (b * p.q_len + token) * p.ldo + h * p.head_dim + c) = t2{(T)(o[0] * f), (T)(o[1] * f)};
}

// The same for many rows: LANES threads a row, eight columns each, part by part.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void k_cross_join_rows(CrossParams p) {
  const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + (int)threadIdx.x / LANES;
  const int e = (int)threadIdx.x % LANES * 8;
  if (row >= p.rows || e >= p.head_dim) return;
  float m = LOWEST;
#pragma unroll 4
  for (int i = 0; i < p.parts; ++i) m = fmaxf(m, p.part_ml[i * p.rows + row].x);
  f32x4 v[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  float sum = 0.f;
#pragma unroll 4
  for (int i = 0; i < p.parts; ++i) {
    const float2 ml = p.part_ml[i * p.rows + row];
    if (ml.y == 0.f) continue;      // (a part of no sum may not have been written; one whose sum weighs nothing here may hold a NaN)
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    sum = fmaf(ml.y, f, sum);
    const f32x4* const at = reinterpret_cast<const f32x4*>(p.part_o + (i * p.rows + row) * p.head_dim + e);
#pragma unroll
    for (int x = 0; x < 2; ++x) v[x] += at[x] * f;
  }
  if (e == 0 && p.lse) p.lse[row] = lse_of(m, sum);
  const int64_t bh = row / p.q_len, token = row - bh * p.q_len, b = bh / p.heads, h = bh - b * p.heads;
  typedef T t8 __attribute__((ext_vector_type(8)));
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  t8 o;
#pragma unroll
  for (int x = 0; x < 8; ++x) o[x] = (T)(v[x / 4][x % 4] * f);
  *reinterpret_cast<t8*>((T*)p.o + (b * p.q_len + token) * p.ldo + h * p.head_dim + e) = o;
}

template <typename T, int LANES>
hipError_t run_join_rows(const CrossParams& p, hipStream_t s) {
  hipLaunchKernelGGL((k_cross_join_rows<T, LANES>), dim3((unsigned)((p.rows * LANES + 255) / 256)), dim3(256), 0, s, p);
  return hipGetLastError();
}

template <typename T, int HDP>
hipError_t run_cross(CrossParams p, const CrossPick& pick, hipStream_t s) {
  p.blocks = pick.blocks;
  p.by_blocks = Divisor(pick.blocks);
  const unsigned wgs = (unsigned)((int64_t)p.batch * (pick.few ? p.kv_heads : p.heads) * pick.blocks * pick.parts);
  if (pick.few) hipLaunchKernelGGL((k_cross_few<T, HDP>), dim3(wgs), dim3(FEW_WAVES * 64), 0, s, p);
  else hipLaunchKernelGGL((k_cross<T, HDP>), dim3(wgs), dim3(CROSS_WAVES * 64), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t cross_t(const CrossParams& p, const CrossPick& pick, hipStream_t s) {
  hipError_t e;
  if (p.head_dim <= 32) e = run_cross<T, 32>(p, pick, s);
  else if (p.head_dim <= 64) e = run_cross<T, 64>(p, pick, s);
  else if (p.head_dim <= 96) e = run_cross<T, 96>(p, pick, s);
  else e = run_cross<T, 128>(p, pick, s);
  if (e != hipSuccess || p.parts == 1) return e;
  switch (pick_join(p.rows, p.head_dim)) {
    case 8: return run_join_rows<T, 8>(p, s);
    case 16: return run_join_rows<T, 16>(p, s);
  }
  hipLaunchKernelGGL((k_cross_join<T>), dim3((unsigned)p.rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

CrossPick pick_of(const CrossShape& c) { return pick_cross(c.batch, c.heads, c.kv_heads, c.head_dim, c.q_len, c.kv_len); }

}  // namespace

int64_t cross_attn_workspace(const CrossShape& c) {
  const int64_t rows = (int64_t)c.batch * c.heads * c.q_len;
  const int parts = rows ? pick_of(c).parts : 1;
  return parts > 1 ? parts * rows * (c.head_dim * 4 + 8) : 0;
}

hipError_t launch_cross_attn(const xema_cross_attn_args& a, hipStream_t s) {
  const CrossPick pick = pick_of({a.batch, a.heads, a.kv_heads, a.head_dim, a.q_len, a.kv_len});
  const int64_t rows = (int64_t)a.batch * a.heads * a.q_len;
  float* const part_o = (float*)a.workspace;
  const CrossParams p{a.q, a.k, a.v, a.o, a.lse, a.kv_lens, part_o, (float2*)(part_o + pick.parts * rows * a.head_dim),
                      a.ldq, a.ldk, a.ldv, a.ldo, rows, a.batch, a.heads, a.kv_heads, a.head_dim, a.q_len, a.kv_len, pick.parts, 0,
                      Divisor(1), Divisor(pick.parts), Divisor(a.batch), Divisor(a.kv_heads), Divisor(a.heads / a.kv_heads), a.scale * LOG2E_F};
  return a.dtype == XEMA_BF16 ? cross_t<bf16>(p, pick, s) : cross_t<f16>(p, pick, s);
}

}  // namespace xema
