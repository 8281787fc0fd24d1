// Gradient of the attention to an encoder's states (xema_cross.h) on gfx950
// MFMA, in two passes that each form the scores again from q, k and lse:
//
// k_cross_dq: a wave holds 32 queries of one head (q, dout and dq in registers),
// the workgroup's four waves share tiles of 32 states.  It forms D from dout and
// o first, and leaves lse and D for the other pass.
//
// k_cross_dkv: a wave holds 32 states (k, v, dk and dv in registers), the
// workgroup's four waves share tiles of 64 tokens, those of all heads that share
// the states' head one after another, so that their sum needs no exchange.  An
// encoder has few states beside the tokens: the tokens are split over workgroups,
// whose sums k_cross_sums adds in order.
//
// k_cross_both: the two in one launch, side by side, for calls too small to fill the
// CUs with either; dk and dv then form D themselves.
//
// 18432 tokens, 32 heads of 128: dq 127 us with 64 states, 280 with 512 (830
// TFLOP/s), 825 with 2048 (1120); dk and dv 95, 305 (1010) and 1065 (1160).  MFMAs are
// busy 9 and 20% of the cycles with 64 states, 40 and 52% with 512 at 2.0 GHz, 57% with
// 2048 at 1.8.  One pass for all three would form five products in place of seven.
// Past the 128 states of a workgroup dq would have to be added up in memory; up to
// there its waves could add it in LDS, which no kernel here does.
//
// Products are formed transposed (cross_tile.h): a column's scores and their
// gradients feed the last product from their registers.
#include "cross.h"
#include "cross_tile.h"

namespace xema {

namespace {

constexpr int KT = 64;                 // tokens per tile of k_cross_dkv
constexpr int BWD_WAVES = 4;

// fp16 keeps p as 2^14 p: its bits last to p = 2^-28, and 2^14 (1 + rounding) is in range.
template <typename T>
constexpr float P_EXP = std::is_same_v<T, f16> ? 14.f : 0.f;
template <typename T>
constexpr float P_UNIT = std::is_same_v<T, f16> ? 0x1p-14f : 1.f;

struct CrossBwd {
  const void *q, *k, *v, *o, *dout;
  const float* lse;
  const int32_t* kv_lens;
  void *dq, *dk, *dv;
  float *stat_l, *stat_d;              // [batch, heads, q_len rounded up to KT]: lse in log2 units less P_EXP (+infinity: no weights, no token), P_UNIT D
  float* dq_parts;                     // [parts][batch * q_len][heads * head_dim]
  float* dkv_parts;                    // [parts][dk, dv][batch * kv_len][kv_heads * head_dim]
  int64_t ldq, ldk, ldv, ldo, ld_do, ld_dq, ld_dk, ld_dv;
  int batch, heads, kv_heads, head_dim, q_len, kv_len, q_parts, kv_parts;
  Divisor by_q_blocks, by_q_parts, by_kv_blocks, by_kv_parts, by_batch, by_group, by_tiles;
  float c, scale;                      // scale * log2(e), scale
};

constexpr int QKT = 32;                // states per tile of k_cross_dq

// What both passes form has the same bits in either.
// lse in log2 units, +infinity for a token of no states and for one whose lse is too
// coarse (their weights are then zeros).  lse has the roundings of scale log2(e) times
// a score, of a sum and of two products, up to 4 half steps: from 2^22 on e^(s - lse)
// would be off by a factor of e or more, and soon 2^14 p past fp16's range.  (Weights
// held at 1 at most, in place of this, cost an instruction each: up to 5% of a pass.)
constexpr float LSE_END = 0x1p22f;
__device__ __forceinline__ float log2_lse(float lse) {
  float l = lse * LOG2E_F;
  asm("" : "+v"(l));                   // (rounded here, not fused with what it is added to)
  return fabsf(lse) >= LSE_END ? INFINITY : l;
}
// A 16-byte slot's share of D; slots are added in pairs, their pairs in pairs, ...  (o
// is the rounded one, all that the caller keeps: the exact D would take the scores and
// dp of all states before the first dS.)
template <typename F>
__device__ __forceinline__ float slot_dot(const F& d, const F& o) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = fmaf((float)d[e], (float)o[e], sum);
  return sum;
}

// Two stages of K and V; the waves' rows of q pass through stage 1 and a third
// part, those of dout, and of dq in the end, through two more.
template <int HDP>
constexpr int DQ_LDS = 5 * 2 * QKT * Rows<HDP>::RB;

// Workgroup wg of `wgs`.
template <typename T, int HDP>
__device__ __forceinline__ void cross_dq(const CrossBwd& p, int wg, int wgs, uint8_t* lds) {
  typedef Rows<HDP> R;
  typedef typename Mfma<T>::frag frag;
  constexpr int KK = R::KK, ND = R::ND, TILE = QKT * R::RB, SLOTS = R::RB / 16, PER = 64 / SLOTS;
  const auto smem = reinterpret_cast<uint8_t(*)[2 * TILE]>(lds);
  static_assert(BWD_WAVES * WaveRows<HDP>::BYTES == 4 * TILE, "rows of four waves");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  const int t = xcd_order(wg, wgs);
  // (an XCD's range holds all sequences of its heads, whose lengths may differ)
  int block, part, b, rest;
  const int h = p.by_batch.divide(p.by_q_parts.divide(p.by_q_blocks.divide(t, &block), &part), &b), kvh = p.by_group.divide(h, &rest);
  const int n = states_of(p.kv_lens, b, p.kv_len), tiles = (n + QKT - 1) / QKT;
  int first, count;
  part_of(tiles, part, p.q_parts, &first, &count);
  if (!p.dq) count = 0;

  // this wave's tokens: q0 .. q0 + 31, of which `left_q` are there
  const int q0 = (block * BWD_WAVES + wave) * 32, left_q = p.q_len - q0;
  const int64_t tok0 = (int64_t)b * p.q_len + q0, at = (int64_t)h * p.head_dim;
  uint8_t* const q_rows = smem[wave < 2 ? 2 : 1] + (wave & 1) * WaveRows<HDP>::BYTES;
  uint8_t* const d_out_rows = smem[3 + wave / 2] + (wave & 1) * WaveRows<HDP>::BYTES;
  WaveRows<HDP>::load((const T*)p.dout + tok0 * p.ld_do + at, (uint32_t)p.ld_do * 2, p.head_dim, left_q, d_out_rows, lane);
  if (p.dq) WaveRows<HDP>::load((const T*)p.q + tok0 * p.ldq + at, (uint32_t)p.ldq * 2, p.head_dim, left_q, q_rows, lane);
  // (o is met row by row: SLOTS lanes a row, eight elements each)
  const int slot = lane % SLOTS;
  frag o[32 / PER];
#pragma unroll
  for (int c = 0; c < 32 / PER; ++c) {
    const int r = c * PER + lane / SLOTS;
    o[c] = frag{};
    if (r < left_q && slot * 8 < p.head_dim) o[c] = *reinterpret_cast<const frag*>((const T*)p.o + (tok0 + r) * p.ldo + at + slot * 8);
  }

  const int64_t kv_row = (int64_t)b * p.kv_len + (int64_t)first * QKT;
  const uint8_t* kb = (const uint8_t*)((const T*)p.k + kv_row * p.ldk + kvh * p.head_dim);
  const uint8_t* vb = (const uint8_t*)((const T*)p.v + kv_row * p.ldv + kvh * p.head_dim);
  const uint32_t ldk = (uint32_t)p.ldk * 2, ldv = (uint32_t)p.ldv * 2;
  TileLoads<HDP, QKT, BWD_WAVES> lk, lv;
  lk.init(ldk, p.head_dim, wave, lane);
  lv.init(ldv, p.head_dim, wave, lane);
  int left = n - first * QKT;
  auto issue = [&](int stage) {
    lk.issue(kb, ldk, left, smem[stage], wave);
    lv.issue(vb, ldv, left, smem[stage] + TILE, wave);
    kb += (int64_t)QKT * ldk;
    vb += (int64_t)QKT * ldv;
    left -= QKT;
  };
  if (count > 0) issue(0);

  const int q = q0 + c32;
  const bool valid = c32 < left_q;
  const float lse = valid ? p.lse[((int64_t)b * p.heads + h) * p.q_len + q] : -INFINITY;
  const float L = log2_lse(lse);
  AlongRows<T, HDP> ra;
  AcrossRows<T, HDP> rx;
  ra.init(lane);
  rx.init(lane);
  frag qf[KK], df[KK];
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  asm volatile("" ::: "memory");
  WaveRows<HDP>::template read<T>(q_rows, ra, qf);
  WaveRows<HDP>::template read<T>(d_out_rows, ra, df);
#pragma unroll
  for (int c = 0; c < 32 / PER; ++c) {
    const int r = c * PER + lane / SLOTS;
    const frag d = *reinterpret_cast<const frag*>(d_out_rows + r * R::RB + ((slot ^ R::swz(r)) << 4));
    float sum = slot_dot(d, o[c]);
#pragma unroll
    for (int x = 1; x < SLOTS; x *= 2) sum += __shfl_xor(sum, x, 64);
    // (in place of the rows of q, which are read: LDS takes a wave's accesses in order)
    if (slot == 0) reinterpret_cast<float*>(q_rows)[r] = sum;
  }
  asm volatile("" ::: "memory");
  const float D = reinterpret_cast<const float*>(q_rows)[c32];
  const int padded = (p.q_len + KT - 1) / KT * KT;
  if (p.stat_l && part == 0 && q < padded && !hi) {
    const int64_t st = ((int64_t)b * p.heads + h) * padded + q;
    p.stat_l[st] = valid ? L - P_EXP<T> : INFINITY;
    p.stat_d[st] = valid ? D * P_UNIT<T> : 0.f;
  }
  if (!p.dq) return;

  f32x16 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  // (stages by name, so that a fragment's address is a register and an immediate)
  auto tile = [&](int i, auto stage) {
    constexpr int ST = decltype(stage)::value;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __syncthreads();
    if (i + 1 < count) issue(ST ^ 1);
    const uint8_t *ks = smem[ST], *vs = ks + TILE;
    const int here = n - (first + i) * QKT;
    f32x16 s, dp;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) s = Mfma<T>::run(ra.read(ks, 0, kk), qf[kk], kk ? s : f32x16{});
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) dp = Mfma<T>::run(ra.read(vs, 0, kk), df[kk], kk ? dp : f32x16{});
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.c, -L)) * (dp[r] - D);
    if (here < QKT) {
      const int mine = here - 4 * hi;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= mine) s[r] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const frag f = pack8<T>(s, u);
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] = Mfma<T>::run(rx.read(ks, 16 * u, d), f, acc[d]);
    }
  };
  for (int i = 0; i < count; i += 2) {
    tile(i, std::integral_constant<int, 0>());
    if (i + 1 < count) tile(i + 1, std::integral_constant<int, 1>());
  }
  if (p.q_parts > 1)
    store_column_f32<ND>(p.dq_parts + (part * (int64_t)p.batch * p.q_len + tok0 + c32) * p.heads * p.head_dim + at, p.head_dim, acc, p.scale, hi, valid);
  else
    WaveRows<HDP>::template store<T>((T*)p.dq + tok0 * p.ld_dq + at, p.ld_dq, p.head_dim, left_q, acc, p.scale, d_out_rows, lane);
}

// Two stages of q, dout, and lse and D of their tokens.
template <int HDP>
constexpr int DKV_LDS = 2 * (2 * KT * Rows<HDP>::RB + 2 * KT * 4);

// Workgroup wg of `wgs`.  OWN: lse and D are taken from their sources here, not from dq's pass.
template <typename T, int HDP, bool OWN>
__device__ __forceinline__ void cross_dkv(const CrossBwd& p, int wg, int wgs, uint8_t* lds) {
  typedef Rows<HDP> R;
  typedef typename Mfma<T>::frag frag;
  constexpr int KK = R::KK, ND = R::ND, TILE = KT * R::RB;
  const auto smem = reinterpret_cast<uint8_t(*)[2 * TILE]>(lds);
  const auto stats = reinterpret_cast<float(*)[2][KT]>(lds + 4 * TILE);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  const int t = xcd_order(wg, wgs);
  int block, part, b;
  const int kvh = p.by_batch.divide(p.by_kv_parts.divide(p.by_kv_blocks.divide(t, &block), &part), &b), group = (int)p.by_group.d;
  const int n = states_of(p.kv_lens, b, p.kv_len);
  const int state0 = (block * BWD_WAVES + wave) * 32, state = state0 + c32;
  // tiles: those of the first head's tokens, the second's, ...
  const int per_head = (p.q_len + KT - 1) / KT;
  int first, count;
  part_of(group * per_head, part, p.kv_parts, &first, &count);
  if (block * BWD_WAVES * 32 >= n) count = 0;       // (no states here: zeros)

  const uint32_t ldq = (uint32_t)p.ldq * 2, ld_do = (uint32_t)p.ld_do * 2;
  typedef RepeatedLoads<HDP, KT, BWD_WAVES> Loads;
  int tile, g = p.by_tiles.divide(first, &tile);        // of the next tile to load
  auto issue = [&](int stage) {
    const int h = kvh * group + g, t0 = tile * KT, rows = p.q_len - t0;
    const int64_t at = (int64_t)b * p.q_len + t0;
    // (tokens past the last repeat it, and weigh 0 by their lse: rows of zeros would make NaN of an infinite k)
    Loads::issue((const uint8_t*)((const T*)p.q + at * p.ldq + (int64_t)h * p.head_dim), ldq, p.head_dim, rows, smem[stage], wave);
    Loads::issue((const uint8_t*)((const T*)p.dout + at * p.ld_do + (int64_t)h * p.head_dim), ld_do, p.head_dim, rows, smem[stage] + TILE, wave);
    if (!OWN && wave < 2) {
      const float* const st = (wave ? p.stat_d : p.stat_l) + (((int64_t)b * p.heads + h) * per_head + tile) * KT;
      load_lds4(make_rsrc(st, 4 * KT), (uint8_t*)stats[stage][wave], lane * 4);
    }
    if (++tile == per_head) {
      tile = 0;
      ++g;
    }
  };
  if (count > 0) issue(0);

  frag kf[KK], vf[KK];
  const int64_t kv_row = (int64_t)b * p.kv_len + min(state, p.kv_len - 1), at = (int64_t)kvh * p.head_dim;
  // (states behind the last one: their columns are not kept, whatever they hold)
  load_column<T, HDP>((const T*)p.k + kv_row * p.ldk + at, p.head_dim, hi, kf);
  load_column<T, HDP>((const T*)p.v + kv_row * p.ldv + at, p.head_dim, hi, vf);
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[d][r] = dv[d][r] = 0.f;
  AlongRows<T, HDP> ra;
  AcrossRows<T, HDP> rx;
  ra.init(lane);
  rx.init(lane);
  const bool busy = state0 < n;
  for (int i = 0; i < count; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (OWN) {
      // four threads a token: 16-byte slots quarter, quarter + 4, ... of its rows of o and dout
      const int th = wave * 64 + lane_again(), r = th >> 2, quarter = th & 3;
      int at_tile;
      const int h = kvh * group + p.by_tiles.divide(first + i, &at_tile), token = at_tile * KT + r;
      const bool there = token < p.q_len;
      const int64_t row = (int64_t)b * p.q_len + token;
      frag o[ND];
      float lse = -INFINITY;
#pragma unroll
      for (int j = 0; j < ND; ++j) {
        const int slot = quarter + 4 * j;
        o[j] = frag{};
        if (there && slot * 8 < p.head_dim) o[j] = *reinterpret_cast<const frag*>((const T*)p.o + row * p.ldo + (int64_t)h * p.head_dim + slot * 8);
      }
      if (there) lse = p.lse[((int64_t)b * p.heads + h) * p.q_len + token];
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      __syncthreads();
      const uint8_t* const rows = smem[i & 1] + TILE + r * R::RB;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < ND; ++j) {
        sum[j] = slot_dot(*reinterpret_cast<const frag*>(rows + (((quarter + 4 * j) ^ R::swz(r)) << 4)), o[j]);
        sum[j] += __shfl_xor(sum[j], 1, 64);
        sum[j] += __shfl_xor(sum[j], 2, 64);
      }
      const float D = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if (quarter == 0) {
        stats[i & 1][0][r] = log2_lse(lse) - P_EXP<T>;
        stats[i & 1][1][r] = there ? D * P_UNIT<T> : 0.f;
      }
    } else {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    }
    __syncthreads();
    if (i + 1 < count) issue((i + 1) & 1);
    if (!busy) continue;
    const uint8_t *qs = smem[i & 1], *ds = qs + TILE;
    const float *sl = stats[i & 1][0], *sd = stats[i & 1][1];
    // (32 tokens at a time: both blocks at once would not fit the registers beside dk and dv of wide heads)
#pragma unroll 1
    for (int blk = 0; blk < 2; ++blk) {
      forget(ra.base);
      forget(rx.base);
      f32x16 s, dp;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) s = Mfma<T>::run(ra.read(qs, 32 * blk, kk), kf[kk], kk ? s : f32x16{});
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) dp = Mfma<T>::run(ra.read(ds, 32 * blk, kk), vf[kk], kk ? dp : f32x16{});
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 L = *reinterpret_cast<const f32x4*>(sl + 32 * blk + 8 * r4 + 4 * hi);
        const f32x4 D = *reinterpret_cast<const f32x4*>(sd + 32 * blk + 8 * r4 + 4 * hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * r4 + e;
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.c, -L[e]));
          dp[r] = s[r] * fmaf(dp[r], P_UNIT<T>, -D[e]);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const frag pf = pack8<T>(s, u), df = pack8<T>(dp, u);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          dv[d] = Mfma<T>::run(rx.read(ds, 32 * blk + 16 * u, d), pf, dv[d]);
          dk[d] = Mfma<T>::run(rx.read(qs, 32 * blk + 16 * u, d), df, dk[d]);
        }
      }
    }
  }
  const int again = lane_again(), half = again >> 5, mine = state0 + (again & 31);
  if (mine >= n) {
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[d][r] = dv[d][r] = 0.f;
  }
  const bool valid = mine < p.kv_len;
  const int64_t row = (int64_t)b * p.kv_len + mine;
  if (p.kv_parts > 1) {
    const int64_t width = (int64_t)p.kv_heads * p.head_dim, one = (int64_t)p.batch * p.kv_len * width;
    float* const out = p.dkv_parts + part * 2 * one + row * width + at;
    store_column_f32<ND>(out, p.head_dim, dk, p.scale, half, valid);
    store_column_f32<ND>(out + one, p.head_dim, dv, P_UNIT<T>, half, valid);
  } else {
    store_column<T, ND>((T*)p.dk + row * p.ld_dk + at, p.head_dim, dk, p.scale, half, valid);
    store_column<T, ND>((T*)p.dv + row * p.ld_dv + at, p.head_dim, dv, P_UNIT<T>, half, valid);
  }
}

template <typename T, int HDP>
__global__ __launch_bounds__(BWD_WAVES * 64, 2) void k_cross_dq(CrossBwd p) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[DQ_LDS<HDP>];
  cross_dq<T, HDP>(p, (int)blockIdx.x, (int)gridDim.x, lds);
}

template <typename T, int HDP>
__global__ __launch_bounds__(BWD_WAVES * 64, 2) void k_cross_dkv(CrossBwd p) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[DKV_LDS<HDP>];
  cross_dkv<T, HDP, false>(p, (int)blockIdx.x, (int)gridDim.x, lds);
}

// Both of a call that leaves CUs idle either way, side by side: kv_wgs workgroups for dk and dv, the rest for dq.
template <typename T, int HDP>
__global__ __launch_bounds__(BWD_WAVES * 64, 2) void k_cross_both(CrossBwd p, int kv_wgs) {
  static_assert(DKV_LDS<HDP> <= DQ_LDS<HDP>);
  __shared__ __attribute__((aligned(1024))) uint8_t lds[DQ_LDS<HDP>];
  const int wg = (int)blockIdx.x;
  if (wg < kv_wgs) cross_dkv<T, HDP, true>(p, wg, kv_wgs, lds);
  else cross_dq<T, HDP>(p, wg - kv_wgs, (int)gridDim.x - kv_wgs, lds);
}

// Outputs from their parts, in order: matrix blockIdx.y of up to two, n elements
// in rows of `width`; part i of it lies i `stride` past its first.
template <typename T>
__global__ __launch_bounds__(256) void k_cross_sums(const float* __restrict__ sums, int parts, int64_t stride, int64_t n, int width, T* out0, T* out1,
                                                    int64_t ld0, int64_t ld1) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= n) return;
  const bool second = blockIdx.y;
  const float* const from = sums + (second ? n : 0) + at;
  f32x4 s = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 4
  for (int i = 1; i < parts; ++i) s += *reinterpret_cast<const f32x4*>(from + i * stride);
  t4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (T)s[e];
  const int64_t r = at / width;
  *reinterpret_cast<t4*>((second ? out1 : out0) + r * (second ? ld1 : ld0) + (at - r * width)) = o;
}

// The sums of `parts` parts to one matrix, or to two.
template <typename T>
hipError_t run_cross_sums(const float* sums, int parts, int64_t rows, int width, T* out0, T* out1, int64_t ld0, int64_t ld1, hipStream_t s) {
  const int64_t n = rows * width;
  const int outs = out1 ? 2 : 1;
  hipLaunchKernelGGL((k_cross_sums<T>), dim3((unsigned)((n / 4 + 255) / 256), outs), dim3(256), 0, s, sums, parts, outs * n, n, width, out0, out1, ld0, ld1);
  return hipGetLastError();
}

template <typename T, int HDP>
hipError_t run_cross_bwd(CrossBwd p, bool both, hipStream_t s) {
  const int64_t q_wgs = (int64_t)p.batch * p.heads * ((p.q_len + 32 * BWD_WAVES - 1) / (32 * BWD_WAVES)) * p.q_parts;
  const int64_t kv_wgs = (int64_t)p.batch * p.kv_heads * ((p.kv_len + 32 * BWD_WAVES - 1) / (32 * BWD_WAVES)) * p.kv_parts;
  const dim3 block(BWD_WAVES * 64);
  if (both && p.dq && p.dk && q_wgs && kv_wgs) {
    p.stat_l = p.stat_d = nullptr;
    hipLaunchKernelGGL((k_cross_both<T, HDP>), dim3((unsigned)(q_wgs + kv_wgs)), block, 0, s, p, (int)kv_wgs);
  } else {
    if (q_wgs) hipLaunchKernelGGL((k_cross_dq<T, HDP>), dim3((unsigned)q_wgs), block, 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.dk && kv_wgs) hipLaunchKernelGGL((k_cross_dkv<T, HDP>), dim3((unsigned)kv_wgs), block, 0, s, p);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.dq && q_wgs && p.q_parts > 1)
    e = run_cross_sums<T>(p.dq_parts, p.q_parts, (int64_t)p.batch * p.q_len, p.heads * p.head_dim, (T*)p.dq, nullptr, p.ld_dq, 0, s);
  if (e == hipSuccess && p.dk && kv_wgs && p.kv_parts > 1)
    e = run_cross_sums<T>(p.dkv_parts, p.kv_parts, (int64_t)p.batch * p.kv_len, p.kv_heads * p.head_dim, (T*)p.dk, (T*)p.dv, p.ld_dk, p.ld_dv, s);
  return e;
}

template <typename T>
hipError_t cross_bwd_t(const CrossBwd& p, bool both, hipStream_t s) {
  if (p.head_dim <= 32) return run_cross_bwd<T, 32>(p, both, s);
  if (p.head_dim <= 64) return run_cross_bwd<T, 64>(p, both, s);
  return p.head_dim <= 96 ? run_cross_bwd<T, 96>(p, both, s) : run_cross_bwd<T, 128>(p, both, s);
}

// The workspace, in floats: lse and D, then the parts of dq, then those of dk and dv.
struct BwdSpace {
  CrossBwdPick pick;
  int64_t stats, dq, dkv;
};
BwdSpace bwd_space(const CrossShape& c) {
  const int64_t q_rows = (int64_t)c.batch * c.q_len, kv_rows = (int64_t)c.batch * c.kv_len;
  BwdSpace w{pick_cross_bwd(c.batch, c.heads, c.kv_heads, c.head_dim, c.q_len, c.kv_len), 0, 0, 0};
  w.stats = (int64_t)c.batch * c.heads * ((c.q_len + KT - 1) / KT * KT);
  w.dq = w.pick.q_parts > 1 ? w.pick.q_parts * q_rows * c.heads * c.head_dim : 0;
  w.dkv = w.pick.kv_parts > 1 ? w.pick.kv_parts * 2 * kv_rows * c.kv_heads * c.head_dim : 0;
  return w;
}

}  // namespace

int64_t cross_attn_bwd_workspace(const CrossShape& c) {
  const BwdSpace w = bwd_space(c);
  return (2 * w.stats + w.dq + w.dkv) * 4;
}

hipError_t launch_cross_attn_bwd(const xema_cross_attn_bwd_args& a, hipStream_t s) {
  const BwdSpace w = bwd_space({a.batch, a.heads, a.kv_heads, a.head_dim, a.q_len, a.kv_len});
  const CrossBwdPick pick = a.dq ? w.pick : without_dq(w.pick);
  float* const ws = (float*)a.workspace;
  auto blocks = [](int n) { return n > 0 ? (n + 32 * BWD_WAVES - 1) / (32 * BWD_WAVES) : 1; };
  const CrossBwd p{a.q, a.k, a.v, a.o, a.dout, a.lse, a.kv_lens, a.dq, a.dk, a.dv, ws, ws + w.stats, ws + 2 * w.stats, ws + 2 * w.stats + w.dq,
                   a.ldq, a.ldk, a.ldv, a.ldo, a.ld_do, a.ld_dq, a.ld_dk, a.ld_dv, a.batch, a.heads, a.kv_heads, a.head_dim, a.q_len, a.kv_len,
                   pick.q_parts, pick.kv_parts, Divisor(blocks(a.q_len)), Divisor(pick.q_parts), Divisor(blocks(a.kv_len)),
                   Divisor(pick.kv_parts), Divisor(a.batch), Divisor(a.heads / a.kv_heads), Divisor(a.q_len > 0 ? (a.q_len + KT - 1) / KT : 1), a.scale * LOG2E_F, a.scale};
  return a.dtype == XEMA_BF16 ? cross_bwd_t<bf16>(p, pick.both, s) : cross_bwd_t<f16>(p, pick.both, s);
}

}  // namespace xema
