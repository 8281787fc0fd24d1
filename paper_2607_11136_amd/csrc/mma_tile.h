// One output tile of a matrix product on MFMA, for operands in either order,
// widths that no tile divides and 16-bit or e4m3 elements: C[m][n] = sum over
// k of A(m, k) B(n, k).
//
// Both operands go through LDS in steps of 128 bytes of k a row (64 16-bit or
// 128 8-bit elements), loaded straight from memory (buffer_load ... lds).  An
// operand stored row by row with k contiguous ("rows") keeps 128-byte LDS rows
// in eight 16-byte slots, slot j of row r at j ^ ((r >> 1) & 7), so that the
// 16 rows that a fragment read meets lie in other banks.  An operand stored k
// by k ("columns": a gradient's transposed product) keeps its k rows, and
// fragments come through the transposing LDS read (ds_read_b64_tr_b16: 16
// lanes read 4 k rows of 16 columns, each lane receives one column's four k);
// its 32-byte chunks are permuted by the k row, so that the eight k rows that
// 32 lanes meet lie in other banks.
//
// Measured, all CUs busy: a 128-byte step of a 256 x 256 tile takes 1.41 us in
// either order and either width (the clock that the power limit leaves; MFMAs
// busy 67 to 76% of the cycles, no LDS bank conflicts), a tile 6.6 us besides;
// 16-bit products of 8192 x 4096 x 22016 run at 1260 to 1360 TFLOP/s, e4m3 of 17776
// x 4096 x 32768 at 2750.
//
// Everything past an operand's end is read as zero: rows and columns by a
// per-lane offset that the buffer's range check refuses, k of the last step
// likewise.  No load leaves the operand.
#pragma once

#include <type_traits>

#include "device_common.h"
#include "mma.h"
#include "tile_rules.h"

namespace xema {

struct e4m3 { uint8_t bits; };
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int KB = 128;                       // bytes of k per row and step
constexpr uint32_t OUT_OF_RANGE = 0x80000000u;

enum OperandOrder { ROWS, COLUMNS };

// 16-byte loads of an LDS tile of R rows, a row of memory being k.
template <int R, int NW>
struct RowLoads {
  static constexpr int LOADS = R / 8 / NW;    // 1 KiB loads per wave and step
  static_assert(LOADS * 8 * NW == R, "load split");
  uint32_t off[LOADS];
  int left[2];                                // bytes of k from this lane's slot on, even and odd loads
  // byte of k of this lane's slot in load c of a step
  static __device__ __forceinline__ int slot(int c, int wave, int lane) {
    return ((lane % 8) ^ row_swz((wave * LOADS + c) * 8 + lane / 8)) * 16;
  }
  // row `i` of the tile lies at (i * ld) bytes, for i < valid; kbytes of k
  __device__ __forceinline__ void init(int valid, uint32_t ld, int kbytes, int wave, int lane) {
#pragma unroll
    for (int c = 0; c < 2; ++c) left[c] = kbytes - slot(c, wave, lane);
#pragma unroll
    for (int c = 0; c < LOADS; ++c) {
      const int row = (wave * LOADS + c) * 8 + lane / 8;
      off[c] = row < valid ? row * ld + slot(c, wave, lane) : OUT_OF_RANGE;
    }
  }
  // Slots past the last k are out of range.  (A step past the last one, which
  // the pipeline asks for, has no k in range; its scalar offset is 0, as the
  // range check may subtract that.)
  __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t r, int c, int kt, int kbytes, uint8_t* st, int wave) const {
    const int k0 = kt * KB;
    load_lds16(r, st + (wave * LOADS + c) * 1024, k0 < left[c & 1] ? off[c] : OUT_OF_RANGE, k0 < kbytes ? (uint32_t)k0 : 0u);
  }
};

// Chunk permutation of a k row of `COLS` 16-bit columns (see the file comment).
template <int COLS>
__device__ __forceinline__ int chunk_swz(int k) {
  return COLS >= 128 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
}

// The same for a tile of 64 k rows of C columns, 16 bits each.
template <int C, int NW>
struct ColumnLoads {
  static constexpr int RB = C * 2, RPL = 1024 / RB;
  static constexpr int LOADS = C / 8 / NW;
  static_assert(LOADS * 8 * NW == C, "load split");
  uint32_t off[LOADS];
  // column i < valid of k row j lies at j * ld + 2 i bytes
  __device__ __forceinline__ void init(int valid, uint32_t ld, int wave, int lane) {
#pragma unroll
    for (int c = 0; c < LOADS; ++c) {
      const int k = (wave * LOADS + c) * RPL + lane * 16 / RB;
      const int at = lane * 16 % RB;
      const int col = ((at / 32) ^ chunk_swz<C>(k)) * 16 + (at % 32) / 2;
      off[c] = col < valid ? k * ld + col * 2 : OUT_OF_RANGE;
    }
  }
  // `left`: k rows from this step on (those past the last are out of range)
  __device__ __forceinline__ void issue(const uint8_t* base, uint32_t ld, int left, int c, uint8_t* st, int wave) const {
    // (a scalar: the median of three is a vector instruction, and descriptors made of it are loaded lane by lane)
    const int rows = __builtin_amdgcn_readfirstlane(max(min(left, 64), 0));
    load_lds16(make_rsrc(base, (uint32_t)rows * ld), st + (wave * LOADS + c) * 1024, off[c], 0);
  }
};

// An operand for the main loop: N rows of the tile (output rows or columns),
// in one or two parts along k.  begin() is called once per step, then issue()
// for each of the LOADS loads.
template <int N, int NW>
struct RowOperand {
  static constexpr int LOADS = RowLoads<N, NW>::LOADS;
  RowLoads<N, NW> l;
  const uint8_t *p0, *p1;
  int64_t bytes;
  int kbytes, steps0, first;
  // rows from `part0` (and, from step `steps0` on, `part1`), `valid` of them;
  // the main loop's step 0 is step `first_`
  __device__ __forceinline__ void init(const void* part0, const void* part1, int64_t valid, int64_t ld_bytes, int kbytes_,
                                       int steps0_, int wave, int lane, int first_ = 0) {
    const int v = valid < N ? (int)valid : N;
    l.init(v, (uint32_t)ld_bytes, kbytes_, wave, lane);
    p0 = (const uint8_t*)part0; p1 = (const uint8_t*)part1;
    bytes = v * ld_bytes;
    kbytes = kbytes_; steps0 = steps0_; first = first_;
  }
  __device__ __forceinline__ void issue(int step, int c, uint8_t* st, int wave) const {
    const int kt = step + first;
    const bool second = kt >= steps0;
    l.issue(make_rsrc(second ? p1 : p0, bytes), c, second ? kt - steps0 : kt, kbytes, st, wave);
  }
};

template <int N, int NW>
struct ColumnOperand {
  static constexpr int LOADS = ColumnLoads<N, NW>::LOADS;
  ColumnLoads<N, NW> l;
  const uint8_t *p0, *p1;
  int k, steps0, first;
  uint32_t ld;
  __device__ __forceinline__ void init(const void* part0, const void* part1, int64_t valid, int64_t ld_bytes, int64_t k_,
                                       int steps0_, int wave, int lane, int first_ = 0) {
    ld = (uint32_t)ld_bytes;
    l.init(valid < N ? (int)valid : N, ld, wave, lane);
    p0 = (const uint8_t*)part0; p1 = (const uint8_t*)part1;
    k = (int)k_; steps0 = steps0_; first = first_;
  }
  __device__ __forceinline__ void issue(int step, int c, uint8_t* st, int wave) const {
    const int kt = step + first;
    const bool second = kt >= steps0;
    const int k0 = (second ? kt - steps0 : kt) * 64;
    l.issue((second ? p1 : p0) + (int64_t)k0 * ld, ld, k - k0, c, st, wave);
  }
};

// Rows of two matrices side by side: of every WC rows of the tile (one wave's
// columns of the output) the first half comes from p0, the second from p1.
template <int N, int NW, int WC>
struct PairOperand {
  static constexpr int LOADS = RowLoads<N, NW>::LOADS;
  RowLoads<N, NW> l;
  const uint8_t *p0, *p1;
  int64_t bytes;
  int kbytes;
  __device__ __forceinline__ void init(const void* part0, const void* part1, int64_t valid, int64_t ld_bytes, int kbytes_,
                                       int wave, int lane) {
    l.init(N, 0, kbytes_, wave, lane);
#pragma unroll
    for (int c = 0; c < LOADS; ++c) {
      const int row = (wave * LOADS + c) * 8 + lane / 8;
      const int src = row / WC * (WC / 2) + row % (WC / 2);
      l.off[c] = src < valid ? src * (uint32_t)ld_bytes + l.slot(c, wave, lane) : OUT_OF_RANGE;
    }
    p0 = (const uint8_t*)part0; p1 = (const uint8_t*)part1;
    bytes = (valid < N / 2 ? valid : N / 2) * ld_bytes;
    kbytes = kbytes_;
  }
  __device__ __forceinline__ void issue(int kt, int c, uint8_t* st, int wave) const {
    const bool second = ((wave * LOADS + c) * 8 / (WC / 2)) & 1;
    l.issue(make_rsrc(second ? p1 : p0, bytes), c, kt, kbytes, st, wave);
  }
};

// Fragment reads: 16 rows (or columns) of a tile for one MFMA.
template <typename T>
struct Frag {
  typedef typename Mfma<T>::frag type;
  static constexpr int KK = 2;                // MFMA k-steps per step
  static __device__ __forceinline__ f32x4 run(type a, type b, f32x4 c) { return Mfma<T>::run16(a, b, c); }
};
template <>
struct Frag<e4m3> {
  typedef i32x8 type;
  static constexpr int KK = 1;
  // one 16x16x128 MFMA, unscaled (scale operands 0)
  static __device__ __forceinline__ f32x4 run(type a, type b, f32x4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
  }
};

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) i16x4* lds_i16x4_t;

// The transposing LDS read.  The restrict parameter gives it an alias scope:
// without one the compiler takes it to depend on every load into LDS in flight
// and waits for all of them before each read (the weights' gradients of 8192 x
// 4096 x 2 11008 2.9 ms, with it 1.15); what it does depend on, the main loops
// wait for themselves.
__device__ __forceinline__ i16x4 read_transposed(lds_i16x4_t __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
}

template <typename T, int N, OperandOrder ORDER>
struct FragReader {
  typedef typename Frag<T>::type frag;
  uint32_t base;
  // fragments of the rows row0 + 16 i (row0 a multiple of 16)
  __device__ __forceinline__ void init(int row0, int lane) {
    const int l16 = lane & 15, l4 = lane >> 4;
    if (ORDER == ROWS) {
      base = (row0 + l16) * KB + ((l4 ^ (l16 >> 1)) * 16);
    } else {
      const int k = l4 * 8 + (l16 >> 2);
      base = k * (N * 2) + (((row0 / 16) ^ chunk_swz<N>(k)) * 32) + (l16 & 3) * 8;
    }
  }
  __device__ __forceinline__ frag read(const uint8_t* st, int kk, int i) const {
    if constexpr (ORDER == ROWS) {
      if constexpr (sizeof(T) == 1) {
        // 32 of a row's 128 k's: the slots l4 and 4 + l4, of both operands alike
        const u32x4 a = *reinterpret_cast<const u32x4*>(st + base + i * 16 * KB);
        const u32x4 b = *reinterpret_cast<const u32x4*>(st + (base ^ 64) + i * 16 * KB);
        return frag{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
      } else {
        return *reinterpret_cast<const frag*>(st + (base ^ (64 * kk)) + i * 16 * KB);
      }
    } else {
      const uint8_t* p = st + (base ^ (32 * i)) + kk * 32 * N * 2;
      const i16x4 a = read_transposed((lds_i16x4_t)p);
      const i16x4 b = read_transposed((lds_i16x4_t)(p + 4 * N * 2));
      const i16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(frag, v);
    }
  }
};

// The tile's shape: BM x BN in WMW x WNW waves.  NS: stages of both operands
// in a ring, or 0 for the deep pipeline (two stages of A, three of B).
template <int BM_, int BN_, int WMW_, int WNW_, int NS_>
struct TileShape {
  static constexpr int BM = BM_, BN = BN_, WMW = WMW_, WNW = WNW_, NS = NS_;
  static constexpr int NW = WMW * WNW, WR = BM / WMW, WC = BN / WNW, MI = WR / 16, NJ = WC / 16;
  static constexpr int A_BYTES = BM * KB, B_BYTES = BN * KB, STAGE = A_BYTES + B_BYTES;
  static constexpr int LDS = NS ? NS * STAGE : 2 * A_BYTES + 3 * B_BYTES;
};

// The tiles that launchers choose from (tile_rules.h), in FfnTile's order.
typedef TileShape<256, 256, 2, 4, 0> Tile256x256;
typedef TileShape<128, 256, 2, 4, 0> Tile128x256;
typedef TileShape<128, 128, 2, 2, 0> Tile128x128;
typedef TileShape<64, 128, 2, 2, 3> Tile64x128;
typedef TileShape<64, 64, 2, 2, 4> Tile64x64;

// run(shape) of the chosen tile.
template <typename F>
hipError_t with_tile(FfnTile t, F&& run) {
  switch (t) {
    case FFN_256x256: return run(Tile256x256());
    case FFN_128x256: return run(Tile128x256());
    case FFN_128x128: return run(Tile128x128());
    case FFN_64x128: return run(Tile64x128());
    default: return run(Tile64x64());
  }
}

// acc += the tile's products over `steps` steps.  Fragments: the B operand's
// is the MFMA's first, so that a lane ends with four consecutive columns of
// one row: acc[i][j][e] is row wm WR + 16 i + lane % 16, column
// wn WC + 16 j + 4 (lane / 16) + e.
template <typename S, typename T, OperandOrder AO, OperandOrder BO, typename AOp, typename BOp, typename F>
__device__ __forceinline__ void tile_products_ring(const AOp& a, const BOp& b, int steps, uint8_t* smem, int wave, int lane,
                                                   f32x4 (&acc)[S::MI][S::NJ], F&& meanwhile) {
  constexpr int LPS = AOp::LOADS + BOp::LOADS, KK = Frag<T>::KK;
  FragReader<T, S::BM, AO> ra;
  FragReader<T, S::BN, BO> rb;
  ra.init(wave / S::WNW * S::WR, lane);
  rb.init(wave % S::WNW * S::WC, lane);
  auto issue = [&](int kt, int s) {
    uint8_t* st = smem + s * S::STAGE;
#pragma unroll
    for (int c = 0; c < AOp::LOADS; ++c) a.issue(kt, c, st, wave);
#pragma unroll
    for (int c = 0; c < BOp::LOADS; ++c) b.issue(kt, c, st + S::A_BYTES, wave);
  };
#pragma unroll
  for (int s = 0; s < S::NS - 1; ++s) issue(s, s);
  meanwhile();
  int cur = 0, fill = S::NS - 1;
  for (int kt = 0; kt < steps; ++kt) {
    // step kt has landed (the NS - 2 steps after it may be in flight), and
    // every wave has read step kt - 1, whose stage step kt + NS - 1 takes
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((S::NS - 2) * LPS));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    issue(kt + S::NS - 1, fill);
    const uint8_t* st = smem + cur * S::STAGE;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      typename Frag<T>::type fa[S::MI], fb[S::NJ];
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) fb[j] = rb.read(st + S::A_BYTES, kk, j);
#pragma unroll
      for (int i = 0; i < S::MI; ++i) fa[i] = ra.read(st, kk, i);
#pragma unroll
      for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) acc[i][j] = Frag<T>::run(fb[j], fa[i], acc[i][j]);
    }
    cur = cur + 1 == S::NS ? 0 : cur + 1;
    fill = fill + 1 == S::NS ? 0 : fill + 1;
  }
  // the loads that ran ahead still write to LDS: let them finish
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
}

// The same with the deep pipeline, for tiles large enough to be bound by their
// MFMAs.  A step is KK MI panels (a 16-row block of A at one MFMA k-step) of NJ
// MFMAs.  A's fragments are read AHEAD panels ahead and B's a k-step ahead, so
// that by panel MEET every wave has read all of step kt, and from there on
// reads step kt + 1.  At the barrier there step kt + 1 has landed, and A of
// step kt + 2 goes to the stage of A freed; B has three stages, so that of step
// kt + 2 goes out at the start of step kt already.  The loads of a step are
// spread over its panels.
template <typename S, typename T, OperandOrder AO, OperandOrder BO, typename AOp, typename BOp, typename F>
__device__ __forceinline__ void tile_products_deep(const AOp& a, const BOp& b, int steps, uint8_t* smem, int wave, int lane,
                                                   f32x4 (&acc)[S::MI][S::NJ], F&& meanwhile) {
  typedef typename Frag<T>::type frag;
  constexpr int MI = S::MI, NJ = S::NJ, KK = Frag<T>::KK, PANELS = KK * MI;
  constexpr int AHEAD = KK == 1 ? (MI == 8 ? 3 : 2) : MI == 8 ? 5 : 4, RING = KK == 1 ? 4 : 8, MEET = PANELS - AHEAD;
  static_assert(PANELS % RING == 0 && RING > AHEAD, "fragment registers");
  // LDS instructions of one fragment of A and of B
  constexpr int RA = AO == COLUMNS || sizeof(T) == 1 ? 2 : 1, RB = BO == COLUMNS || sizeof(T) == 1 ? 2 : 1;
  constexpr int B1 = MI == 8 ? 3 : 0;         // KK = 2: the panel from which B of the second k-step is read, over four
  static_assert(KK == 1 || (B1 + 4 <= MEET && MEET + 4 <= PANELS), "step read before the barrier");
  static_assert(AOp::LOADS <= 2 * AHEAD && BOp::LOADS <= 2 * MEET, "loads of a step");
  FragReader<T, S::BM, AO> ra;
  FragReader<T, S::BN, BO> rb;
  ra.init(wave / S::WNW * S::WR, lane);
  rb.init(wave % S::WNW * S::WC, lane);
  uint8_t* const b_ring = smem + 2 * S::A_BYTES;
  frag fx[RING], fw[2][NJ];
  int bs = 0;                                 // the stage of B of step kt
  // PARITY: of the step, where fw holds one step's B and the next's (KK = 1)
  auto step = [&](int kt, auto parity) {
    constexpr int P = KK == 1 ? decltype(parity)::value : 0;
    uint8_t* a_here = smem + (kt & 1) * S::A_BYTES;
    const uint8_t* a_next = smem + ((kt & 1) ^ 1) * S::A_BYTES;
    const uint8_t* b_here = b_ring + bs * S::B_BYTES;
    bs = bs + 1 == 3 ? 0 : bs + 1;
    const uint8_t* b_next = b_ring + bs * S::B_BYTES;
    uint8_t* b_free = b_ring + (bs + 1 == 3 ? 0 : bs + 1) * S::B_BYTES;
#pragma unroll
    for (int m = 0; m < PANELS; ++m) {
      if (m == MEET) {
        // A and B of step kt + 1 have landed; B of step kt + 2 may be in flight
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(BOp::LOADS));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
      const int kk = m / MI, i = m % MI, n = m + AHEAD;
      fx[n % RING] = n < PANELS ? ra.read(a_here, n / MI, n % MI) : ra.read(a_next, (n - PANELS) / MI, (n - PANELS) % MI);
      // B of the second k-step, or of step kt + 1, spread over the panels from b0 on
      constexpr int SPREAD = KK == 1 ? AHEAD : 4;
      const bool rb1 = KK == 2 && m >= B1 && m < B1 + SPREAD, rb0 = m >= MEET && m < MEET + SPREAD;
      const int nb = rb1 ? m - B1 : m - MEET, j0 = nb * NJ / SPREAD, j1 = (nb + 1) * NJ / SPREAD;
#pragma unroll
      for (int j = j0; j < j1; ++j) {
        if (rb1) fw[1][j] = rb.read(b_here, 1, j);
        if (rb0) fw[KK == 1 ? P ^ 1 : 0][j] = rb.read(b_next, 0, j);
      }
      int loads = 0;
#pragma unroll
      for (int c = 0; c < BOp::LOADS; ++c)
        if (m < MEET && (BOp::LOADS <= MEET ? c : c * MEET / BOp::LOADS) == m) {
          b.issue(kt + 2, c, b_free, wave);
          ++loads;
        }
#pragma unroll
      for (int c = 0; c < AOp::LOADS; ++c)
        if (m >= MEET && c * AHEAD / AOp::LOADS == m - MEET) {
          a.issue(kt + 2, c, a_here, wave);
          ++loads;
        }
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = Frag<T>::run(fw[KK == 1 ? P : kk][j], fx[m % RING], acc[i][j]);
      // the panel's MFMAs around its LDS reads and loads
      __builtin_amdgcn_sched_group_barrier(0x008, NJ / 2, 0);
      const int reads = RA + (rb1 || rb0 ? (j1 - j0) * RB : 0);
      if (reads == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      else if (reads == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      else if (reads == 3) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
      else if (reads == 4) __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
      else __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
      if (loads == 1) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      else if (loads == 2) __builtin_amdgcn_sched_group_barrier(0x020, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, NJ - NJ / 2, 0);
    }
  };
#pragma unroll
  for (int c = 0; c < AOp::LOADS; ++c) a.issue(0, c, smem, wave);
#pragma unroll
  for (int c = 0; c < BOp::LOADS; ++c) b.issue(0, c, b_ring, wave);
#pragma unroll
  for (int c = 0; c < BOp::LOADS; ++c) b.issue(1, c, b_ring + S::B_BYTES, wave);
#pragma unroll
  for (int c = 0; c < AOp::LOADS; ++c) a.issue(1, c, smem + S::A_BYTES, wave);
  meanwhile();
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(AOp::LOADS + BOp::LOADS));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int j = 0; j < NJ; ++j) fw[0][j] = rb.read(b_ring, 0, j);
#pragma unroll
  for (int m = 0; m < AHEAD; ++m) fx[m] = ra.read(smem, m / MI, m % MI);
  if constexpr (KK == 1) {
    int kt = 0;
    for (; kt + 1 < steps; kt += 2) {
      step(kt, std::integral_constant<int, 0>());
      step(kt + 1, std::integral_constant<int, 1>());
    }
    if (kt < steps) step(kt, std::integral_constant<int, 0>());
  } else {
    for (int kt = 0; kt < steps; ++kt) step(kt, std::integral_constant<int, 0>());
  }
  // the loads that ran ahead still write to LDS: let them finish
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
}

// meanwhile() runs once while the first steps' loads are in flight (it may use
// acc, and load into registers).
struct Nothing {
  __device__ __forceinline__ void operator()() const {}
};
template <typename S, typename T, OperandOrder AO, OperandOrder BO, typename AOp, typename BOp, typename F = Nothing>
__device__ __forceinline__ void tile_products(const AOp& a, const BOp& b, int steps, uint8_t* smem, int wave, int lane,
                                              f32x4 (&acc)[S::MI][S::NJ], F&& meanwhile = F()) {
  if constexpr (S::NS == 0) tile_products_deep<S, T, AO, BO>(a, b, steps, smem, wave, lane, acc, meanwhile);
  else tile_products_ring<S, T, AO, BO>(a, b, steps, smem, wave, lane, acc, meanwhile);
}

// Tile (tm, tn) of workgroup wg among tiles_m x tiles_n: each XCD (wg % 8)
// walks a contiguous range, `group` tile rows at a time, so that the tiles it
// runs at once share operand panels in its L2.
__device__ __forceinline__ void tile_of(int wg, int tiles_m, int tiles_n, int group, int* tm, int* tn) {
  const int total = tiles_m * tiles_n, xcd = wg & 7, slot = wg >> 3;
  const int per = total >> 3, rem = total & 7;
  const int t = xcd * per + min(xcd, rem) + slot;
  const int g = t / (group * tiles_n), first = g * group;
  const int size = min(tiles_m - first, group);
  const int in = t - g * group * tiles_n;
  // (scalars: the buffer descriptors made from them must be)
  *tm = __builtin_amdgcn_readfirstlane(first + in % size);
  *tn = __builtin_amdgcn_readfirstlane(in / size);
}

// Up to 32 columns of one row (NB 16-column blocks of a wave, a lane holding
// columns 4 l4 .. + 3 of each) as 16-bit values; blocks whose 8 columns lie
// past `cols` are not written (cols a multiple of 8).
template <typename CT, int NB>
__device__ __forceinline__ void store_row(CT* row, int col0, int cols, const float (&v)[NB][4], int l4, bool valid) {
  typedef CT c4 __attribute__((ext_vector_type(4)));
  c4 o[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = from_f32<CT>(v[j][e]);
  if constexpr (NB % 2 == 0) {
#pragma unroll
    for (int j = 0; j < NB; j += 2)
      store_block_pair<CT>(row + col0 + 16 * j, o[j], o[j + 1], l4,
                           valid && col0 + 16 * j + 16 * (l4 & 1) + 8 * (l4 >> 1) < cols);
  } else {
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (valid && col0 + 16 * j + 4 * l4 < cols) *reinterpret_cast<c4*>(row + col0 + 16 * j + 4 * l4) = o[j];
  }
}

}  // namespace xema
