// What the cross-attention kernels share: LDS tiles of rows that are read both
// along a row (an MFMA operand whose k are the row's elements) and across rows
// (an operand whose k are the rows, through the transposing LDS read).
//
// MFMAs are 32x32x16.  Products are formed transposed, so that a lane holds one
// column (a query in the forward pass and dq, a state in dk and dv) and the
// scores of that column feed the next product from their registers: result
// register r of a lane is row 8 (r / 4) + 4 (lane / 32) + r % 4, and an operand
// whose k is a tile's row gives k = 8 (lane / 32) + i the row 16 u + 8 (i / 4) +
// 4 (lane / 32) + i % 4 of its 16-row step u, which are the rows of registers
// 8 u + i.
//
// LDS rows are 128 bytes (head dims to 64) or 256, in 16-byte slots, slot j of
// row r at j ^ swz(r): along a row 16 lanes meet 16 rows at one slot and across
// rows 32 lanes meet four rows at four slots, both in distinct banks.
#pragma once

#include "device_common.h"
#include "mma.h"
#include "mma_tile.h"

namespace xema {

namespace {

constexpr float LOG2E_F = 1.4426950408889634f;

template <int HDP>
struct Rows {
  static constexpr int RB = HDP <= 64 ? 128 : 256;       // bytes of a row
  static constexpr int KK = HDP / 16, ND = HDP / 32;     // MFMA steps along a row, 32-column blocks
  static __device__ __forceinline__ int swz(int r) {
    return RB == 128 ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
  }
};

// 4 bytes per lane from buffer offset voff straight into LDS (256 bytes at dst).
__device__ __forceinline__ void load_lds4(__amdgpu_buffer_rsrc_t r, uint8_t* dst, uint32_t voff) {
#if __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)dst, 4, voff, 0, 0, 0);
#endif
}

// The loads of a tile of N rows into LDS, by NW waves: 1 KiB each.
template <int HDP, int N, int NW>
struct TileLoads {
  static constexpr int RB = Rows<HDP>::RB, RPL = 1024 / RB, LOADS = N / RPL / NW;
  static_assert(LOADS * RPL * NW == N, "load split");
  uint32_t off[LOADS];
  // row i of the tile lies i * ld_bytes from its first; head_dim elements of it are there, the rest are zeros
  __device__ __forceinline__ void init(uint32_t ld_bytes, int head_dim, int wave, int lane) {
#pragma unroll
    for (int c = 0; c < LOADS; ++c) {
      const int row = (wave * LOADS + c) * RPL + lane / (RB / 16);
      const int slot = (lane % (RB / 16)) ^ Rows<HDP>::swz(row);
      off[c] = slot * 8 < head_dim ? row * ld_bytes + slot * 16 : OUT_OF_RANGE;
    }
  }
  // `rows` of them are there (the buffer's end), from `base` on
  __device__ __forceinline__ void issue(const uint8_t* base, uint32_t ld_bytes, int rows, uint8_t* st, int wave) const {
    const int n = __builtin_amdgcn_readfirstlane(max(min(rows, N), 0));
    const __amdgpu_buffer_rsrc_t r = make_rsrc(base, (int64_t)n * ld_bytes);
#pragma unroll
    for (int c = 0; c < LOADS; ++c) load_lds16(r, st + (wave * LOADS + c) * 1024, off[c], 0);
  }
};

// Keeps the compiler from holding every address that it forms from x: they are formed again where they are used.
template <typename I>
__device__ __forceinline__ void forget(I& x) { asm volatile("" : "+v"(x)); }

// The lane, formed anew: no register holds it until here.
__device__ __forceinline__ int lane_again() {
  uint32_t all = ~0u;
  asm volatile("" : "+s"(all));
  return (int)__builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0));
}

// The same loads with rows past the last (rows >= 1) repeating it.  In rows of
// 256 bytes their offsets are formed at each tile: beside the sums of wide heads,
// offsets kept over the loop spill.
template <int HDP, int N, int NW>
struct RepeatedLoads {
  static constexpr int RB = Rows<HDP>::RB, RPL = 1024 / RB, LOADS = N / RPL / NW;
  static_assert(LOADS * RPL * NW == N && LOADS == (RB == 128 ? 2 : 4), "a load's rows move the swizzle by a constant");
  static __device__ __forceinline__ void issue(const uint8_t* base, uint32_t ld_bytes, int head_dim, int rows, uint8_t* st, int wave) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(base, (int64_t)min(rows, N) * ld_bytes);
    const int lane = RB == 128 ? (int)(threadIdx.x & 63) : lane_again();
    const int row0 = wave * LOADS * RPL + lane / (RB / 16), slot0 = (lane % (RB / 16)) ^ Rows<HDP>::swz(lane / (RB / 16));
    uint32_t off[LOADS];
    if (rows >= N) {
#pragma unroll
      for (int c = 0; c < LOADS; ++c) off[c] = row0 * ld_bytes + c * RPL * ld_bytes;
    } else {
#pragma unroll
      for (int c = 0; c < LOADS; ++c) off[c] = min(row0 + c * RPL, rows - 1) * ld_bytes;
    }
#pragma unroll
    for (int c = 0; c < LOADS; ++c) {
      const int slot = slot0 ^ (RB == 128 ? c << 1 : c);
      load_lds16(r, st + (wave * LOADS + c) * 1024, slot * 8 < head_dim ? off[c] + slot * 16 : OUT_OF_RANGE, 0);
    }
  }
};

// Fragments along rows: rows row0 + lane % 32, elements 16 kk + 8 (lane / 32) + 0..7.
template <typename T, int HDP>
struct AlongRows {
  typedef typename Mfma<T>::frag frag;
  uint32_t base;
  __device__ __forceinline__ void init(int lane) {
    // (the swizzle of a row is that of the rows 32 from it)
    base = (lane & 31) * Rows<HDP>::RB + (((lane >> 5) ^ Rows<HDP>::swz(lane & 31)) << 4);
  }
  // row0 a multiple of 32
  __device__ __forceinline__ frag read(const uint8_t* st, int row0, int kk) const {
    return *reinterpret_cast<const frag*>(st + row0 * Rows<HDP>::RB + (base ^ (kk << 5)));
  }
};

// Fragments across rows: the rows 16 u + ... of a lane's k (see above), columns 32 d + lane % 32.
template <typename T, int HDP>
struct AcrossRows {
  typedef typename Mfma<T>::frag frag;
  uint32_t base;
  __device__ __forceinline__ void init(int lane) {
    const int row = 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int slot = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1);
    base = row * Rows<HDP>::RB + (slot ^ Rows<HDP>::swz(row)) * 16 + (lane & 1) * 8;
  }
  // row0 a multiple of 16
  __device__ __forceinline__ frag read(const uint8_t* st, int row0, int d) const {
    constexpr int RB = Rows<HDP>::RB;
    const uint8_t* p = st + row0 * RB;
    const i16x4 a = read_transposed((lds_i16x4_t)(p + (base ^ (d << 6))));
    // (eight rows on, bit 3 of the row moves slots by two)
    const i16x4 b = read_transposed((lds_i16x4_t)(p + 8 * RB + (base ^ (d << 6) ^ 32)));
    const i16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(frag, v);
  }
};

// A lane's column of a matrix [columns, elements] as an operand: KK fragments of
// the row at p, elements past head_dim zero.
template <typename T, int HDP>
__device__ __forceinline__ void load_column(const T* p, int head_dim, int hi, typename Mfma<T>::frag (&f)[Rows<HDP>::KK]) {
  typedef typename Mfma<T>::frag frag;
#pragma unroll
  for (int kk = 0; kk < Rows<HDP>::KK; ++kk) {
    const int e = kk * 16 + hi * 8;
    f[kk] = frag{};
    if (e < head_dim) f[kk] = *reinterpret_cast<const frag*>(p + e);
  }
}

// 8 registers of a result as the operand of the next product: P and dS are rounded
// here, to the 16 bits of the other operand (the MFMA takes no wider one; a second
// product with what the rounding leaves would double their cost).
template <typename T>
__device__ __forceinline__ typename Mfma<T>::frag pack8(const f32x16& s, int u) {
  typename Mfma<T>::frag f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (T)s[8 * u + e];
  return f;
}

__device__ __forceinline__ float pair_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float pair_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Elements 16 g + 8 (lane / 32) ... + 7 of a lane's column of a transposed result's
// block of 32, times f: the halves of the wave exchange quarters of each 16.
template <typename T>
__device__ __forceinline__ u32x4 eight_of(const f32x16& acc, int g, float f) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 a, b;          // elements 16 g + 4 (lane / 32) ... and eight further on
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    a[e] = (T)(acc[8 * g + e] * f);
    b[e] = (T)(acc[8 * g + 4 + e] * f);
  }
  const u32x2 ua = __builtin_bit_cast(u32x2, a), ub = __builtin_bit_cast(u32x2, b);
  // the low half takes both halves' a, the high half both halves' b
  const auto r0 = __builtin_amdgcn_permlane32_swap(ua[0], ub[0], false, false);
  const auto r1 = __builtin_amdgcn_permlane32_swap(ua[1], ub[1], false, false);
  return u32x4{r0[0], r1[0], r0[1], r1[1]};
}

// 32 rows of a matrix [rows, elements] through 32 RB bytes of LDS that a wave has
// to itself, so that 16 lanes (8 at 128 bytes a row) load or store a row's
// consecutive bytes: straight between memory and a lane's column each load meets
// 32 rows' lines (18432 tokens, 32 heads of 128, 64 states: 75 us, through LDS 65;
// with 512 states, where the products take longer, 205 either way).
template <int HDP>
struct WaveRows {
  static constexpr int BYTES = 32 * Rows<HDP>::RB;
  typedef TileLoads<HDP, 32, 1> Loads;
  // rows past the last (rows <= 0: all) are zeros
  static __device__ __forceinline__ void load(const void* base, uint32_t ld_bytes, int head_dim, int rows, uint8_t* at, int lane) {
    Loads l;
    l.init(ld_bytes, head_dim, 0, lane);
    l.issue((const uint8_t*)base, ld_bytes, rows, at, 0);
  }
  // a lane's column of it, once it has landed
  template <typename T>
  static __device__ __forceinline__ void read(const uint8_t* at, const AlongRows<T, HDP>& r, typename Mfma<T>::frag (&f)[Rows<HDP>::KK]) {
#pragma unroll
    for (int kk = 0; kk < Rows<HDP>::KK; ++kk) f[kk] = r.read(at, 0, kk);
  }
  // The columns of a transposed result (ND blocks of 32 elements) times f as rows
  // of 16-bit values, `rows` of them.
  template <typename T>
  static __device__ __forceinline__ void store(T* base, int64_t ld, int head_dim, int rows, const f32x16 (&acc)[Rows<HDP>::ND], float f, uint8_t* at,
                                               int lane) {
    constexpr int RB = Rows<HDP>::RB, SLOTS = RB / 16;
    const int c32 = lane & 31, hi = lane >> 5;
#pragma unroll
    for (int d = 0; d < Rows<HDP>::ND; ++d)
#pragma unroll
      for (int g = 0; g < 2; ++g)
        *reinterpret_cast<u32x4*>(at + c32 * RB + (((d * 4 + g * 2 + hi) ^ Rows<HDP>::swz(c32)) << 4)) = eight_of<T>(acc[d], g, f);
    // (the wave's own writes: LDS takes a wave's accesses in order)
    const int slot = lane % SLOTS;
#pragma unroll
    for (int c = 0; c < 32 * SLOTS / 64; ++c) {
      const int row = c * (64 / SLOTS) + lane / SLOTS;
      const u32x4 v = *reinterpret_cast<const u32x4*>(at + row * RB + ((slot ^ Rows<HDP>::swz(row)) << 4));
      if (row < rows && slot * 8 < head_dim) *reinterpret_cast<u32x4*>(base + row * ld + slot * 8) = v;
    }
  }
};

// A lane's column of a transposed result times f, as 16-bit values at `row`, 16
// bytes a lane.  `valid`: whether the column is there.
template <typename T, int ND>
__device__ __forceinline__ void store_column(T* row, int head_dim, const f32x16 (&acc)[ND], float f, int hi, bool valid) {
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const u32x4 o = eight_of<T>(acc[d], g, f);
      const int e = d * 32 + g * 16 + hi * 8;
      if (valid && e < head_dim) *reinterpret_cast<u32x4*>(row + e) = o;
    }
}
// A lane's column of a transposed result times f, as fp32 values at `row`.
// `valid`: whether the column is there.
template <int ND>
__device__ __forceinline__ void store_column_f32(float* row, int head_dim, const f32x16 (&acc)[ND], float f, int hi, bool valid) {
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int e = d * 32 + g * 8 + hi * 4;
      const f32x4 o = {acc[d][4 * g] * f, acc[d][4 * g + 1] * f, acc[d][4 * g + 2] * f, acc[d][4 * g + 3] * f};
      if (valid && e < head_dim) *reinterpret_cast<f32x4*>(row + e) = o;
    }
}

// Division by a number that the host knows, in scalar instructions: the product
// with floor(2^32 / d) is the quotient or one less (n below 2^31).
struct Divisor {
  uint32_t d, m;
  Divisor() = default;
  explicit Divisor(int64_t by) : d((uint32_t)by), m(by == 1 ? 0xffffffffu : (uint32_t)(((uint64_t)1 << 32) / (uint64_t)by)) {}
  __device__ __forceinline__ int divide(int n, int* rest) const {
    uint32_t q = __umulhi((uint32_t)n, m), r = (uint32_t)n - q * d;
    if (r >= d) {
      ++q;
      r -= d;
    }
    *rest = (int)r;
    return (int)q;
  }
};

// Workgroup wg of `total` in an order that gives each XCD (wg % 8) a contiguous
// range, so that workgroups that share operands share an L2.
__device__ __forceinline__ int xcd_order(int wg, int total) {
  const int xcd = wg & 7, per = total >> 3, rem = total & 7;
  return xcd * per + min(xcd, rem) + (wg >> 3);
}

// States of sequence b.
__device__ __forceinline__ int states_of(const int32_t* kv_lens, int b, int kv_len) {
  return kv_lens ? __builtin_amdgcn_readfirstlane(min(max(kv_lens[b], 0), kv_len)) : kv_len;
}

// Part `part` of `parts` of n tiles: [first, first + count).
__device__ __forceinline__ void part_of(int n, int part, int parts, int* first, int* count) {
  const int each = (n + parts - 1) / parts;
  *first = min(part * each, n);
  *count = min(each, n - *first);
}

}  // namespace

}  // namespace xema
