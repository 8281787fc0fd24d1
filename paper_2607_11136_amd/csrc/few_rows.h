// Products of few rows with a wide matrix (the next tokens of a few requests):
// bound by reading the weights once.  A workgroup of WAVES waves takes NB
// blocks of 16 weight rows and up to 16 MT rows of x, its waves interleaved
// 128-byte pieces of k, so that together they read 1 or 2 KiB of each weight row
// at a time, straight into registers (no LDS on the way: every weight is used by
// one wave alone).  UNROLL pieces are in flight per wave.  The waves' sums
// meet in LDS, added in wave order.  One row of 2 x 16384 x 4096 16-bit weights: 46 us
// (5.8 TB/s); 16 rows of 2 x 4096 x 4096: 17 us, of which the weights take 13.  Every
// workgroup reads all of x, which sets the limit on rows.
#pragma once

#include "mma_tile.h"

namespace xema {

template <int MT, int NB, int WAVES_>
struct FewRows {
  static constexpr int WAVES = WAVES_;
  static constexpr int ROWS = 16 * MT, COLS = 16 * NB, ROW = COLS + 4;     // (padded against bank conflicts)
  static constexpr int FLOATS = WAVES * ROWS * ROW;
};

// One 16-row operand piece: the 32 bytes of a lane, zero past the last k.
template <typename T>
__device__ __forceinline__ void load_piece(const uint8_t* row, int at, int kbytes, u32x4 (&v)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    v[h] = u32x4{0, 0, 0, 0};
    if (at + 64 * h < kbytes) v[h] = *reinterpret_cast<const u32x4*>(row + at + 64 * h);
  }
}

// The waves' sums over k of x row m and weight row n at
// red[(wave * 16 MT + m) * ROW + n], for the weight rows w[b] (each lane's own
// row lane % 16 of block b) and the rows x[i] of x (rows past the last may
// repeat one).  Ends with a barrier.
template <typename T, int MT, int NB, int WAVES, int UNROLL>
__device__ __forceinline__ void few_rows_products(const uint8_t* const (&x)[MT], const uint8_t* const (&w)[NB], int kbytes, float* red) {
  typedef FewRows<MT, NB, WAVES> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, l4 = lane >> 4;
  f32x4 acc[MT][NB];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = wave * KB; k0 < kbytes; k0 += WAVES * KB * UNROLL) {
    u32x4 vw[UNROLL][NB][2], vx[UNROLL][MT][2];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int at = k0 + u * WAVES * KB + l4 * 16;
#pragma unroll
      for (int b = 0; b < NB; ++b) load_piece<T>(w[b], at, kbytes, vw[u][b]);
#pragma unroll
      for (int i = 0; i < MT; ++i) load_piece<T>(x[i], at, kbytes, vx[u][i]);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          typedef typename Frag<T>::type frag;
          if constexpr (sizeof(T) == 1) {
            acc[i][b] = Frag<T>::run(__builtin_bit_cast(frag, vw[u][b]), __builtin_bit_cast(frag, vx[u][i]), acc[i][b]);
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              acc[i][b] = Frag<T>::run(__builtin_bit_cast(frag, vw[u][b][h]), __builtin_bit_cast(frag, vx[u][i][h]), acc[i][b]);
          }
        }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b)
      *reinterpret_cast<f32x4*>(red + (wave * 16 * MT + 16 * i + l16) * S::ROW + 16 * b + 4 * l4) = acc[i][b];
  __syncthreads();
}

// Row m, columns n .. n + 3 of the product, the waves' sums in wave order.
template <typename S>
__device__ __forceinline__ f32x4 few_rows_sum4(const float* red, int m, int n) {
  f32x4 s = *reinterpret_cast<const f32x4*>(red + m * S::ROW + n);
#pragma unroll
  for (int v = 1; v < S::WAVES; ++v) s += *reinterpret_cast<const f32x4*>(red + (v * S::ROWS + m) * S::ROW + n);
  return s;
}
template <typename S>
__device__ __forceinline__ float few_rows_sum(const float* red, int m, int n) {
  float s = red[m * S::ROW + n];
#pragma unroll
  for (int v = 1; v < S::WAVES; ++v) s += red[(v * S::ROWS + m) * S::ROW + n];
  return s;
}

}  // namespace xema
