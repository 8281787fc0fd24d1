// Products of few rows with a wide matrix (the next tokens of a few requests):
// bound by reading the weights once.  A workgroup of WAVES waves takes NB
// blocks of 16 weight rows and up to 16 MT rows of x, its waves interleaved
// 128-byte pieces of k, so that together they read 1 or 2 KiB of each weight row
// at a time, straight into registers (no LDS on the way: every weight is used by
// one wave alone).  UNROLL pieces are in flight per wave.  The waves' sums
// meet in LDS, added in wave order.
#pragma once

#include "mma_tile.h"

namespace xema {

template <int MT, int NB, int WAVES_>
struct FewRows {
  static constexpr int WAVES = WAVES_;
  static constexpr int COLS = 16 * NB, ROW = COLS + 4;     // (padded against bank conflicts)
  static constexpr int FLOATS = WAVES * 16 * MT * ROW;
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

// red[m * ROW + n] (of wave 0) = sum over k of x row m and weight row n, for
// the weight rows w[b] (each lane's own row lane % 16 of block b) and the rows
// x[i] of x (rows past the last may repeat one).  Ends with a barrier.
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
  for (int at = threadIdx.x; at < 16 * MT * S::COLS; at += WAVES * 64) {
    float* p = red + at / S::COLS * S::ROW + at % S::COLS;
    float s = p[0];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) s += p[v * 16 * MT * S::ROW];
    p[0] = s;
  }
  __syncthreads();
}

}  // namespace xema
