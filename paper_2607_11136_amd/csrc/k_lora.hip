// A projection shared by requests with low-rank adapters of their own
// (xema_op_lora_linear, xema_ffn.h).
#include <utility>

#include "device_common.h"
#include "ffn.h"
#include "mma_tile.h"

namespace xema {

namespace {

typedef TileShape<256, 256, 2, 4, 0> Big;
typedef TileShape<128, 128, 2, 2, 3> Mid;
typedef TileShape<64, 64, 2, 2, 4> Small;

struct LoraParams {
  const void *x, *w; const uint16_t* bias;
  const void *a, *b; const float* scale;
  const int32_t* ids;
  void *y, *t;                 // t: [rows, 2 rank], the scaled x a^T as rounded value and remainder
  int64_t rows, ldx, ldy;
  int dim, out_dim, rank, n_adapters;
};

// t[r] = scale[i] x[r] a[i]^T, as value and remainder.  A wave per row and rank.
template <typename T>
__global__ __launch_bounds__(256) void k_lora_reduce(LoraParams p) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  const int64_t r = blockIdx.x;
  const int id = p.ids[r];
  if (id < 0 || id >= p.n_adapters) return;
  const int lane = threadIdx.x & 63;
  const T* x = (const T*)p.x + r * p.ldx;
  for (int q = threadIdx.x >> 6; q < p.rank; q += 4) {
    const T* a = (const T*)p.a + ((int64_t)id * p.rank + q) * p.dim;
    float s = 0.f;
    for (int k = lane * 8; k < p.dim; k += 512) {
      const t8 u = *reinterpret_cast<const t8*>(x + k), v = *reinterpret_cast<const t8*>(a + k);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf((float)u[e], (float)v[e], s);
    }
    s = wave_sum(s) * p.scale[id];
    if (lane == 0) {
      T* t = (T*)p.t + r * 2 * p.rank + q;
      const T hi = (T)s;
      t[0] = hi;
      t[p.rank] = (T)(s - (float)hi);
    }
  }
}

template <typename F, int... J>
__device__ __forceinline__ void each_block(F&& f, std::integer_sequence<int, J...>) {
  (f(std::integral_constant<int, J>()), ...);
}

// acc += t[r] b[i]^T for the rows of each adapter among the wave's rows, one
// adapter at a time.  Products of a row with another request's adapter are
// formed beside and dropped, never multiplied by zero: that adapter may hold
// infinities.
template <typename T, typename S>
__device__ __forceinline__ void add_adapters(const LoraParams& p, int64_t m0, int n0, int wave, int lane, const int (&id)[S::MI],
                                             f32x4 (&acc)[S::MI][S::NJ]) {
  typedef typename Frag<T>::type frag;
  const int l16 = lane & 15, l4 = lane >> 4;
  const int slots = p.rank / 4, rs = p.rank / 8;       // 16-byte slots of a row of t and of a row of b
  int todo = 0;                                        // blocks of this lane whose row's adapter is to come
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
    if (id[i] >= 0 && id[i] < p.n_adapters) todo |= 1 << i;
  for (;;) {
    const uint64_t any = __ballot(todo != 0);
    if (!any) break;
    int first = -1;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) first = first < 0 && (todo >> i & 1) ? id[i] : first;
    const int cur = __builtin_amdgcn_readlane(first, __builtin_ctzll(any));
    int hit = 0;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) hit |= (id[i] == cur) << i;
    const T* bw = (const T*)p.b + (int64_t)cur * p.out_dim * p.rank;
    auto block = [&](auto jc) {
      constexpr int j = decltype(jc)::value;
      const int n = min(n0 + 16 * j + l16, p.out_dim - 1);
      f32x4 sum[S::MI];
#pragma unroll
      for (int i = 0; i < S::MI; ++i) sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < slots; k += 4) {
        const int at = k + l4;
        frag fb{};
        if (at < slots) fb = *reinterpret_cast<const frag*>(bw + (int64_t)n * p.rank + (at < rs ? at : at - rs) * 8);
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
          frag ft{};
          // (a row past the end, or without this adapter, contributes nothing)
          if (at < slots && id[i] == cur) ft = *reinterpret_cast<const frag*>((const T*)p.t + (m0 + 16 * i + l16) * 2 * p.rank + at * 8);
          sum[i] = Frag<T>::run(fb, ft, sum[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = id[i] == cur ? acc[i][j][e] + sum[i][e] : acc[i][j][e];
    };
    each_block(block, std::make_integer_sequence<int, S::NJ>());
    todo &= ~hit;
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
  int id[S::MI];
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const int64_t m = mw + 16 * i + l16;
    id[i] = m < p.rows ? p.ids[m] : -2;
  }
  f32x4 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  tile_products<S, T, ROWS, ROWS>(a, b, (kbytes + KB - 1) / KB, smem, wave, lane, acc);
  if (p.n_adapters) add_adapters<T, S>(p, mw, nw, wave, lane, id, acc);

  float bv[S::NJ][4];
#pragma unroll
  for (int j = 0; j < S::NJ; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) bv[j][e] = p.bias ? bf16_bits_to_f32(p.bias[min(nw + 16 * j + 4 * l4 + e, p.out_dim - 1)]) : 0.f;
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const bool valid = id[i] >= -1;
    float v[S::NJ][4];
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j][e] = id[i] < p.n_adapters ? acc[i][j][e] + bv[j][e] : __builtin_nanf("");
    store_row<YT, S::NJ>((YT*)p.y + (valid ? mw + 16 * i + l16 : 0) * p.ldy, nw, p.out_dim, v, l4, valid);
  }
}

template <typename T, typename YT, typename S>
hipError_t run_project(const LoraParams& p, hipStream_t s) {
  const int64_t tiles = (p.rows + S::BM - 1) / S::BM * ((p.out_dim + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((k_lora_project<T, YT, S>), dim3((unsigned)tiles), dim3(S::NW * 64), 0, s, p);
  return hipGetLastError();
}

template <typename T, typename YT>
hipError_t lora_t(const LoraParams& p, hipStream_t s) {
  if (p.n_adapters) {
    hipLaunchKernelGGL((k_lora_reduce<T>), dim3((unsigned)p.rows), dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  auto tiles = [&](int t) { return (p.rows + t - 1) / t * ((p.out_dim + t - 1) / t); };
  if (tiles(256) >= 192) return run_project<T, YT, Big>(p, s);
  return tiles(128) >= 192 ? run_project<T, YT, Mid>(p, s) : run_project<T, YT, Small>(p, s);
}

}  // namespace

hipError_t launch_lora_linear(const xema_lora_args& a, hipStream_t s) {
  const LoraParams p{a.x, a.w, (const uint16_t*)a.bias, a.a, a.b, a.scale, a.row_adapter, a.y, a.workspace,
                     a.rows, a.ldx, a.ldy, a.dim, a.out_dim, a.rank, a.n_adapters};
  if (a.dtype == XEMA_BF16) return a.y_dtype == XEMA_BF16 ? lora_t<bf16, bf16>(p, s) : lora_t<bf16, f16>(p, s);
  return a.y_dtype == XEMA_BF16 ? lora_t<f16, bf16>(p, s) : lora_t<f16, f16>(p, s);
}

}  // namespace xema
