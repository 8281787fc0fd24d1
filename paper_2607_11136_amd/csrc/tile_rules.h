// Which tile a call takes: the launchers' rules on sizes, free of device code
// so that they can be examined (and tested) on the host alone.
#pragma once

#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

namespace xema {

constexpr int RULE_CUS = 256;

// ---------------------------------------------------------------------------
// GEMM
// ---------------------------------------------------------------------------

// Completion time of n_big full tiles, then n_small half-height tiles costing
// `half` of a full one, dealt in order to the first free of the CUs (tiles
// freed at the same time form one group).
inline double tile_makespan(int64_t n_big, int64_t n_small, double half) {
  constexpr int64_t CUS = RULE_CUS;
  const int64_t rounds = n_big / CUS, extra = n_big % CUS;
  std::vector<std::pair<double, int64_t>> free_at;  // (time, CUs)
  if (CUS - extra) free_at.push_back({(double)rounds, CUS - extra});
  if (extra) free_at.push_back({(double)rounds + 1.0, extra});
  double end = free_at.back().first;
  if (n_big == 0) end = 0.0;
  while (n_small > 0) {
    size_t i = 0;
    for (size_t j = 1; j < free_at.size(); ++j)
      if (free_at[j].first < free_at[i].first) i = j;
    const double t = free_at[i].first;
    const int64_t k = std::min(free_at[i].second, n_small);
    n_small -= k;
    end = std::max(end, t + half);
    if (free_at[i].second == k) free_at.erase(free_at.begin() + i);
    else free_at[i].second -= k;
    bool merged = false;
    for (auto& g : free_at)
      if (g.first == t + half) { g.second += k; merged = true; }
    if (!merged) free_at.push_back({t + half, k});
  }
  return end;
}

// Rows [0, split) go to 256-row tiles, the rest to 128-row tiles: the split
// with the least modelled completion time.  A half-height tile costs 0.56 of a full
// one (8192 and 20480 rows of 12288 columns in either alone: 0.54 to 0.57, with the
// gated epilogue 0.52 to 0.60; any value from 0.53 to 0.62 gives the block's sizes the
// same times).  *rounds receives that time in full tiles.
inline int64_t gemm_row_split(int64_t M, int tiles_n, double* rounds) {
  constexpr double HALF = 0.56;
  const int64_t tm = (M + 255) / 256;
  int64_t best_split = M;
  double best = tile_makespan(tm * tiles_n, 0, HALF);
  for (int64_t t1 = tm - 1; t1 >= 0 && t1 >= tm - 16; --t1) {
    const int64_t rest = (M - t1 * 256 + 127) / 128;
    const double cost = tile_makespan(t1 * tiles_n, rest * tiles_n, HALF);
    if (cost < best - 1e-9) { best = cost; best_split = t1 * 256; }
  }
  *rounds = best;
  return best_split;
}

// The tiles of k_gemm_192 and k_gemm_ring, and last that of k_gemm, with the
// microseconds one 64-wide K step of a tile takes and what a tile costs beside its
// steps when every CU holds one (its pipeline's start and the latency of its
// epilogue; the time of the stores themselves is the same for all tiles).  A CU
// fetches about 55 GB/s from beyond its L2, so the small tiles cost their operand
// bytes and only the 256-row ones their MFMAs.
enum GemmTile { G256x192, G256x128, G128x192, G128x128, G128x96, G64x128, G64x64, GEMM_MAIN };
struct GemmCost { int rows, cols; double step_us, tile_us; };
constexpr GemmCost kGemmCost[] = {{256, 192, 1.14, 3},  {256, 128, 0.86, 3}, {128, 192, 0.76, 3}, {128, 128, 0.6, 2},
                                  {128, 96, 0.45, 1.5}, {64, 128, 0.33, 1},  {64, 64, 0.23, 1},  {256, 256, 1.44, 4}};

// The tile for an M x N problem of depth K: the fewest rounds over the CUs times a
// round's time; `split` is k_gemm's.  heads_dim: 64 or 128 for the QKV epilogue,
// which needs 64 columns a wave and, at 128, two waves a row.
//
// Over 950 problems (16 to 20480 rows, N of 256 to 12288, K of 64 to 12288, the three
// epilogues) the picked tile takes 0.5% more than the fastest one in the mean and
// 7% at most; with no fixed cost for the smaller tiles it was 3.8%, and up to 39% at
// K = 256.  k_gemm alone and the picked tile, us:
//   256 x 3072 x 12288    64 x 64    118 and 47
//   512 x 3072 x 3072     64 x 128    39 and 20
//   1000 x 3072 x 12288   128 x 96   123 and 94
//   6000 x 768 x 768      128 x 192   32 and 19
//   9216 x 768 x 768      256 x 128   33 and 25
//   2048 x 12288 x 3072   256 x 192  165 and 134
//   4000 x 3072 x 3072    256 x 192   80 and 74
//   20480 x 12288 x 256   256 x 256  211 (256 x 128: 258)
// At 2048 x 3072 x 3072 and 12288 128 x 192 tiles and half-height ones are within 4%
// alone; beside the attention of the next chunk the former are 1% ahead.
struct GemmPick { int tile; int64_t split; };
inline GemmPick gemm_pick(int64_t M, int N, int K, int heads_dim) {
  GemmPick pick{GEMM_MAIN, 0};
  double rounds;
  pick.split = gemm_row_split(M, N / 256, &rounds);
  const double steps = K / 64;
  const GemmCost& full = kGemmCost[GEMM_MAIN];
  double cost = rounds * (full.step_us * steps + full.tile_us);
  for (int t = 0; t < GEMM_MAIN; ++t) {
    const GemmCost& c = kGemmCost[t];
    if (N % c.cols) continue;
    if (heads_dim && c.cols != 128 && !(heads_dim == 64 && t == G64x64)) continue;
    const int64_t tiles = ((M + c.rows - 1) / c.rows) * (N / c.cols);
    const double us = (double)((tiles + RULE_CUS - 1) / RULE_CUS) * (c.step_us * steps + c.tile_us);
    if (us < cost - 1e-9) { cost = us; pick.tile = t; }
  }
  return pick;
}

// ---------------------------------------------------------------------------
// The feed-forward sub-block's products (mma_tile.h)
// ---------------------------------------------------------------------------
enum FfnTile { FFN_256x256, FFN_128x256, FFN_128x128, FFN_64x128, FFN_64x64, FFN_TILES };
// Microseconds of a 128-byte step of k with few CUs busy and with all of them,
// and of a tile beside its steps.  The first two tiles fill a CU.  Of the others
// two share one, each hiding the other's latency: full_us is then the step of
// such a pair.
struct FfnCost { int rows, cols; double alone_us, full_us, tile_us; bool shares; };
constexpr FfnCost kFfnCost[FFN_TILES] = {{256, 256, 1.03, 1.41, 6.6, false}, {128, 256, 0.63, 0.85, 4.1, false},
                                         {128, 128, 0.52, 0.97, 4.2, true},  {64, 128, 0.35, 0.56, 3.2, true},
                                         {64, 64, 0.265, 0.41, 2.7, true}};

inline double ffn_tile_us(const FfnCost& c, int64_t m, int64_t n, int64_t steps, int64_t times = 1) {
  const int64_t tiles = (m + c.rows - 1) / c.rows * ((n + c.cols - 1) / c.cols) * times;
  const int64_t slots = c.shares ? 2 * RULE_CUS : RULE_CUS, rounds = tiles / slots, rest = tiles % slots;
  // the last round runs at the few CUs' pace while half of them idle, and pairs
  // are faster by up to 15% while few CUs have one
  const double last = rest == 0                       ? 0
                      : c.shares && rest > RULE_CUS   ? c.full_us * (0.85 + 0.15 * (rest - RULE_CUS) / RULE_CUS)
                      : c.shares || rest <= RULE_CUS / 2 ? c.alone_us
                                                         : c.alone_us + (c.full_us - c.alone_us) * (rest - RULE_CUS / 2) / (RULE_CUS / 2);
  const double ends = (double)rounds + (rest ? 1 : 0);
  return c.tile_us * (c.shares ? 0.5 + 0.5 * ends : ends) + (double)steps * (rounds * c.full_us + last);
}

// The tile for an m x n result of `steps` steps of k.  Over 304 calls (16 to 4096
// rows, widths of 512 to 11008, the five products) the picked tile takes 0.8%
// more than the fastest in the mean and 15% at most.  us, 256 x 256 tiles and
// the picked one: 48 x 2 4096 x 4096 73 and 19; 777 x 2 4096 x 4096 76 and 53;
// 1024 x 4096 x 4096 (projection) 75 and 39; 2048 x 2 11008 x 4096 271 and 271.
inline FfnTile pick_tile(int64_t m, int64_t n, int64_t steps) {
  int best = 0;
  double least = 0;
  for (int t = 0; t < FFN_TILES; ++t) {
    const double us = ffn_tile_us(kFfnCost[t], m, n, steps);
    if (t == 0 || us < least) { best = t; least = us; }
  }
  return (FfnTile)best;
}

// Rows of a product in two launches: the first `rows`, any number of 256-row blocks
// that leaves less than 48 of them, in tiles of 256 x 256, and the rest in the tile
// that finishes soonest, where the model has the two take less than one (a second
// launch costs 3 us).  Most often the rest is what lies past whole rounds of tiles.
// Every tile sums in the same order, so the values do not depend on it.  129 sizes
// (1063 to 31706 rows, 536 to 15992 columns, k of 320 to 11264), what two launches
// take off one's time: where the model gives less than 2%, -6 to 9%, 0.8% in the mean
// (so small gains are taken too); from 2 to 8%, -3 to 10%, 3.2%; past that 1 to 31%, 13%.
// us, rows x columns x k, one and two: 4608 x 4096 x 4096 149 and 129, 9216 rows 270
// and 245; 8192 x 11008 x 4096, 0.6% by the model, 570 and 571; 10793 x 4456 x 512,
// 0.8%, 64 and 68; 9854 x 15872 x 320, 0.1%, 155 and 141.
struct FfnRows { int64_t rows; FfnTile rest; };
inline FfnRows pick_rows(int64_t m, int64_t n, int64_t steps) {
  FfnRows best{0, pick_tile(m, n, steps)};
  double least = ffn_tile_us(kFfnCost[best.rest], m, n, steps);
  const int64_t whole = m / 256;
  for (int64_t k = whole; k > 0 && k > whole - 48; --k) {
    if (k * 256 == m) continue;
    const FfnTile t = pick_tile(m - k * 256, n, steps);
    const double us = ffn_tile_us(kFfnCost[FFN_256x256], k * 256, n, steps) + 3.0 + ffn_tile_us(kFfnCost[t], m - k * 256, n, steps);
    if (us < least) { best = {k * 256, t}; least = us; }
  }
  return best;
}

// A product whose k may be split: `parts` sums over consecutive steps, kept in
// fp32 and added by a launch of their own (3 us, and the sums' bytes at about 7
// TB/s there and back, for most stay in the caches).  For small results of long k
// (dx of a short batch, the weights' gradients of a narrow layer), whose tiles leave
// most CUs idle.  us whole and split: 333 x 512, 44 steps 16 and 8; 64 x 4096, 344
// steps 96 and 40; 2 1024 x 512, 469 steps 141 and 69.
struct FfnSplit { FfnTile tile; int parts; };
inline FfnSplit pick_split(int64_t m, int64_t n, int64_t steps) {
  FfnSplit best{pick_tile(m, n, steps), 1};
  double least = ffn_tile_us(kFfnCost[best.tile], m, n, steps);
  for (int64_t want = 2; want <= 16 && steps / want >= 8; want *= 2) {
    const int64_t each = (steps + want - 1) / want, parts = (steps + each - 1) / each;
    if (m * n * parts > ((int64_t)1 << 24)) break;      // (64 MiB of sums)
    for (int t = 0; t < FFN_TILES; ++t) {
      const double us = ffn_tile_us(kFfnCost[t], m, n, each, parts) + 3.0 + (double)m * n * 8 * parts / 7e6;
      if (us < least) { best = {(FfnTile)t, (int)parts}; least = us; }
    }
  }
  return best;
}

// Few rows (few_rows.h), in blocks of 16 rows and of 16 columns a workgroup; no
// blocks: tiles.  The gated feed-forward's workgroups have 16 hidden units (weights
// from HBM, us, that kernel and the best tile: 16 x 2 4096 x 4096 17 and 21, 32 rows
// 20 and 22; 16 x 2 11008 x 4096 40 and 39, 32 rows 51 and 40).
struct FewPick { int rows16, cols16; };
inline FewPick pick_gated_few(int64_t rows, int hidden) {
  if (rows <= 16) return {1, 1};
  if (rows <= 32 && hidden <= 8192) return {2, 1};
  return {0, 0};
}
// The projection with adapters: one round of workgroups (one a CU), 16, 32 or 64
// columns each, 64 also where that takes more rounds.  Past that, and past 64
// rows (32 beside 64 columns), every workgroup's reading all of x costs more
// than the tiles (us, with the reduction; columns 16, 32, 64, tiles):
//   48 x 4096 x 4096   25, 29, -, 32     16 x 4096 x 11008  35, 34, 30, 33
//   48 x 4096 x 6144   41, 30, -, 33     1 x 4096 x 16384   35, 34, 34, 38
//   48 x 4096 x 11008  59, 52, -, 34     16 x 4096 x 32768  86, 69, 62, 75
//   24 x 4096 x 8192   31, 25, -, 32     32 x 4096 x 32768  -, 83, 70, 78
inline FewPick pick_lora_few(int64_t rows, int out_dim) {
  const int rows16 = (int)((rows + 15) / 16);
  if (rows <= 64 && out_dim <= 4096) return {rows16, 1};
  if (rows <= 64 && out_dim <= 8192) return {rows16, 2};
  if (rows <= 32) return {rows16, 4};
  return {0, 0};
}

// The adapters' reduction, in blocks of 16 rows and of 16 ranks a workgroup; no
// blocks: a workgroup per row.  A row by itself reads all of its adapter's a,
// which pays while the rows are few (and then likely single tokens, each with an
// adapter of its own): rows of 4096, with a projection to 72, us, row by row and in
// blocks,
//                          one adapter   50 rows a request   drawn of 24 per row
//   4096 rows, rank 8         44, 29           45, 37              53, 128
//   1024 rows, rank 32        37, 30           39, 39              51, 139
//   256 rows, rank 128        40, 33           46, 44              93, 170
// and past the limit
//   2048 rows, rank 32        49, 30           51, 39              66, 156
//   512 rows, rank 128        52, 33           59, 45              111, 171
// The more rows share a's lines the better, while every CU
// has a workgroup (18432 x 4096 from HBM, us, 32 and 48 rows each: rank 32 71 and
// 65, rank 128 144 and 110; 5000 x 4096, rank 16 32 and 41).  Then the most ranks,
// to 64, that still give each CU a workgroup, as each reads all of its rows' x
// (1000 rows of 4096, rank 64: 21 us with all ranks in one workgroup, 10 in four;
// with 50 rows a request 39 and 19; with an adapter drawn for every row 276 and 124).
struct ReducePick { int rows16, ranks16; };
inline ReducePick pick_reduce(int64_t rows, int rank) {
  if (rows * rank <= 32768) return {0, 0};
  const int rows16 = rows > 48 * RULE_CUS ? 3 : rows > 16 * RULE_CUS ? 2 : 1;
  const int64_t blocks = (rows + 16 * rows16 - 1) / (16 * rows16);
  for (int ranks16 = 4; ranks16 > 1; ranks16 /= 2)
    if (rank > 8 * ranks16 && blocks * ((rank + 16 * ranks16 - 1) / (16 * ranks16)) >= RULE_CUS) return {rows16, ranks16};
  return {rows16, 1};
}

// ---------------------------------------------------------------------------
// Attention to an encoder's states (k_cross.hip, k_cross_bwd.hip)
// ---------------------------------------------------------------------------
// few: the kernel of single tokens, whose blocks are 32 rows (tokens of all heads
// that share a state's head); otherwise blocks of 128 of a head's queries.  us, few
// and not: 64 rows, 4 sequences of 4096 states, 8 state heads of 128, 24 and 40;
// 96 rows 49 and 40; with fewer states (1024, 512, 77) they are within 15%.
//
// parts: of the states, for calls of few workgroups, which k_cross_join adds up.
// Single tokens: one round of two workgroups a CU (us, at 512 and 1024 workgroups:
// 8 sequences of 4096 states 33 and 39, 64 of 1024 52 and 58), no part below 128
// states, and none at all where the half of the CUs has work and the states are so
// few that the join costs more (256 sequences' heads of 64, 512 states: whole 9.2,
// two parts 10.8).  Otherwise parts of 256 states or more, from 1024 states on (us,
// whole and in the parts picked: 2 x 500 tokens, 8 heads of 128, 512 states 13.4
// and 17.0; 1000 tokens, 8 heads of 64, 1024 states 18.1 and 15.3; 256 tokens, 4
// heads of 128, 4096 states 80 and 18).
constexpr int FEW_WGS = 2 * RULE_CUS;
struct CrossPick { bool few; int blocks, parts; };
// Of the states, for `wgs` workgroups of 128 queries: the forward pass, and dq.
inline int cross_parts(int64_t wgs, int kv_len) {
  if (wgs == 0 || kv_len < 1024) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>({2 * RULE_CUS / wgs, kv_len / 256, 16}));
}
inline CrossPick pick_cross(int batch, int heads, int kv_heads, int head_dim, int q_len, int kv_len) {
  const int64_t rows = (int64_t)q_len * (heads / kv_heads);
  if (rows > 64) {
    const int blocks = (q_len + 127) / 128;
    return {false, blocks, cross_parts((int64_t)batch * heads * blocks, kv_len)};
  }
  const int blocks = (int)((rows + 31) / 32);
  const int64_t wgs = (int64_t)batch * kv_heads * blocks;
  const int64_t most = wgs >= RULE_CUS / 2 && kv_len <= 768 ? 1 : ((int64_t)kv_len + 127) / 128;
  return {true, blocks, wgs ? (int)std::max<int64_t>(1, std::min<int64_t>({(FEW_WGS + wgs - 1) / wgs, most, 64})) : 1};
}

// Threads that join a row's parts: a workgroup for each of few rows (k_cross_join),
// otherwise eight columns a thread (k_cross_join_rows).  us of the call with a
// workgroup a row and with threads a row: 128 rows in 16 parts 47 and 54; 512 in 4
// either 47; 8192 in 2 21 and 14.
inline int pick_join(int64_t rows, int head_dim) { return rows <= 1024 ? 256 : head_dim <= 64 ? 8 : 16; }

// The gradient.  dq: as the forward pass (us, whole and in parts: 512 states 17.9
// and 19.5, 1024 states 19.8 and 15.6, 4096 states 100 and 21).  dk and dv: parts of
// the tokens of all heads that share a state's head, for workgroups of 128 states;
// as many as the CUs hold (two each, three at head dims to 64), of two tiles of 64
// tokens or more, their sums within 256 MiB (us of dk and dv, whole and in the parts
// picked: 4608 tokens, 32 heads of 128, 512 states 194 and 96; 2 x 577 tokens, 4
// heads of 64 for 16, 120 states 82 and 19; 4 x 1024, 12 heads of 72, 77 states 33 and 18).
//
// both: one launch, where dq leaves dk and dv a quarter of the CUs' places or more,
// for two parts of theirs if they have as many (us, in turn and in one launch: 3 x 577
// tokens, 16 heads of 72 on 4, 120 states 26.5 and 21.5; 2048 tokens, 16 heads of 128, 512
// states 63 and 51; 20 heads of 64, 256 states 38 and 32; 24 heads of 128, 512
// states, whose dk and dv would be whole, 81 and 125).
struct CrossBwdPick { int q_parts, kv_parts; bool both; };
inline CrossBwdPick pick_cross_bwd(int batch, int heads, int kv_heads, int head_dim, int q_len, int kv_len) {
  const int64_t q_wgs = (int64_t)batch * heads * ((q_len + 127) / 128);
  const int q_parts = cross_parts(q_wgs, kv_len);
  const int64_t wgs = (int64_t)batch * kv_heads * ((kv_len + 127) / 128), tiles = (int64_t)heads / kv_heads * ((q_len + 63) / 64);
  if (!wgs) return {q_parts, 1, false};
  const int64_t sums = 2 * (int64_t)batch * kv_len * kv_heads * head_dim, left = 2 * RULE_CUS - q_wgs * q_parts;
  const bool both = left >= RULE_CUS / 2 && left >= (tiles >= 4 ? 2 : 1) * wgs;
  const int64_t slots = both ? left : (head_dim <= 64 ? 3 : 2) * RULE_CUS;
  return {q_parts, (int)std::max<int64_t>(1, std::min<int64_t>({slots / wgs, tiles / 2, 32, ((int64_t)1 << 26) / sums})), both};
}

// Without dq, its pass leaves lse and D for dk and dv, of every token once and
// whatever the states: one part, no launch of both.  kv_parts, which the workspace and
// the bytes of dk and dv go by, stay as they are.
inline CrossBwdPick without_dq(const CrossBwdPick& p) { return {1, p.kv_parts, false}; }

// ---------------------------------------------------------------------------
// k_upconv.  A tile is RG R fragments of 16 corners (a corner: the four outputs
// between four source pixels) and 128 / RG channels.
// ---------------------------------------------------------------------------
enum UpconvShape { ROWS_SHAPE, COLUMNS_SHAPE, FLAT_SHAPE };
constexpr int UT = 16;                    // corners of a fragment
constexpr int UBK = 64;                   // channels per K step
constexpr int UNWAVES = 8;
constexpr int UUNITS = 4, UHALF = 7;      // units of a K step, weight panels of a unit
constexpr int UXS = 2, UWS = 3;           // LDS stages: steps of x, units of weights

struct UpconvSize { int n, h, w, ci, co, row_begin, row_count; };
struct UpconvTile { int rg, r; UpconvShape shape; double step_us, tile_us; };

// The 1 KiB loads that a stage of x holds.
constexpr int upconv_x_loads(int rg, int r, UpconvShape shape) {
  const int w_bytes = UWS * UHALF * 16 * (UNWAVES / rg) * UBK * 2;
  return shape == FLAT_SHAPE      ? (160 * 1024 - w_bytes) / UXS / 1024
         : shape == COLUMNS_SHAPE ? ((rg + 1) * (UT * r + 1) + 7) / 8
                                  : ((rg * r + 1) * (UT + 1) + 7) / 8;
}

// Rows of a frame in the row of all corners: the row past a frame's last one is
// the row before the next one's first, unless these are rows of the images.
constexpr int upconv_frame_rows(int h, int row_begin, int row_count) {
  return row_count + (row_begin == 0 && row_count == h ? 1 : 2);
}

// The tiles of the first n frames.
inline int64_t upconv_tiles(const UpconvSize& p, int64_t n, int rg, int r, UpconvShape shape) {
  const int64_t corners = UT * rg * r, frame = (int64_t)upconv_frame_rows(p.h, p.row_begin, p.row_count) * (p.w + 1);
  const int64_t pixels = shape == FLAT_SHAPE      ? (n * frame + corners - 1) / corners
                         : shape == COLUMNS_SHAPE ? n * (p.row_count / rg + 1) * (p.w / (UT * r) + 1)
                                                  : n * (p.row_count / (rg * r) + 1) * (p.w / UT + 1);
  return pixels * (p.co / (16 * UNWAVES / rg));
}

// Whether the tiles of 16 rg r corners in a row can be used: x of a step fits its
// stage, and a tile's outputs lie within 2^31 bytes.
inline bool upconv_flat_fits(const UpconvSize& p, int rg, int r) {
  const int64_t corners = UT * rg * r, frame = (int64_t)upconv_frame_rows(p.h, p.row_begin, p.row_count) * (p.w + 1);
  return corners + p.w + 2 <= 8 * upconv_x_loads(rg, r, FLAT_SHAPE) &&
         (corners / frame + 2) * 8 * p.h * p.w * p.co < ((int64_t)1 << 31);
}

// The tiles, with the microseconds of a K step of 64 channels and what a tile
// costs beside its steps, all CUs busy (8 x 240 x 360, 256 and 512 -> 256
// channels; FLAT 64 x 16 x 16, 256 -> 256).  ROWS tiles fetch least per corner but
// round a call's corner rows up to 16 or 12 and its columns to 16; COLUMNS round
// to 4 and 48, for bands of few rows; FLAT ones round nothing, but hold x of W + 2
// corners more, so they are for narrow images, and the small ones for small calls.
constexpr UpconvTile kUpconvTiles[] = {{4, 4, ROWS_SHAPE, 4.4, 2.4},    {4, 3, ROWS_SHAPE, 3.4, 2.2},
                                       {4, 3, COLUMNS_SHAPE, 3.4, 2.3}, {4, 3, FLAT_SHAPE, 3.4, 2.3},
                                       {8, 2, FLAT_SHAPE, 2.5, 1.6},    {8, 1, FLAT_SHAPE, 1.75, 1.3}};
constexpr int kNumUpconvTiles = (int)(sizeof(kUpconvTiles) / sizeof(kUpconvTiles[0]));

// The tile with the fewest rounds over the CUs times what one takes.  Over 60
// shapes (1 to 8 frames of 3 x 1000 to 540 x 960, whole and in bands) the picked tile
// was within 7% of the fastest of the six; in us, picked against always 4 x 4 ROWS:
// 64 x 16 x 16, 256 -> 256 channels 61 and 142; 33 of 67 rows of 90, 512 -> 512 49 and
// 73; one of 540 rows of 960, 2 frames, 128 -> 256 20 and 44.
inline int upconv_pick(const UpconvSize& p) {
  int best = 0;
  double cost = 0;
  for (int t = 0; t < kNumUpconvTiles; ++t) {
    const UpconvTile& c = kUpconvTiles[t];
    if (c.shape == FLAT_SHAPE && !upconv_flat_fits(p, c.rg, c.r)) continue;
    const int64_t rounds = (upconv_tiles(p, p.n, c.rg, c.r, c.shape) + RULE_CUS - 1) / RULE_CUS;
    const double us = (double)rounds * (p.ci / UBK * c.step_us + c.tile_us);
    if (t == 0 || us < cost) { best = t; cost = us; }
  }
  return best;
}

}  // namespace xema
