// Host-side rules of a mixture-of-experts layer in training: limits, sizes of workspaces, and which kernel a call takes, by its sizes alone.
#pragma once
#include <algorithm>

#include "tl_host.h"

namespace tl {

// ---- rows sorted by expert
constexpr int kMaxChoices = 32;         // topk
constexpr int kMaxSortExperts = 256;
constexpr int kMaxSortRows = 1 << 20;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;

inline int sort_rows_per_thread(long n) {
  int r = 1;
  while (r < 8 && (n + (long)kSortThreads * r - 1) / ((long)kSortThreads * r) > 128) r *= 2;
  return r;
}

inline int sort_chunks(long n) { const long c = (long)kSortThreads * sort_rows_per_thread(n); return (int)((n + c - 1) / c); }

// ---- rows of tokens <-> rows sorted by expert
// From here on sorted rows go past the caches -- counted as all there can be, for how many take part is known on the device only.  Stores: beyond the
// dies' L2 together (1024 tokens of 4096, top-8, gradients of combine: 33.2 us, streaming stores 24.4).  Loads: beyond the memory's own cache,
// and beyond half of it in the gradient of combine, whose rows are the forward pass's (16384 tokens of 2048, top-2: 67 us, streaming loads 57).
constexpr long kStreamStores = 32L << 20, kStreamLoads = 256L << 20;
inline long sorted_bytes(int T, int H, int topk, int max_rows) {
  const long rows = (long)T * topk;
  return (rows < max_rows ? rows : max_rows) * H * 2;
}

// The gradient of combine: up to here a row is a wave's alone (14000 tokens of 160, top-6: 18 us, 39 with four waves a token; 8192 of 1024, top-5, 37 and 41;
// 4096 of 2048, top-8, 78 and 56).
constexpr int kWaveRow = 1024;

// Which of a row kernel's variants a call takes.
struct RowsChoice {
  bool stream_loads, stream_stores;
  int waves;               // of a token
};
inline RowsChoice dispatch_choice(int T, int H, int topk, int max_rows) { return {false, sorted_bytes(T, H, topk, max_rows) > kStreamStores, 1}; }
inline RowsChoice gather_choice(int T, int H, int topk, int max_rows) { return {sorted_bytes(T, H, topk, max_rows) > kStreamLoads, false, 1}; }
inline RowsChoice combine_grad_choice(int T, int H, int topk, int max_rows) {
  const long bytes = sorted_bytes(T, H, topk, max_rows);
  return {bytes >= kStreamLoads / 2, bytes > kStreamStores, H <= kWaveRow ? 1 : 4};
}

// ---- the routing weights' gradient: lanes of a token, logits of a lane
inline int route_lanes(int topk) { return topk <= 16 ? 16 : 32; }
inline int route_per(int E, int lanes) {
  int per = 1;
  while (per * lanes < E) per *= 2;
  return per;
}

// ---- the experts' products
constexpr int kMaxProductExperts = 256;
constexpr int kMaxParts = 8;              // of a cut sum
constexpr int kPartUnit = 64;             // values of Y's and dX's sums that parts are made of
constexpr int few_columns(bool grad_x, bool wide) { return (grad_x ? 32 : 64) * (wide ? 2 : 1); }     // of a unit of the few-row kernel

// Which kernel Y and dX take, by all rows; how they fall to the experts is known on the device only.  Times below are of even rows and of uneven
// ones (shares exp(0.7 gauss), one expert without).
//
// The few-row kernel takes a wide unit (128 columns; dX 64) of up to 64 rows at the speed of a compute unit's loads, so rows beyond 64 of an
// expert cost a whole unit more.  With more than a unit for each compute unit it is taken up to 48 rows an expert in the mean (32 experts
// of 2048 x 1536 with 40 rows: 42 and 42 us, tiles 50 and 50), dX, whose tiles load less, up to 32 (with 40 rows 40 and 56, tiles 45 and 45).  With
// fewer units tiles need one round, too: with a sum up to 2048 Y gains nothing from it beyond 4 rows (8 of 1024 x 4096 with 12 rows 15 and 16 us, tiles 15
// and 15; with 40 rows 17 and 26, tiles 16 and 18; but a single row through 2048 x 2048 8.8, tiles 11.6), with a longer one up to 32 rows (8 of 4096 x 2048 with 24 rows 31 and 29, tiles 38 and 37; with 40 33
// and 60, tiles 39 and 36), dX up to 48.  Not where few tiles of 128 x 128 share a long sum, which is then cut: a single row through 8192 x 1024 28 ->
// 13 us, 128 rows of 2 experts of 8192 x 512 45 -> 17, 160 of 4 of 7168 x 2048 59 -> 31; dX's few rows, whose weights arrive in whole lines, gain
// nothing at 4096.
//
// Otherwise tiles of 256 or of 128, the last round's sums cut or not, whichever takes less by this model, in us: a round of large tiles takes 1.6
// for 64 values of the sum, one of small ones 0.65; a last round that is not full half of that and its share of the other half, for its
// tiles have the memory and the chip's power to themselves; a cut one its part; the join of large tiles' parts 35, of small ones' 10.  Cut only
// sums beyond 2048: of the shorter ones as many lose by the join's launch, 3 us of 100, as gain.  8 experts of 4096 x 2048 with 2048 rows each
// 270 -> 243 us, dX of 8 of 4096 x 14336 with 512 rows 696 -> 488, 2 of 4096 x 4096 with 2048 150 -> 122.  Over 460 calls of 96 to 4096 rows an
// expert the choice takes 2 % more than the best of the four -- in buffers of as many rows as there are.  With room for two and four times as many the choice is
// that of more rows: mostly the same time, up to 26 us more (Y of 1024 rows of 32 experts of 4096 x 1792 82, 95 and 108 us, dX of 4096 rows of 8 of
// 1024 x 2816 42, 67 and 67).
constexpr int kCutSum = 2048;
struct ProductShape {
  int tile;                // 0: the few-row kernel
  bool cut;
  size_t ws_bytes;
};
// Rounds of tiles: whole ones, and one that is partly filled for more than every other expert.
inline double product_rounds(const tl_ctx* ctx, int max_rows, int E, int ndim, int tile, bool cut) {
  const double rounds = (((long)max_rows + tile - 1) / tile + 0.6 * (std::min(max_rows, E) - 1)) * ceil_div(ndim, tile) / ctx->num_cus;
  const double whole = (double)(long)rounds, rest = rounds - whole;
  if (rest <= 0) return whole;
  if (cut && rest <= 0.5) return whole + 1.0 / (rest * kMaxParts < 1 ? kMaxParts : (int)(1 / rest));
  return whole < 1 && !cut ? 1.0 : whole + 0.5 + 0.5 * rest;
}
inline ProductShape product_shape(const tl_ctx* ctx, bool grad_x, int max_rows, int K, int N, int E) {
  const int kdim = grad_x ? N : K, ndim = grad_x ? K : N;
  const long used = std::min(max_rows, E), units = used * ceil_div(ndim, few_columns(grad_x, true));
  const long mean = units > ctx->num_cus ? (grad_x ? 32 : 48) : grad_x ? 48 : kdim <= 2048 ? 4 : 32;
  const bool long_sum = 3 * ((long)max_rows / 128 + used) * ceil_div(ndim, 128) <= ctx->num_cus && kdim > (grad_x ? 4096 : 2048);
  if (max_rows <= mean * E && !long_sum) return {0, false, 256};
  ProductShape s = {};
  double least = 0;
  for (int tile = 128; tile <= 256; tile += 128)
    for (int cut = 0; cut <= (kdim > kCutSum); cut++) {
      const double us = kdim / 64.0 * (tile == 128 ? 0.65 : 1.6) * product_rounds(ctx, max_rows, E, ndim, tile, cut) + (!cut ? 0 : tile == 128 ? 10 : 35);
      if (s.tile && us >= least) continue;
      least = us;
      s.tile = tile;
      s.cut = cut;
    }
  s.ws_bytes = 256 + (s.cut ? (size_t)ctx->num_cus * s.tile * s.tile * sizeof(float) : 0);
  return s;
}

// How the few-row kernel is launched: width of its units, waves that share one, units side by side in a workgroup.
//
// A compute unit takes about 60 GB/s whatever its waves are, and more of them with longer lines, so: the widest units that leave none
// with twice the others' share.  Wide ones side by side where there is more than one for each compute unit (31 experts of
// 2048 x 1536: 30 us, one a workgroup with two waves for the summed axis 39); one a workgroup, two waves, where there is one for each or for
// more than half (320 rows of 8 of 4096 x 4096: 48 us, side by side 76, 16 rows 42 and 52; 64 rows of 6 of 4096 x 3584 37, narrow 54); else
// narrow ones, with two or four waves (7 of 4096 x 2048: 26 us against 39 with one; a single one of 4096 x 4096: 19 us against 21 with two).
struct FewChoice {
  bool wide;
  int waves, beside;
};
inline FewChoice few_choice(const tl_ctx* ctx, bool grad_x, int max_rows, int E, int ndim) {
  const int narrow = few_columns(grad_x, false);
  const long used = std::min(max_rows, E), wide = used * ceil_div(ndim, few_columns(grad_x, true));
  if (wide > ctx->num_cus) return {true, 1, 2};
  if (wide * 2 > ctx->num_cus) return {true, 2, 1};
  return {false, used * ceil_div(ndim, narrow) * 2 >= ctx->num_cus ? 2 : 4, 1};
}

// ---- the gradient of the experts' weights
constexpr int kMinPart = 256;             // rows
struct GradWExpert {                      // (a 16-byte load)
  int row, rows;                          // of x and dy
  unsigned what;                          // expert, parts << 8
  int place;                              // of its first part's sums
};
// At the front of the workspace: the experts by their rows, most first (of many rounds only those with many more than the mean), each
// with the number of its first item.  Items of an expert: part by part, all tiles of each.
struct GradWPlan {
  int first[kMaxProductExperts];
  GradWExpert expert[kMaxProductExperts];
  int n_items, n_cut;                     // cut tiles
};
constexpr int kPlanThreads = 256;

struct GradWShape {
  int bm, bn, nbm, nbn, places, run;
  long grid;                                   // items at most, in whole runs for every die
  size_t partial_at, ws_bytes;
};
inline GradWShape grad_w_shape(const tl_ctx* ctx, int max_rows, int K, int N, int E) {
  GradWShape s;
  const int cus = std::min(ctx->num_cus, 1 << 16);
  // By the rounds that tiles of 256 x 256 would make.  Up to 0.6: 128 x 128 (8 experts of 1024 x 1024 over 512 rows 23 us, 128 x 256 24, large 29; over
  // 2048 47, 57, 73).  Beyond: 128 x 256 with two workgroups a compute unit, whose beginnings and ends run beside another's sum (4 of
  // 2048 x 2048 over 512 rows 29 us, large 32, small 38; 32 of 2048 x 1536 over 256 rows 73, 81, 118).  Large ones, which need less loaded for a product, where sums
  // are long, in 2.5 rounds and more (16 of 1024 x 2816 over 1024 rows 100 us, half ones 111; 32 of 2048 x 1536 199 and 212) or cut evenly (one
  // of 8192 x 1024 over 8192 rows 137, small ones 160).
  const long tiles = (long)E * ceil_div(K, 256) * ceil_div(N, 256);
  const bool small = 5 * tiles <= 3L * cus, large = (2 * tiles >= 5L * cus || (small && E == 1)) && tiles * max_rows / E >= 2500L * cus;
  s.bm = large ? 256 : 128;
  s.bn = small && !large ? 128 : 256;
  s.nbm = ceil_div(K, s.bm);
  s.nbn = ceil_div(N, s.bn);
  const long per = (long)s.nbm * s.nbn;
  // A share is all rows x tiles over the compute units, and no sum is longer than all rows: none is cut where every expert has a tile for every
  // unit.  A cut one of n rows has fewer than 2 n / share parts in each of its tiles, all together fewer than two for every unit.
  // Nor are sums of fewer than 1536 rows in the mean, where the cut and its join cost more than uneven ones (16 of 1024 x 2816 over 1024 rows 100 us, cut 107).
  s.places = per < cus && max_rows >= 1536L * E ? 2 * cus : 0;
  s.run = (int)std::min((per + 3) / 4, 64L);
  const long span = (long)s.run * kXcds;
  s.grid = (E * per + s.places + span - 1) / span * span;
  auto up = [](size_t b) { return (b + 127) / 128 * 128; };
  s.partial_at = up(sizeof(GradWPlan));
  s.ws_bytes = up(s.partial_at + (size_t)s.places * s.bm * s.bn * sizeof(float));
  return s;
}

}  // namespace tl
