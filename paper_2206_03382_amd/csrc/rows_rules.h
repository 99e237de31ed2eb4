// Which kernel a product of experts' rows that lie one behind the other takes (ragged.hip): plain host arithmetic on sizes, kept apart from the kernels so that a
// test can ask it without a GPU.  half: bf16, else fp32.  The experts' fills are on the device: what decides is the rows' mean.
#pragma once
#include "ffn_rules.h"

namespace moe {

constexpr int kThinK = 64, kThinColumns = 64, kThinWaves = 4;       // rows_thin.h: K-step, columns of a tile, waves that cut its reduction

// Rows and parts of a thin launch's tiles; ri = 0: the other tiles are the faster.
struct ThinPlan { int ri, parts; };

// The sizes that the tests and the figures of rows_thin.h are at decide nothing but these borders.  Experts: where those that can have a row leave units without a block (the measured 2 to 8 rows); with
// all experts live the streaming tiles win (16 rows of 128 experts 26.4 and 24.5, 32 rows 55 and 41).  One matrix: as few rows to a tile as leave two blocks to share its reduction
// beyond 2048 k (48 x 4096 x 4096: 16 rows, not shared 18.8, 32 rows, two blocks 15.8), one block up to there (a second launch costs more than 8 K-steps of a wave: 16 x 2048 x
// 2048 8.0 and 9.4).
static inline ThinPlan thin_plan(bool experts, int64_t E, int64_t R, int64_t K, int64_t N) {
  if (K < 1024) return {0, 1};                                      // no chain to be cut: 6.9 and 7.2 at 776 x 1544
  const int64_t strips = tiles_in(N, kThinColumns);
  if (experts) return {(E < R ? E : R) * strips <= 128 && R <= 16 ? 1 : 0, 1};
  const bool cut = K > 2048;
  for (int ri = 1; ri <= (cut ? 4 : 2); ri *= 2) {
    const int64_t tiles = tiles_in(R, 16 * ri) * strips, turns = tiles_in(K, kThinK * kThinWaves * 2);
    if (tiles > (cut ? 128 : 256)) continue;
    const int64_t parts = cut ? (256 / tiles < turns ? 256 / tiles : turns) : 1;
    return {ri, (int)(parts < 16 ? parts : 16)};
  }
  return {0, 1};
}

// Whether the tile with one stage of rows_short.h takes a product that choose_tile would give `tile`, of at least so many tiles of 128 x 128: by the reduction's length and what comes behind it
// (0.93 to 1.5 times as fast over 200 launches of 256 to 2048 columns; on average 1.17 with an activation, 1.10 with a residual alone, 1.12 without either).
static inline bool short_takes(Tile tile, int64_t tiles, int64_t K, bool act, bool joined) {
  if ((tile != Tile::k128 && tile != Tile::k256) || tiles < 256) return false;
  return K <= (act ? (tile == Tile::k256 ? 768 : 1024) : joined ? 512 : 256);
}

// How many blocks share the reduction over an expert's rows: where the tiles of dW are too few to fill the chip.  Times in us, fitted to some 400 launches of this and of other numbers of
// parts (E = 1 to 32, 256 to 4096 columns, 512 to 65536 rows): a launch 6; a K-step 0.46 of a 128 x 128 bf16 tile alone on its unit, 0.86 of two, 0.5 of a 64 x 64 fp32 tile, 0.45 for each of
// several; the second launch 3.5; the sums, written and read once, at 5 TB/s and 0.05 a part of a chain of loads.  A 256 x 256 tile takes 1.1 a K-step of 64, 1.65 where all units have one.
// Measured: 32768 rows, 512 x 512 552 (16 large tiles' fourth) -> 37, 8192 rows 147 -> 17, 8192 rows, 1024 x 1024 63 -> 32, 4 experts of 16384 rows, 512 x 512 123 -> 47.
static inline int weight_grad_parts(bool half, bool large_ok, int64_t E, double mean, int64_t K, int64_t N) {
  const int64_t tiles = E * tiles_in(K, half ? 128 : 64) * tiles_in(N, half ? 128 : 64), k = (int64_t)ceil(mean / (half ? 64 : 32));
  const double sums = (double)E * K * N * 8.0 / 5e6;
  auto cost = [&](int64_t parts) -> double {
    const int64_t blocks = tiles * parts, steps = tiles_in(k, parts);
    double t = 6.0;
    if (half) t += (double)steps * (blocks <= 256 ? 0.46 : 0.86 * (double)tiles_in(blocks, 512));
    else t += (double)steps * (blocks <= 256 ? 0.5 : 0.45 * (double)tiles_in(blocks, 256));
    return parts > 1 ? t + 3.5 + (double)parts * (sums + 0.05) : t;
  };
  double other = cost(1);
  if (half && large_ok) {
    const double t256 = (double)(E * tiles_in(K, 256) * tiles_in(N, 256)), one = 6.0 + (double)k * ceil(t256 / 256.0) * (1.1 + 0.55 * (t256 < 256.0 ? t256 / 256.0 : 1.0));
    other = one < other ? one : other;
  }
  int best = 1;
  double least = 0.93 * other;
  for (int parts = 2; parts <= 32 && parts * 2 <= k && tiles * parts <= 2048; ++parts) {
    const double c = cost(parts);
    if (c < least) { least = c; best = parts; }
  }
  return best;
}

// Whether the tile with one stage of rows_outer.h takes a bf16 product that is not shared: few rows, or few enough for many tiles.
static inline bool outer_takes(int64_t E, double mean, int64_t K, int64_t N) {
  return mean <= 64.0 || (mean <= 256.0 && E * tiles_in(K, 128) * tiles_in(N, 128) >= 512);
}

// The kernels.  kTile: the tile that `tile` names of ffn_large.h, ffn_ring.h or ffn_tile.h.
enum class RowsKernel { kTile, kThin, kShort, kOuter, kParts, kFp32, kFp32Split };

struct RowsPlan {
  RowsKernel kernel;
  Tile tile;
  int ri;                       // kThin: rows of its tile, in 16s
  int parts;                    // blocks that share a tile's reduction: kThin, kParts
};

static inline int64_t mean_rows(int64_t R, int64_t E) { return tiles_in(R, E); }

// Whether the large tile takes a product of K x N weights; gather_rows > 0: of rows of a matrix that its 32-bit offsets reach, below 4 GiB (beyond, 128 x 128 at most).
static inline bool large_takes(int64_t E, int64_t K, int64_t N, int64_t gather_rows, int64_t gather_width) {
  return K % kLargeK == 0 && N % kLargeTile == 0 && E <= kMaxExperts && gather_rows * gather_width * 2 < ((int64_t)1 << 32);
}

// fp32 of few tiles that can have rows: the reduction of 32 x 32 cut among a block's waves (fp32_split).  168 rows of 6 experts, 2856 x 528,
// which have 11 such row tiles at most: 53 us on the tiles of 64 x 64 that experts full of rows would want, 23 so.
static inline RowsPlan fp32_plan(int64_t E, int64_t R, int64_t K, int64_t N) {
  return {fp32_split(live_row_tiles(E, R, R, kSplitTile), K, N) ? RowsKernel::kFp32Split : RowsKernel::kFp32, Tile::k64, 0, 1};
}

// R rows of E experts through K x N (kNN; gather_rows: of the matrix that they are gathered from, or 0).  experts: there are offsets.  act: an activation; joined: a residual or kept values.
static inline RowsPlan product_plan(bool half, bool experts, int64_t E, int64_t R, int64_t K, int64_t N, int64_t gather_rows, bool act, bool joined) {
  if (!half) return fp32_plan(E, R, K, N);
  const ThinPlan thin = thin_plan(experts, E, R, K, N);
  if (thin.ri > 0) return {RowsKernel::kThin, Tile::k64, thin.ri, thin.parts};
  const Tile tile = choose_tile(kNN, large_takes(E, K, N, gather_rows, K), false, E, R, (double)mean_rows(R, E), K, N, gather_rows > 0, true);
  return {short_takes(tile, (R / 128) * tiles_in(N, 128), K, act, joined) ? RowsKernel::kShort : RowsKernel::kTile, tile, 0, 1};
}

// Gradients of width N back through K x N (kNT).  grad: times the derivative of the activation before.
static inline RowsPlan product_nt_plan(bool half, int64_t E, int64_t R, int64_t K, int64_t N, bool grad) {
  if (!half) return fp32_plan(E, R, N, K);
  const Tile tile = choose_tile(kNT, large_takes(E, N, K, 0, 0), false, E, R, (double)mean_rows(R, E), N, K, false, true);
  return {short_takes(tile, (R / 128) * tiles_in(K, 128), N, grad, false) ? RowsKernel::kShort : RowsKernel::kTile, tile, 0, 1};
}

// Weight gradients K x N of R rows (kTN).  Shared reductions are priced as if rows in place could take the large tile, so that a workspace needs no number of gathered rows.
static inline RowsPlan weight_grad_plan(bool half, int64_t E, int64_t R, int64_t K, int64_t N, int64_t gather_rows) {
  auto large = [&](int64_t rows) { return K % kLargeTile == 0 && N % kLargeTile == 0 && large_takes(E, K, N, rows, K); };
  const double mean = (double)mean_rows(R, E);
  const int parts = weight_grad_parts(half, large(0), E, mean, K, N);
  if (parts > 1) return {RowsKernel::kParts, Tile::k128, 0, parts};
  if (!half) return {RowsKernel::kFp32, Tile::k64, 0, 1};
  if (outer_takes(E, mean, K, N)) return {RowsKernel::kOuter, Tile::k128, 0, 1};
  return {RowsKernel::kTile, choose_tile(kTN, large(gather_rows), false, E, K, mean, R, N, gather_rows > 0, true), 0, 1};
}

}  // namespace moe
