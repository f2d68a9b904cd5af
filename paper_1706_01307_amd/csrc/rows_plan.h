// Which kernels and tiles the grouped products and their weight gradient take
// (rows_grouped.hip), by rules on sizes, types and alignment: plain arithmetic on the
// host, apart from the kernels so that it can be asked without a GPU.
#pragma once

#include <cstddef>
#include <cstdint>

#include "spconv_rows.h"

namespace spc {

// (groups never have more tiles than this)
inline int64_t tile_bound(int64_t m, int64_t groups, int64_t BM) {
  return m / BM + (groups < m ? groups : m);
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------
enum class GroupedKernel { kFew, kAny, kShort, kTiles };
struct GroupedPlan {
  GroupedKernel kernel;
  int tile;                    // kAny, kTiles: its rows and columns
  int ring;                    // kTiles: stages in LDS; kShort: stages of the reduction
};

// Positions of a k_grouped_short workgroup.
constexpr int kShortRows = 256;

// Whether k_grouped_few is the faster for at most 32 positions of whole pieces, by
// an estimate of both in us: tiles take 0.2 (bf16) or 0.34 a stage however few rows
// they have; the few kernel's workgroups, above 64 of them, take turns.  (One
// position, 2048 -> 512: bf16 17.2 and 9.7 us, fp32 48 and 7.8; four of as many
// groups, 512 -> 2048: bf16 8.3 and 14.6.)
inline bool few_is_faster(bool f32, int64_t m, int E, int red, int cols) {
  const int64_t piece = f32 ? 4 : 8;
  if (m > 32 || cols % piece) return false;
  const double tiles = 5.0 + (f32 ? 0.34 / 16 : 0.2 / 32) * red;
  const double blocks = static_cast<double>(tile_bound(m, E, 4)) * cols / (4 * piece);
  const double k = red / 2048.0, over = blocks > 64 ? (blocks - 64) / 192 : 0.0;
  return 6.4 + 2.5 * k + over * (4.0 + 10.0 * k) < tiles;
}

// Which kernel: k_grouped_few by the estimate above; k_grouped_any where pieces may
// be cut or unaligned; k_grouped_short for bf16 reductions of at most 256 with at least
// 2^28 results of more than 256 columns, in groups of a workgroup's rows on average,
// fp32 results of whole 128-byte lines (256 -> 1024 of 16 groups, us of it and of the
// tiles: 700,000 positions 586 and 690, 524,288 433 and 492, 262,144 232 and 229, 65,536
// 118 and 70; 64 -> 256, 700,000: 100 and 100; 256 -> 256, 262,144: 122 and 80; 256 ->
// 1024 of 256 groups, 16,384: 79 and 47; 128 -> 384, 700,000: 179 and 291; to fp32 245
// and 354, but 40 -> 264, 1,016,800, to fp32 671 and 358; 256 -> 768, 349,525: 263 and
// 240); else k_grouped.  Its tiles are 64 x 64 for few columns and where 128 x 128
// would not fill the card twice (bf16 512 -> 512, 8,000 positions: 20 us against 26),
// for fp32 four times or without wasting columns (80 -> 144, 492,252 positions: 235
// us against 300 of 128 x 128; 1024 -> 1024, 65,536: 1,250 against 1,160); for bf16
// 256 x 256 where they fill it twice and waste little (2048 -> 2048, 65,536: 603 us
// against 692).  64 x 64 tiles have a ring of four stages while the card holds all of
// them, four a compute unit, at once (bf16 256 -> 1024, 2,000 positions: 13 us, a
// ring of three 17), else of three, for six a compute unit to hide one another's
// beginnings and ends (fp32 64 -> 64, 300,000: 43 us against 47; bf16 512 -> 512,
// 8,000 of 8 groups: 16 against 18).
// `backward`: the input gradient; red, cols: its reduction and output columns; whole:
// rows and weights are of whole aligned 16-byte pieces.
inline GroupedPlan grouped_plan(int in_dt, int out_dt, bool backward, int64_t m, int E, int red,
                                int cols, bool whole) {
  const bool f32 = in_dt == SPCONV_F32;
  if (!backward && few_is_faster(f32, m, E, red, cols)) return {GroupedKernel::kFew, 0, 0};
  const int64_t c256 = (cols + 255) / 256, c128 = (cols + 127) / 128, c64 = (cols + 63) / 64;
  const int64_t tiles = tile_bound(m, E, 128) * c128;
  const bool waste = c64 % 2 && c64 > 2 && c64 < 16;   // of the last 128 columns
  const bool small = cols <= 64 || m <= 64ll * E || (f32 ? tiles < 2048 || waste : tiles < 1024);
  if (!whole) return {GroupedKernel::kAny, small ? 64 : 128, 1};
  if (!f32) {
    if (red <= 256 && cols > 256 && cols % (out_dt == SPCONV_F32 ? 32 : 8) == 0 && m >= 16384 &&
        m >= 256ll * E && m * cols >= 1ll << 28)
      return {GroupedKernel::kShort, kShortRows,
              red <= 64 ? 2 : red <= 128 ? 4 : red <= 192 ? 6 : 8};
    if (!small && 20 * c256 <= 11 * c128 + 1 && m / 256 * c256 >= 512)
      return {GroupedKernel::kTiles, 256, 4};
  }
  if (!small) return {GroupedKernel::kTiles, 128, 4};
  return {GroupedKernel::kTiles, 64, tile_bound(m, E, 64) * c64 > 1024 ? 3 : 4};
}

// ---------------------------------------------------------------------------
// Weight gradient
// ---------------------------------------------------------------------------
// How the weight gradient is cut: tiles of dw of 64, 128 or (bf16, whole pieces)
// 256 squared, and the positions of a group into chunks (chunk = 0: each group is
// one, and its sums go straight to dw).
struct DwPlan {
  int tile;
  int64_t chunk, jobs, tiles;
  size_t bytes;
};
// The estimate it is chosen by, in us.  A stage of a tile (64 bytes a column: 16 or 32
// positions) takes `alone` with one workgroup a compute unit and `full` with four,
// two or (256) one, which `slots` counts (another one or two fit and even out the
// rest; counted too they were slower as often as faster); a workgroup 3 us besides
// its stages; the chunks' sums are written and read at 4 MB a us.  A group may have
// three times the mean.  (At eleven sizes, 1,000 to 696,416 positions, 64 x 256 to 2048 x
// 2048, within 18 % of the best of the tiles with thirteen chunks each: fp32 512 x 512 of
// 8 groups, 65,536 positions 428 us against 362, fp32 96 x 200 of 8, 1,000 positions 21
// against 18, bf16 256 x 512 of 16, 2,000 positions 16.4 against 15.0, the others within
// 6 %.)
inline double dw_cost(bool f32, int64_t m, int64_t groups, double values, int tile, double tiles,
                      int64_t chunk) {
  const int t = tile == 64 ? 0 : tile == 128 ? 1 : 2;
  static const double alone[2][3] = {{0.63, 0.98, 1.27}, {0.75, 1.6, 4.0}};
  static const double full[2][3] = {{0.8, 1.2, 1.5}, {1.35, 2.2, 4.2}};
  const double stage = f32 ? 16.0 : 32.0, slots = t == 0 ? 1024.0 : t == 1 ? 512.0 : 256.0;
  const double mean = static_cast<double>(m) / groups, longest = groups > 1 ? 3.0 * mean : mean;
  const double jobs = chunk ? static_cast<double>(m) / chunk + groups : groups;
  const double rounds = jobs * tiles / slots, fill = rounds < 1.0 ? rounds : 1.0;
  const double us = alone[f32][t] + (full[f32][t] - alone[f32][t]) * fill;
  const double length = chunk && chunk < longest ? static_cast<double>(chunk) : longest;
  const double unit = length / stage * us + 3.0, even = mean / stage * us + 3.0;
  if (!chunk) return rounds * even > unit ? rounds * even : unit;
  const double whole = static_cast<int64_t>(rounds) + (rounds > 3.0 ? 0.5 : 1.0);
  return unit * whole + 4.0 + jobs * values * 8.0 / 4e6;
}
inline DwPlan dw_plan(int dt, int64_t m, int E, int C_in, int C_out, bool wide) {
  const bool f32 = dt == SPCONV_F32;
  const int64_t groups = m < 1 ? 1 : E < m ? E : m;
  const double values = static_cast<double>(C_in) * C_out + C_out;
  const int64_t least = C_in < C_out ? C_in : C_out, widest = C_in < C_out ? C_out : C_in;
  DwPlan best{64, 0, E, 0, 0};
  double cost = 0.0;
  auto consider = [&](int tile, int64_t tiles, int64_t chunk) {
    const double c = dw_cost(f32, m, groups, values, tile, static_cast<double>(tiles), chunk);
    if (best.tiles && !(c < cost)) return;
    cost = c;
    best.tile = tile;
    best.tiles = tiles;
    best.chunk = chunk;
  };
  for (int tile = 64; tile <= 256; tile *= 2) {
    if (tile == 128 && widest <= 64) break;
    if (tile == 256 && (f32 || !wide || least <= 128)) break;
    const int64_t tiles = ((C_in + tile - 1ll) / tile) * ((C_out + tile - 1ll) / tile);
    consider(tile, tiles, 0);
    for (int64_t chunk = 64; chunk < m; chunk *= 2) consider(tile, tiles, chunk);
    // and what fills one to four rounds of the card
    const int64_t slots = tile == 64 ? 1024 : tile == 128 ? 512 : 256;
    for (int rounds = 1; rounds <= 4; ++rounds) {
      const int64_t chunks = rounds * slots / tiles - groups;
      const int64_t chunk = chunks > 0 ? ((m + chunks - 1) / chunks + 63) / 64 * 64 : 0;
      // (one less than a whole number of rounds, by the estimate's rounding up)
      if (chunk && chunk < m) consider(tile, tiles, chunk + 64);
    }
  }
  if (best.chunk) {
    best.jobs = m / best.chunk + groups;
    best.bytes = static_cast<size_t>(best.jobs) * (static_cast<size_t>(C_in) * C_out + C_out) * 4;
  }
  return best;
}
// The runs (1 or 8) that the chunks' sums of a group are added in (k_grouped_dw_sum).
inline int dw_sum_runs(const DwPlan& p, int E, int64_t values) {
  return (values + 1023) / 1024 * E < 1024 && p.jobs > 4ll * E ? 8 : 1;
}

}  // namespace spc
