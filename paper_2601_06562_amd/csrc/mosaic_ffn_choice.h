// Which kernel and tiles a product of the feed-forward block takes (mosaic_ffn.hip), from its sizes alone: host code without
// a GPU's headers, so that the choice for any size can be asked for where there is none.
#ifndef MOSAIC_FFN_CHOICE_H_
#define MOSAIC_FFN_CHOICE_H_

#include <stdint.h>

#include <initializer_list>

#include "mosaic_layer.h"

namespace mosaic {
namespace ffn {

constexpr int kStepK = 64;
constexpr int kCus = 256;

enum { kForward, kRecompute, kDx, kDw };
constexpr bool gated_mode(int mode) { return mode == kForward || mode == kRecompute; }

inline int64_t tiles(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

// Rows of one launch; rows past them go to further ones.  It bounds the tiles of a launch, which the kernels number in 32 bits:
// the smallest are of 64 rows by 64 features (a weight gradient's by 128 columns, of both at once), and dx has parts of K only
// where parts times rows stay within kPartRows.
constexpr int64_t kLaunchRows = (int64_t)1 << 17;
static_assert((kLaunchRows / 64) * (MOSAIC_MAX_ROW / 64) <= INT32_MAX &&
                  (2 * (int64_t)MOSAIC_MAX_ROW / 64) * (MOSAIC_MAX_ROW / 128) <= INT32_MAX,
              "tiles of a launch of the projections, or dx, and of the weight gradients");

// The tiles there are, what one step of 64 k takes all CUs at work, in us, and what filling a long ring adds.  A block's step is
// bound by the latency of its copies or by the matrix cores, so a tile takes the same where it is alone and a launch takes
// whole rounds of tiles.  Tiles of 96 features for the rounds that those of 64 or 128 would leave part empty (d 4096, F 12288:
// 300 rows in 77 us for 87, 1000 in 160 for 183; d 3584, F 18944: 500 in 131 for 155).  Few rows are bound by how many
// bytes are under way: there the rings take all LDS (37 rows of d 3584, F 18944 in 50.8 us by 96 features and five slots, of
// 128 features 56.4; 32 rows of d 4096, F 12288 in 37.9 with six slots, 41.2 with three in two blocks a CU).
// Each tile forced in turn, 16 to 8192 rows of 12288 x 4096, 18944 x 3584, 5632 x 2048, 4096 x 1024 and 2048 x 512, weights from
// memory, all four products, 270 times: the choice is within 2% of the fastest in 216 and within 5% in 256.  The most it loses is
// 13%, where the projections of the backward pass would do better with 192 x 256 (1024 rows of 12288 x 4096, 194 us for 173).
// Up to how many rows dg and du have a second number an element, what the rounding of the first left over.  Twice the rows then
// still fit one tile of rows for dx and one step of K for the weights' gradients, so it costs up to 3% of a call (32 rows of d
// 4096, F 12288: 148 us for 144; 1 row 139 either way).  In the gradients of few rows few terms count, and the rounding of
// those does not average out: with it the error against 64 bits was up to 1.57 times that of the results' own rounding (1 to 3
// rows of d 512, F 2048); from 33 rows on it is 1.44 at most, about the square root of 2.
constexpr int64_t kHalvesRows = 32;
inline bool with_low_halves(int64_t T) { return T > 0 && T <= kHalvesRows; }

struct Tile { int p, q; double step, step_alone, fill; int per_cu; };
constexpr Tile kTiles[] = {
    {256, 256, 1.50, 1.50, 0.0, 1}, {128, 256, 0.91, 0.91, 0.0, 1}, {256, 128, 0.92, 0.92, 0.0, 1}, {128, 128, 0.60, 0.60, 0.0, 1},
    {256, 64, 0.80, 0.80, 0.0, 1},  {128, 64, 0.84, 0.57, 0.0, 2},  {128, 64, 0.55, 0.55, 0.6, 1},  {192, 64, 0.70, 0.70, 0.0, 1},
    {192, 128, 0.77, 0.85, 0.0, 1}, {192, 256, 1.26, 1.26, 0.0, 1},
};

// The launch of a product in tile `i`: its tiles, dealt to `blocks` blocks in turn.
struct TileGrid { int32_t p, q; int64_t n; int32_t blocks; };
inline TileGrid tile_grid(int mode, int i, int64_t rows_p, int64_t rows_q, int64_t splits) {
  const Tile& t = kTiles[i];
  TileGrid g = {(int32_t)tiles(rows_p, gated_mode(mode) ? t.p / 2 : t.p), (int32_t)tiles(rows_q, t.q), 0, 0};
  g.n = (int64_t)g.p * g.q * splits;
  g.blocks = (int32_t)(g.n < kCus * t.per_cu ? g.n : kCus * t.per_cu);
  return g;
}

struct Choice { int tile; double us; };
inline Choice choose_tile(int mode, int64_t rows_p, int64_t rows_q, int64_t steps, int64_t splits) {
  Choice best = {-1, 0.0};
  for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
    const Tile& t = kTiles[i];
    if (t.p == 192 && !gated_mode(mode)) continue;   // across K its rows would not be a power of two
    if (t.q > 64 && gated_mode(mode) && rows_q <= 64) continue;   // (slower; and the tiles of 64 rows write low halves)
    const int64_t n = tile_grid(mode, i, rows_p, rows_q, splits).n;
    const double us = (double)tiles(n, kCus * t.per_cu) * (double)tiles(steps, splits) * (n <= kCus ? t.step_alone : t.step) + t.fill;
    if (best.tile < 0 || us < best.us) best = {i, us};
  }
  return best;
}

// How the gradients of a backward pass are taken: in how many parts of K dx is summed, and in which tiles both products go
// out together (-1: in launches of their own).  The parts follow from the sizes alone, whichever gradients a call wants: dx
// has the same bits in every call.
struct GradientPlan { int32_t splits, tile; };
constexpr int64_t kMostParts = 16, kPartRows = 8192;   // parts, and parts times rows
constexpr double kLaunchUs = 4.0, kJoinBytesPerUs = 4e6;   // joining parts: a launch, and 8 bytes an element and part
inline GradientPlan plan_gradients(int64_t T, int32_t d, int32_t F) {
  GradientPlan plan = {1, -1};
  if (T == 0 || T > kLaunchRows) return plan;
  const int64_t steps_x = 2 * tiles(F, kStepK), steps_w = tiles(T, kStepK);
  const double dw = choose_tile(kDw, d, 2 * (int64_t)F, steps_w, 1).us;
  double least = 0.0;
  for (int32_t s = 1; s == 1 || (s <= kMostParts && s * T <= kPartRows && s * 4 <= steps_x); ++s) {
    const int32_t parts = with_low_halves(T) ? 2 * s : s;
    const double join = parts == 1 ? 0.0 : kLaunchUs + (double)(T * d) * 8.0 * parts / kJoinBytesPerUs;
    const double apart = choose_tile(kDx, d, T, steps_x, s).us + dw + kLaunchUs + join;
    if (s == 1 || apart < least) {
      least = apart;
      plan = {s, -1};
    }
    for (int i : {0, 1, 3}) {
      const Tile& t = kTiles[i];
      const int64_t each_x = tiles(steps_x, s), n_x = tiles(d, t.p) * tiles(T, t.q) * s;
      const int64_t n_w = tiles(d, t.p) * tiles(2 * (int64_t)F, t.q);
      if (n_x + n_w > 8 * kCus) continue;
      const int64_t longest = each_x > steps_w ? each_x : steps_w;
      double rounds = (double)(n_x * each_x + n_w * steps_w) / kCus;      // as even as the blocks allow
      if (n_x + n_w > kCus) rounds += 0.5 * (double)steps_w;
      if (rounds < (double)longest) rounds = (double)longest;
      const double together = rounds * t.step + join;
      if (together < least) {
        least = together;
        plan = {s, i};
      }
    }
  }
  return plan;
}

// Whether these rows go to the kernel for few: where its blocks are no more than the CUs, up to its 64 rows; beyond, while what
// the blocks read of x is little beside the weights (rows of d 4096, F 8192: 16 in 27.6 us, the tiles 30.9; 32 in 37.4 and
// 32.4; F 12288: 8 in 37.0 and 37.4, 16 in 39.4 and 37.6; d 3584, F 18944: 4 in 49.2 and 49.6, 16 in 57.1 and 50.0).  Past the
// features that tiles of 96 take in one round the tiles read faster (d 8192, F 28672: 1 row in 157 us for 173).  The rule has no
// d in it: up to F 4096 this kernel was the faster one for 1, 8, 16, 32 and 64 rows of every d from 1024 to 16384 (64 rows of F
// 4096, d 16384: 110 us and 112); at F 8192, 1 to 16 rows, up to d 8192 (there 47 to 49 us and 52 to 54), but not at d 16384
// (138 to 148 us and 102 to 108).
inline bool few_rows(int64_t T, int32_t F) {
  return T <= 64 && (F <= 16 * kCus || (F <= 96 * kCus && T * F <= (int64_t)1 << 17));
}

}  // namespace ffn
}  // namespace mosaic
#endif
