// How the matrix products are cut into tiles, parts and launches, and the workspaces that they
// take: rules on sizes and types, host code only.
#pragma once

#include <algorithm>
#include <cstdint>

#include "hg.h"

namespace hg {

template <typename T>
constexpr T ceil_div(T a, T b) {
  return (a + b - 1) / b;
}

inline int64_t align16(int64_t b) { return (b + 15) / 16 * 16; }
inline int64_t size_of(int32_t dtype) {
  return dtype == HG_DT_F32 ? 4 : (dtype == HG_DT_E4M3 ? 1 : 2);
}
// Elements of q in 128 bytes of what the matrix instructions take.
inline int64_t slab_of(int32_t dtype) { return dtype == HG_DT_F32 ? 32 : 64; }

// How a product is cut: its tiles, how many slabs are in LDS, and the parts of its depth.
// A compute unit that multiplies one tile waits for its loads unless several slabs are in
// flight; with two tiles each covers the other's waits.
//  kLarge   256 x 256, 2 slabs, one block on a unit: 1.24 to 1.28 PF/s in 16 bits at 8192^3.
//           From depths of 8 slabs on (32768 rows, 2048 columns, by depth: 128 49 us, kMedium
//           45; 256 60, 57; 512 84, 84; 1024 133, 141), and not in 32 bits, whose products
//           take too long for its uneven last round
//  kMedium  128 x 128, 2 slabs, two blocks: loading a slab takes as long as multiplying it
//           (64 bytes a clock), 1.0 PF/s at 8192^3, but its tiles fill the units better
//  kSmall   64 x 64, 4 slabs, two blocks: for too few tiles of the others (1024^3: 8.8 us,
//           kMedium 18), unless the depth is long enough to be cut (rows of 512 and 1024
//           columns' gradient over 65537 rows: 172 us, kMedium 112)
//  kTall    256 x 128 in slabs of 64 bytes, two blocks: the weight gradients' operands,
//           whose slabs are read across (8192^3: 1.20 PF/s, kLarge 1.11, kMedium 1.04)
// kLarge needs two rounds of tiles: with fewer, what counts is how full the last one is, which
// the rule does not look at (us, kLarge / kMedium, tiles of 256 x 256: 16384 x 4096 x 1024, 256
// tiles, 119 / 138; 12288 x 1024 x 2048, 384, 65 / 54; 16384 x 2048 x 1792, 448, 112 / 128;
// 8192 x 4096 x 4096, 512, 224 / 262; 12288 x 2048 x 3328, 624, 167 / 160).  kTall needs half a
// round of its tiles (gradients of n x k weights over m rows, m x k x n, kTall / without:
// 16384 x 2048 x 4096, 256 tiles, 295 / 313; 16385 x 1024 x 4096, 128, 168 / 175; 8192 x 2048 x
// 2048, 128, 87 / 86; 65537 x 512 x 1024, 16, 120 / 109).
enum class Cut { kLarge, kMedium, kSmall, kTall };
struct Plan {
  Cut cut;
  int64_t tile_i, tile_j, splits, per_split;
  int64_t rows;  // of C that this plan is for; the rest have one of their own
};
constexpr int64_t kUnits = 256;

// A grid has fewer than 2^32 threads: this many tiles at most, each with 512 (of 128 x 128 where
// there are so many, whatever the plan's).  A product of more columns is made in parts of them,
// one of more rows in several launches.
constexpr int64_t kMostTiles = (int64_t(1) << 23) - 1;
constexpr int64_t kMostCols = int64_t(1) << 28;

inline int64_t tiles_of(int64_t rows, int64_t cols, int64_t ti, int64_t tj) {
  return ceil_div<int64_t>(rows, ti) * ceil_div<int64_t>(cols, tj);
}
// The share of the last round of blocks that is full, over all rounds.
inline double filled(int64_t tiles, int64_t at_once) {
  return double(tiles) / double(ceil_div<int64_t>(tiles, at_once) * at_once);
}

inline Plan plan_of(int64_t rows, int64_t cols, int64_t depth, int64_t slab, bool both, bool direct) {
  Plan p{Cut::kMedium, 128, 128, 1, 0, rows};
  if (rows > 0 && cols > 0) {
    const int64_t large = tiles_of(rows, cols, 256, 256), tall = tiles_of(rows, cols, 256, 128);
    const int64_t medium = tiles_of(rows, cols, 128, 128);
    if (both && tall >= kUnits && slab == 64)
      p = Plan{Cut::kTall, 256, 128, 1, 0, rows};
    else if (!both && large >= 2 * kUnits && depth >= 8 * slab && slab == 64)
      p = Plan{Cut::kLarge, 256, 256, 1, 0, rows};
    else if (medium <= kUnits / 2 && medium * (depth / (32 * slab)) <= kUnits / 2)
      p = Plan{Cut::kSmall, 64, 64, 1, 0, rows};
    // blocks of the small tiles whose slabs go through registers have one slab in LDS, and
    // one in flight: four on a unit (dx of 6 x 2752 by 2752 x 6874 in float32: 38 us, by
    // two 51)
    const int64_t at_once = p.cut == Cut::kLarge                 ? kUnits
                            : p.cut == Cut::kSmall && !direct ? 4 * kUnits
                                                              : 2 * kUnits;
    const int64_t tiles = tiles_of(rows, cols, p.tile_i, p.tile_j);
    if (tiles < at_once) {
      // the depth in parts of at least 8 slabs; where half the blocks are there anyway, only
      // a depth that is long next to the writing and adding of the parts: as many that their
      // rounds take least, a part's writing and adding taken as 1/32 of a slab (5408 x 912
      // over 26506 rows in float32, 344 tiles: 1825 us as 4 parts each, 2354 as one)
      const bool most_there = 2 * tiles >= at_once;
      const int64_t long_ = p.cut == Cut::kSmall ? 16 * slab : 64 * slab;
      const int64_t most = depth / (most_there ? long_ : 8 * slab);
      if (most_there) {
        double least = 0.0;
        for (int64_t s = 1; s <= std::min<int64_t>(8, most); ++s) {
          const double t = double(ceil_div<int64_t>(tiles * s, at_once)) * double(depth) /
                               double(s * slab) + (s > 1 ? 8.0 + double(s * tiles) / 32.0 : 0.0);
          if (s == 1 || t < least) p.splits = s, least = t;
        }
      } else {
        const int64_t want = std::min<int64_t>(at_once / tiles, 256);
        p.splits = std::max<int64_t>(1, std::min(want, most));
      }
    } else if (tiles <= 6 * at_once && filled(tiles, at_once) < 0.9 && depth >= 16 * slab) {
      // the rows of whole rounds; the last round's few tiles would leave most units idle
      // for as long as a full one takes, and are cut finer (us, cut / not: 25000 x 1024 x 2048,
      // rounds filled by 0.77, 110 / 124; 28000 x 2048 x 2048, 0.86, 220 / 228; 30000 x 1024 x
      // 2048, 0.92, 142 / 128; by depth, 0.80: 65537 x 1024 x 1024 137 / 145, and with 8 slabs
      // 65537 x 512 x 1024 82 / 85, but 137 / 133 with residual and pre)
      const int64_t down = tiles / at_once * at_once / ceil_div<int64_t>(cols, p.tile_j);
      if (down > 0) p.rows = down * p.tile_i;
    }
    p.rows = std::min(p.rows, kMostTiles / ceil_div<int64_t>(cols, 128) * 128);
    // any operands: tiles of 128 x 128 or 64 x 64; the parts and rows stay as planned
    if (!direct && p.cut != Cut::kSmall) p.cut = Cut::kMedium, p.tile_i = p.tile_j = 128;
  }
  p.per_split = ceil_div<int64_t>(ceil_div<int64_t>(depth, slab), p.splits) * slab;
  if (p.per_split < slab) p.per_split = slab;
  p.splits = depth > 0 ? ceil_div<int64_t>(depth, p.per_split) : 1;
  return p;
}
// Bytes of the parts of a product, its rows taken plan by plan, whatever its operands'
// alignment.  (So many columns that they are taken in parts make more tiles than are ever cut.)
inline int64_t parts_bytes(int64_t rows, int64_t cols, int64_t depth, int64_t slab, bool both) {
  int64_t most = 0;
  if (cols > kMostCols) return 0;
  for (const bool direct : {false, true})
    for (int64_t left = rows; left > 0 && cols > 0;) {
      const Plan p = plan_of(left, cols, depth, slab, both, direct);
      if (p.splits > 1) most = std::max(most, p.splits * p.rows * cols * 4);
      left -= p.rows;
    }
  return most;
}

// The elements of a row laid out in whole pieces.
inline int64_t padded(int64_t cols, int64_t size) { return align16(cols * size) / size; }

// Whether a product's operands whose rows are not whole 16-byte pieces are first copied
// into rows that are, for the kernel of aligned operands: where the product is large and
// every element is used often enough (us, forward / dx / dw, without and with the copies):
//   bfloat16  13222 x 2594 x 3968  401 / 630 / 865, 335 / 325 / 359
//              4096 x  255 x 4097   41 / 128 /  82,  41 /  64 /  68
//             16385 x  515 x  515   29 /  45 /  95,  45 /  50 /  69
//              1000 x 1001 x 1003   15 /  21 /  30,  20 /  34 /  35
//   float32   13222 x 2594 x 3968  2363 / 2669 / 2969, 1708 / 1660 / 1719
//              1000 x 1001 x 1003   37 /  47 /  51,  42 /  52 /  52
// (Operands of 16 GiB and more are not copied.)
inline bool is_laid(int64_t m, int64_t k, int64_t n, int64_t size) {
  return std::min(m, std::min(k, n)) >= 250 && double(m) * double(k) * double(n) >= 4e9 &&
         double(std::max(m, n)) * double(padded(k, size) * size) < 1.6e10;
}

// Products of few rows have a kernel of their own.  (A grid has fewer than 2^32 threads.)
constexpr int64_t kFew = 32;
inline bool is_few(int64_t rows, int64_t cols) { return rows <= kFew && cols <= int64_t(1) << 26; }

// Few rows: blocks of 4 wavefronts, or of 16 where there are few columns; with very few,
// the depth is cut too, in parts of at least two steps of 128 bytes for a wavefront.
struct FewPlan {
  int64_t blocks, waves, splits, per_split;
};
inline FewPlan few_plan(int64_t cols, int64_t depth, int64_t size) {
  FewPlan p;
  p.blocks = ceil_div<int64_t>(cols, 16);
  p.waves = p.blocks >= 512 ? 4 : 16;
  const int64_t step = p.waves * (128 / size);
  const int64_t want = p.blocks < 128 && p.blocks > 0 ? 256 / p.blocks : 1;
  const int64_t most = depth / (2 * step);
  p.splits = want < most ? want : most;
  if (p.splits < 1) p.splits = 1;
  p.per_split = ceil_div<int64_t>(ceil_div<int64_t>(depth, step), p.splits) * step;
  if (p.per_split < step) p.per_split = step;
  p.splits = depth > 0 ? ceil_div<int64_t>(depth, p.per_split) : 1;
  return p;
}

constexpr int64_t kSumRows = 64;  // rows of C that one part of the column sums covers

struct LinearSpace {  // byte offsets in the workspace
  int64_t w, x, parts, total;
  bool laid;
};
inline LinearSpace linear_space(int64_t m, int64_t k, int64_t n, int32_t dtype) {
  LinearSpace s{0, 0, 0, 0, false};
  if (is_few(m, n)) {
    const int64_t splits = few_plan(n, k, size_of(dtype)).splits;
    s.total = splits > 1 ? splits * m * n * 4 : 0;
    return s;
  }
  const int64_t size = size_of(dtype), row = padded(k, size);
  s.laid = row != k && is_laid(m, k, n, size);
  if (s.laid) {
    s.x = n * row * size;
    s.parts = s.x + m * row * size;
  }
  s.total = s.parts + parts_bytes(m, n, k, slab_of(dtype), false);
  return s;
}

struct GradSpace {  // byte offsets in the workspace
  int64_t dz, sums, x, w, parts, total;
  int64_t dz_stride;  // of dz in the workspace
  bool dz_laid, laid;
};
inline GradSpace grad_space(int64_t m, int64_t k, int64_t n, int32_t dtype, int32_t act) {
  GradSpace g{};
  const int64_t slab = slab_of(dtype);
  const int64_t size = size_of(dtype), row = padded(k, size);
  g.dz_stride = padded(n, size);
  g.laid = row != k && is_laid(m, k, n, size);
  if (double(m) * double(g.dz_stride) * double(size) > 0x1p61) {  // (of broadcast rows: no array is)
    g.total = INT64_MAX;
    return g;
  }
  g.dz_laid = act != HG_ACT_NONE || (g.dz_stride != n && is_laid(m, k, n, size));
  g.sums = g.dz_laid ? m * g.dz_stride * size : 0;
  g.x = g.sums + align16(ceil_div<int64_t>(m, kSumRows) * n * 4);
  g.w = g.x + (g.laid ? m * row * size : 0);
  g.parts = g.w + (g.laid ? n * row * size : 0);
  const int64_t a = parts_bytes(m, k, n, slab, false), b = parts_bytes(n, k, m, slab, true);
  g.total = g.parts + align16(a > b ? a : b);
  return g;
}

}  // namespace hg
