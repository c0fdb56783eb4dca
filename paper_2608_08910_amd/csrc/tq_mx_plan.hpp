// How the gradients through MXFP4 weights run: the kernel, its tile, the splits, and the workspace. Sizes and types alone, on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/tq.h"

namespace tq {

constexpr int kStep = 64;     // rows of the weights a step
constexpr int kFewWaves = 8;  // waves of the kernel for few rows

inline int parts_of(int32_t type) { return type == TQ_F32 ? 3 : type == TQ_F16 ? 2 : 1; }
inline int64_t pad_of(int n) { return ((int64_t)n + 63) / 64 * 64; }

// How `mats` gradients of np parts meet the weights: the kernel for few rows or a tile; the splits of the steps where there are few
// tiles; and whether a gradient's parts stand below each other as np t rows of one pass (the weights are read and converted
// once; joined like splits), are passes of their own, or are split off in the tile (rows of whole pieces); and whether, past full rounds of workgroups, only the tiles of the last one are
// split, so that it is full too (7168 x 8192 of 64 steps, 3.5 rounds: 429 us, 408 so; of 128 717, 648; 5120 x 1700 of 128, 140 tiles
// of 256 x 256 181, 256 x 128 so 152). By measured times (us): of a compute unit's step with each; of a round of
// workgroups, 2.5; of a launch of the tiles, 1.8 more, and 3 where the parts are made for them alone; of joining, 3.5 and 0.05 for
// each sum and their bytes at 6 TB/s.
// Measured, columns x rows of so many steps (us):
//   1024 x 8, 8 steps      few rows 3.1                  (128 x 32 in 4 splits 6.3; in fp32 3.8, 9.3)
//   512 x 64, 128          few rows in 8 splits 10.1     (128 x 32 in 32 12.8; in fp32 12.6, 128 x 64 in its type in 32 16.1)
//   4096 x 33, 32          few rows 10.6                 (128 x 32 in 4 11.3)
//   7168 x 16, 64          128 x 32 in 4 15.8            (few rows 17.8; in fp32 128 x 64 19.8, few rows 23.9)
//   4096 x 128, 64         128 x 128 in 8 21.8           (128 x 64 in 4 20.5, 256 x 128 in 8 24.0, few rows 31.8)
//   1536 x 700, 48         256 x 128 in 4 25.6           (128 x 128 in 2 26.8, 256 x 256 in 8 26.9)
//   2048 x 2048, 64        128 x 128 48.8                (256 x 128 in 2 48.7, 256 x 256 in 4 52.7, 128 x 64 82.9)
//   4096 x 2047, 64        256 x 128 80                  (256 x 256 in 2 84, 128 x 128 108)
//   7168 x 8192, 64        256 x 256 429                 (256 x 128 501, 128 x 128 743)
//   256 x 6546, 82, fp32   256 x 128 in its type, 4 65   (256 x 256 in 8 of parts 140 with making them)
//   4096 x 128, 32, fp32   128 x 64 in its type, 4 21    (128 x 64 of parts 29 with making them)
//   4096 x 33, 32, fp32    128 x 64 in its type, 8 13.1  (few rows 14.0)
//   2048 x 2048, 64, fp32  256 x 128 in its type, 2 99   (256 x 256 in 4 of parts 120 with making them; in fp16 72, 87)
struct BwdTile {
  int bc, bn;
  float us[3];  // by the parts of a value; of parts as passes the same for each
  bool in_type;
};
constexpr BwdTile kBwdTiles[] = {{128, 32, {0.54f, 0.54f, 0.54f}, false}, {128, 64, {0.58f, 0.58f, 0.58f}, false},
                                 {128, 128, {0.75f, 0.75f, 0.75f}, false}, {256, 128, {1.06f, 1.06f, 1.06f}, false},
                                 {256, 256, {1.50f, 1.50f, 1.50f}, false}, {128, 64, {0, 0.98f, 1.15f}, true}, {256, 128, {0, 1.75f, 2.40f}, true}};
// A step for few rows, us, by the type's parts: `none` and `row` for each row of dy up to `rows`.
constexpr struct {
  double none, row;
  int rows;
} kFewStep[3] = {{0.165, 0.0045, 16}, {0.20, 0.0035, 16}, {0.235, 0.0055, 32}};
constexpr int kPlaces = 256, kMaxSplits = 32;  // compute units; partial sums only where these hold all tiles at once

struct BwdPlan {
  int tile = -1, splits = 1;  // -1: few rows
  int64_t whole = 0;          // tiles of full rounds, where only those of the last one are split
  bool stacked = false;
};
inline double join_us(double elements, int sums) { return 3.5 + 0.05 * sums + sums * elements * 8 / 6e6; }

// Rows of dy whose 16-byte pieces are whole.
inline bool whole_rows(int n, int32_t type) { return (int64_t)n * (type == TQ_F32 ? 4 : 2) % 16 == 0; }

// What making the parts costs: a launch that reads one gradient, or the planes that the gated block's element-wise pass writes beside its two.
inline double parts_us(int64_t t, int n, int mats, int32_t type) {
  if (type == TQ_BF16 && whole_rows(n, type)) return 0.0;
  const double rows = (double)t * pad_of(n);
  return mats == 1 ? 3.0 + rows * ((type == TQ_F32 ? 4 : 2) + 2 * parts_of(type)) / 5e6 : rows * 2 * 2 * parts_of(type) / 5e6;
}

inline BwdPlan plan_bwd(int64_t t, int kb, int n, int mats, int32_t type) {
  const int np = parts_of(type);
  BwdPlan best;
  double least = 1e30;
  for (int splits = 1, steps = (n + 63) / 64 * mats; splits == 1 || (splits <= kMaxSplits && splits * kFewWaves <= steps); splits *= 2) {
    const int64_t wgs = (int64_t)kb * 8 * ((t + 31) / 32) * splits;
    if (splits > 1 && wgs > 2 * kPlaces) break;
    const double step = kFewStep[np - 1].none + kFewStep[np - 1].row * std::min<int64_t>(t, kFewStep[np - 1].rows);
    const double us = 2.5 + (wgs + kPlaces - 1) / kPlaces * ((steps + splits - 1) / splits * step) + (splits > 1 ? join_us((double)t * kb * 256, splits) : 0.0);
    if (us < least) {
      least = us;
      best.splits = splits;
    }
  }
  for (int stacked = 0; stacked <= (np > 1 ? 1 : 0); ++stacked) {
    const int64_t rows = stacked ? t * np : t;
    for (int i = 0; i < (int)(sizeof(kBwdTiles) / sizeof(kBwdTiles[0])); ++i) {
      const BwdTile& c = kBwdTiles[i];
      if (c.in_type && (stacked || np == 1 || !whole_rows(n, type))) continue;
      const int steps = (n + kStep - 1) / kStep * mats * (stacked || c.in_type ? 1 : np);
      const double step = c.us[np - 1];
      const int64_t tiles = (int64_t)kb * (256 / c.bc) * ((rows + c.bn - 1) / c.bn);
      const double first = 1.8 + (c.in_type ? 0.0 : parts_us(t, n, mats, type));
      for (int splits = 1; splits <= kMaxSplits && splits <= steps; splits *= 2) {
        const bool joined = splits > 1 || stacked;
        const double share = (steps + splits - 1) / splits * step + 2.5;
        if (!joined || tiles * splits <= kPlaces) {
          const int64_t rounds = (tiles * splits + kPlaces - 1) / kPlaces;
          const double us = first + rounds * share + (joined ? join_us((double)t * kb * 256, splits * (stacked ? np : 1)) : 0.0);
          if (us < least) {
            least = us;
            best.tile = i, best.splits = splits, best.whole = 0, best.stacked = stacked;
          }
        }
        const int64_t whole = tiles / kPlaces * kPlaces, others = tiles - whole;
        if (!stacked && splits > 1 && whole && others && others * splits <= kPlaces) {
          const double us = first + tiles / kPlaces * (steps * step + 2.5) + share + join_us((double)others * c.bc * c.bn, splits);
          if (us < least) {
            least = us;
            best.tile = i, best.splits = splits, best.whole = whole, best.stacked = false;
          }
        }
      }
    }
  }
  return best;
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Room for the parts of `mats` gradients, then for partial sums: at most kPlaces tiles of 256 columns and 256 rows.
inline size_t bwd_bytes(int n, int32_t type, int64_t t, int mats) {
  const size_t planes = (size_t)mats * parts_of(type) * t * pad_of(n) * 2;
  return up256(planes) + (size_t)kPlaces * 256 * 4 * std::min<int64_t>(parts_of(type) * t, 256) + 256;
}

}  // namespace tq
