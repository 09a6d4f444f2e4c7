// Which rows a workgroup of a grouped product computes.  The group boundaries lie
// on the device (a router writes them), so a launch has a workgroup for every tile
// that the rows could make, and each finds its own tile, or that it has none.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "gnmr_internal.h"
#include "lane_ops.h"

namespace gnmr {

// Group e's rows [*begin, *end): never outside [0, rows), whatever the boundaries hold.
__device__ __forceinline__ void group_rows(const GroupArgs& g, int e, int* begin, int* end) {
  if (g.offsets == nullptr) {
    *begin = 0;
    *end = e == 0 ? g.rows : 0;
    return;
  }
  const int a = e == 0 ? 0 : min(max(g.offsets[e], 0), g.rows);
  *begin = a;
  *end = e < g.num ? min(max(g.offsets[e + 1], a), g.rows) : g.rows;
}

__device__ __forceinline__ bool group_wanted(const GroupArgs& g, int e) {
  return g.mask == nullptr || int(g.mask[e] != 0) == g.mask_value;
}

// Position w of `total` in an order where workgroups w, w + 8, ... (which run on
// one XCD) take consecutive positions, so that they share panels in its L2.
__device__ __forceinline__ int xcd_order(int w, int total) {
  const int xcd = w % kNumXcd, q = total / kNumXcd, r = total % kNumXcd;
  return xcd * q + (xcd < r ? xcd : r) + w / kNumXcd;
}

// Position v of tiles_m x tiles_n tiles walked in groups of kRows tile rows, column by
// column: tiles taken at one time share their operands.
template <int kRows>
__device__ __forceinline__ void walk(int v, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int per = kRows * tiles_n, first = v / per * kRows;
  const int rows = min(tiles_m - first, kRows), at = v % per;
  *tm = first + at % rows;
  *tn = at / rows;
}

// Position v of the tiles on and above the diagonal of a square of tiles, by columns.
__device__ __forceinline__ void walk_triangle(int v, int* tm, int* tn) {
  int c = int((sqrtf(8.0f * float(v) + 1.0f) - 1.0f) * 0.5f);
  if (c * (c + 1) / 2 > v) --c;  // the root is rounded
  if ((c + 1) * (c + 2) / 2 <= v) ++c;
  *tn = c;
  *tm = v - c * (c + 1) / 2;
}

struct RowTile {
  int group;   // g.num: rows that no group owns
  int row;     // first row of the tile
  int rows;    // rows of the group from there on
  int tn;
};

// The tile of workgroup w among those that have rows; false where there are fewer.
// Tiles are kT rows high; the rows behind the last group make a group of their own.
template <int kT>
__device__ __forceinline__ bool find_row_tile(const GroupArgs& g, int tiles_n, int w, int lane,
                                              RowTile* t) {
  if (g.offsets == nullptr) {
    if (!group_wanted(g, 0)) return false;
    const int tiles_m = (g.rows + kT - 1) / kT;
    if (w >= tiles_m * tiles_n) return false;
    int tm;
    walk<8>(xcd_order(w, tiles_m * tiles_n), tiles_m, tiles_n, &tm, &t->tn);
    t->group = 0;
    t->row = tm * kT;
    t->rows = g.rows - t->row;
    return true;
  }
  // A lane to a group, 64 groups at a time: all tiles counted, then ours looked up.
  auto high = [&](int e, int* begin, int* end) {
    *begin = *end = 0;
    if (e <= g.num && (e == g.num || group_wanted(g, e))) group_rows(g, e, begin, end);
    return (*end - *begin + kT - 1) / kT;
  };
  int begin, end, n = 0, upto = 0, total = 0;
  for (int e0 = 0; e0 <= g.num; e0 += 64) {
    n = high(e0 + lane, &begin, &end);
    upto = int(wave_prefix(uint32_t(n)));
    total += int(lane_of(uint32_t(upto), 63));
  }
  if (w >= total * tiles_n) return false;
  const int v = xcd_order(w, total * tiles_n);
  int before = 0;
  for (int e0 = 0; e0 <= g.num; e0 += 64) {
    if (g.num >= 64) {
      n = high(e0 + lane, &begin, &end);
      upto = int(wave_prefix(uint32_t(n)));
    }
    const uint64_t here = __ballot((before + upto - n) * tiles_n <= v && v < (before + upto) * tiles_n);
    if (here != 0) {
      const int src = __ffsll((unsigned long long)here) - 1;
      const int tiles_m = int(lane_of(uint32_t(n), src));
      const int first = (before + int(lane_of(uint32_t(upto), src)) - tiles_m) * tiles_n;
      int tm;
      walk<8>(v - first, tiles_m, tiles_n, &tm, &t->tn);
      t->group = e0 + src;
      t->row = int(lane_of(uint32_t(begin), src)) + tm * kT;
      t->rows = int(lane_of(uint32_t(end), src)) - t->row;
      return true;
    }
    before += int(lane_of(uint32_t(upto), 63));
  }
  return false;
}

// Microseconds that tiles of 256 x 256 (one workgroup per CU) or 128 x 128 (two per CU) take,
// `steps` K steps of 128 bytes each, with the whole chip at work.  A 256 tile does twice as much
// per byte that passes the L1 (the 128 tile's bound: its 32 KiB a step take as long as its
// matrix-core work), but there are a quarter as many.  Measured a step and beside them: 1.45 and
// 9 us; 1.05 (two at once; 0.6 alone on a CU) and 8 us.
inline double us_of_256(double tiles, double steps) {
  return ceil(tiles / 256.0) * (1.45 * steps + 9.0);
}
inline double us_of_128(double tiles, double steps) {
  const double rest = tiles - 512.0 * floor(tiles / 512.0);
  return floor(tiles / 512.0) * (1.05 * steps + 8.0) +
         (rest <= 0.0 ? 0.0 : (rest <= 256.0 ? 0.6 : 1.05) * steps + 8.0);
}

// Whether a grouped product over `rows` rows and N columns runs in 256 tiles.  The groups' sizes
// are not known here: each is taken to leave half a tile empty.
inline bool grouped_in_256(const GroupArgs& g, int N, double steps) {
  const double empty = g.offsets == nullptr ? 0.0 : 0.5 * std::min<double>(g.num, g.rows);
  auto tiles = [&](double t) { return ceil(g.rows / t + empty) * ceil(N / t); };
  return us_of_256(tiles(256.0), steps) < us_of_128(tiles(128.0), steps);
}

// Tiles of kT rows that `rows` rows in g.num groups (and the rest) can make at most.
inline int64_t most_row_tiles(const GroupArgs& g, int kT) {
  if (g.offsets == nullptr) return (int64_t(g.rows) + kT - 1) / kT;
  return g.rows / kT + std::min<int64_t>(int64_t(g.num) + 1, g.rows);
}

}  // namespace gnmr
