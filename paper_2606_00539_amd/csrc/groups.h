// Which rows a workgroup of a grouped product computes.  The group boundaries lie
// on the device (a router writes them), so a launch has a workgroup for every tile
// that the rows could make, and each finds its own tile, or that it has none.
#pragma once

#include <hip/hip_runtime.h>
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

// Tiles of kT rows that `rows` rows in g.num groups (and the rest) can make at most.
inline int64_t most_row_tiles(const GroupArgs& g, int kT) {
  if (g.offsets == nullptr) return (int64_t(g.rows) + kT - 1) / kT;
  return g.rows / kT + std::min<int64_t>(int64_t(g.num) + 1, g.rows);
}

}  // namespace gnmr
