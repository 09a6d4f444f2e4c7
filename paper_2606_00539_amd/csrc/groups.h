// Which rows a workgroup of a grouped product computes.  The group boundaries lie
// on the device (a router writes them), so a launch has a workgroup for every tile
// that the rows could make, and each finds its own tile, or that it has none.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

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
__host__ __device__ inline int xcd_order(int w, int total) {
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

// Stores v at p, past the caches or through them.  (Without the empty statements around it the
// compiler joins the two stores into one of the ordinary kind.)
template <class V>
__device__ __forceinline__ void put(V* p, const V& v, bool past) {
  if (past) {
    asm volatile("");
    __builtin_nontemporal_store(v, p);
    asm volatile("");
  } else {
    *p = v;
  }
}

// Whether a product's bf16 rows are written past the caches: where they are more than those keep
// beside the operands anyway.  us through and past them, alone and with a pass over the output
// behind it: 66 MB of 64 experts 190 and 180, 217 and 216; 216 MB of 13824 features 880 and 848, 956
// and 938; 24 MB 59 and 58, but 67 and 68.
inline bool past_caches(int64_t rows, int64_t cols) { return rows * cols * 2 > int64_t(32) << 20; }

struct RowTile {
  int group;   // g.num: rows that no group owns
  int row;     // first row of the tile
  int rows;    // rows of the group from there on
  int tn;
};

// Which of a launch's tiles a kernel takes: all; or of 256 tiles those that make whole rounds over
// the chip, and the rest, cut into quarters, where the rest is at most half a round.
enum Share { kAll, kRounds, kRest };
__host__ __device__ inline int whole_rounds(int tiles) {
  const int rest = tiles % 256;
  return rest <= 128 ? tiles - rest : tiles;
}

// Position of workgroup w in the order of `total` tiles, and for kRest its quarter; false where
// the kernel's share is smaller.
template <Share kShare>
__device__ __forceinline__ bool place_of(int w, int total, int* v, int* part) {
  const int whole = kShare == kAll ? total : whole_rounds(total);
  const int mine = kShare == kRest ? 4 * (total - whole) : whole;
  if (w >= mine) return false;
  *v = xcd_order(w, mine);
  *part = 0;
  if (kShare == kRest) {
    *part = *v & 3;
    *v = whole + (*v >> 2);
  }
  return true;
}

// The tile of workgroup w among those that have rows; false where there are fewer.  Tiles
// are kT rows high; the rows behind the last group make a group of their own.  kRest (kT =
// 128): quarters of 256 tiles, tiles_n of which lie side by side; a quarter may have no rows.
template <int kT, Share kShare>
__device__ __forceinline__ bool find_row_tile(const GroupArgs& g, int tiles_n, int w, int lane,
                                              RowTile* t) {
  static_assert(kShare != kRest || kT == 128, "quarters of 256 tiles");
  constexpr int kHigh = kShare == kRest ? 256 : kT;
  int v, part, tm;
  auto quarter = [&] {
    if constexpr (kShare == kRest) {
      t->row += kT * (part >> 1);
      t->rows -= kT * (part >> 1);
      t->tn = 2 * t->tn + (part & 1);
    }
    return t->rows > 0;
  };
  if (g.offsets == nullptr) {
    if (!group_wanted(g, 0)) return false;
    const int tiles_m = (g.rows + kHigh - 1) / kHigh;
    if (!place_of<kShare>(w, tiles_m * tiles_n, &v, &part)) return false;
    walk<8>(v, tiles_m, tiles_n, &tm, &t->tn);
    t->group = 0;
    t->row = tm * kHigh;
    t->rows = g.rows - t->row;
    return quarter();
  }
  // A lane to a group, 64 groups at a time: all tiles counted, then ours looked up.
  auto high = [&](int e, int* begin, int* end) {
    *begin = *end = 0;
    if (e <= g.num && (e == g.num || group_wanted(g, e))) group_rows(g, e, begin, end);
    return (*end - *begin + kHigh - 1) / kHigh;
  };
  int begin, end, n = 0, upto = 0, total = 0;
  for (int e0 = 0; e0 <= g.num; e0 += 64) {
    n = high(e0 + lane, &begin, &end);
    upto = int(wave_prefix(uint32_t(n)));
    total += int(lane_of(uint32_t(upto), 63));
  }
  if (!place_of<kShare>(w, total * tiles_n, &v, &part)) return false;
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
      walk<8>(v - first, tiles_m, tiles_n, &tm, &t->tn);
      t->group = e0 + src;
      t->row = int(lane_of(uint32_t(begin), src)) + tm * kHigh;
      t->rows = int(lane_of(uint32_t(end), src)) - t->row;
      return quarter();
    }
    before += int(lane_of(uint32_t(upto), 63));
  }
  return false;
}

// Microseconds that `tiles` tiles of kT x kT take, `steps` K steps of 128 bytes each, where the
// product touches `bytes` of memory.  A 256 tile (one to a CU) does twice as much per byte that
// passes the L1 as a 128 tile (two to a CU), whose bound that is (its 32 KiB a step take as long
// there as its matrix-core work), and a 64 tile (two to a CU) a quarter; but of the smaller ones
// there are 4 and 16 times as many to spread over the chip.  Fitted to products of 128 G x 128 G
// x K, us in tiles of 64 / 128 / 256:
//   K        512               2048              8192
//   G = 4    9.1  9.1  14.3    9.0 14.9  36.0    25  74 127
//   G = 11   8.6  8.4  15.0   14.0 22.5  38.0    47  76 128
//   G = 16  11.7  8.6  15.5   27.0 24.0  39.0    90  74 130
//   G = 22  19.5 17.5  16.9   48.4 31.6  40.3   178 110 134
//   G = 32  37.1 23.4  30.3   96.1 62.0  56.3   366 223 192
//   G = 45  71.7 41.7  53.8  195  119   142     730 437 491
// and to what the memory-side cache cannot hold, where a 128 tile's step takes longer and a 256
// tile's does not: 24,576 rows, 2048 to 1408, in 1, 32 and 64 groups 146, 174 and 194, and 154,
// 159 and 181; 64 products 1408 x 1408 x 2048 633 and 549.
template <int kT>
double us_of_tiles(double tiles, double steps, double bytes) {
  constexpr double kRound = kT == 256 ? 256 : 512;  // tiles that run at once
  constexpr double kCacheBytes = 256e6;
  const double rounds = floor(tiles / kRound), rest = tiles - rounds * kRound;
  if (kT == 256)  // (with few tiles the clock is higher)
    return rounds * (1.35 * steps + 16.0) +
           (rest <= 0.0 ? 0.0 : (0.95 + 0.48 * rest / 256.0) * steps + 8.0);
  const double two = kT == 64 ? 0.31 : bytes > kCacheBytes ? 1.08 : 0.84;
  const double alone = kT == 64 ? 0.15 : 0.53;
  return rounds * (two * steps + 5.0) +
         (rest <= 0.0 ? 0.0 : (rest <= 256.0 ? alone : two) * steps + 6.0);
}

// Whether the last tiles of a launch of 256 tiles get a launch of their own (which ends at once
// where the groups leave it none, and takes 5 us then): from this many K steps on what it can save
// outweighs it.  8,191 rows in 8 groups, 11008 to 4096 (576 tiles): 773 us in one launch, 709 in
// two, of which the quarters take 155 to 210 (us_of_tiles would say 97).
constexpr int kSplitSteps = 32;

// Microseconds that a tile's end takes for `beside` bytes beside each value of its result: in a 256
// tile nothing covers them, in smaller ones the CU's other workgroup does in part.  d of 24,576 rows in
// 64 groups, 2048 to 1408 (6 bytes): 289 us in 256 tiles, 237 in 128 tiles.
template <int kT>
double us_beside(double tiles, double beside) {
  return tiles * kT * kT * beside / (kT == 256 ? 4.6e6 : 6.4e6);
}

// The tile edge of a product of grouped rows, N columns and `steps` K steps, whose weights have
// `weight` bytes a value, and each value of the result `beside` more than its own two.  The groups'
// sizes are not known here: each is taken to leave half a tile empty.
inline int grouped_tile(const GroupArgs& g, int N, int K, int weight, double beside = 0.0,
                        double* us = nullptr) {
  const double rows = g.rows, steps = ceil(double(K) * weight / 128.0);
  const double used = std::min<double>(g.num, rows);  // groups with rows, at most
  const double empty = g.offsets == nullptr ? 0.0 : 0.5 * used;
  const double bytes = rows * (double(K) * weight + 2.0 * N) + used * N * double(K) * weight;
  auto tiles = [&](double t) { return ceil(rows / t + empty) * ceil(N / t); };
  const double us64 = us_of_tiles<64>(tiles(64.0), steps, bytes) +
                      us_beside<64>(tiles(64.0), beside);
  const double us128 = us_of_tiles<128>(tiles(128.0), steps, bytes) +
                      us_beside<128>(tiles(128.0), beside);
  const double us256 = us_of_tiles<256>(tiles(256.0), steps, bytes) +
                       us_beside<256>(tiles(256.0), beside);
  if (us != nullptr) *us = std::min(us64, std::min(us128, us256));
  return us64 <= us128 && us64 <= us256 ? 64 : us128 <= us256 ? 128 : 256;
}

// Tiles of products one after the other on a CU (mm_stream.h), and whether that is the way for a
// product of grouped rows, `bytes` of memory to each value of whose result are read and written at its
// tiles' ends.  A call takes 4 us, a step `step` and the bytes of a tile's end 64 KB to a us.  With the
// products and for the gradient fitted to 65 shapes (300 to 65,536 rows, up to 128 groups, K 256 to 4096): for
// 5 of their 130 calls the slower way is taken by 5 to 10%, for the others by less or not at all.  us one after
// the other, and in tiles of the best edge: 24,640 rows in 64 groups, 2048 to 2 x 1408, both products and h
// (3 bytes) 344 and 423, the gradient (8) 222 and 235; 5,000 rows in 64 groups, 4096 to 2 x 2752, 573 and 749;
// 9,000 rows in 8 groups, 320 to 2 x 688, 20.8 and 24.8; but 8,192 rows, 4096 to 2 x 11008, 1,151 and 1,103,
// 5120 to 2 x 13824, 2,100 and 1,910.
constexpr int kStreamM = 128, kStreamN = 256;
inline bool streams(const GroupArgs& g, int N, int K, double beside, double bytes, double step = 0.70) {
  if (K % 64 != 0 || K < 256) return false;     // (whole steps, two rounds of three at least)
  double tiles_us;
  grouped_tile(g, N, K, 2, beside, &tiles_us);
  const double used = std::min<double>(g.num, g.rows);
  const double tiles = ceil(double(g.rows) / kStreamM + (g.offsets == nullptr ? 0.0 : 0.5 * used)) *
                       ceil(double(N) / kStreamN);
  const double steps = ceil(K / 192.0) * 3.0;
  return 4.0 + ceil(tiles / 256.0) * (step * steps + kStreamM * kStreamN * bytes / 64e3) < tiles_us;
}

// The launches of a batch of products of K8: X X^T and A A, symmetric (tiles on and above the
// diagonal), and P X, with X m x n.
enum class BatchProduct { kOfRows, kOfSquares, kOntoRows };
struct BatchLaunch {
  int64_t all, large;   // tiles of 256, and how many of them, from the first, run as such
  int edge;             // of the tiles that the others are cut into (0: there are none)
};
// All tiles of one edge, or 256 tiles in whole rounds over the chip and the rest, which would not
// fill another, in smaller ones; whichever takes the least by us_of_tiles.
inline BatchLaunch batch_launch(BatchProduct what, int count, int m, int n) {
  const bool square = what != BatchProduct::kOntoRows;
  // tiles of an edge that lie in the products; of the smaller ones a share makes up the rest
  auto tiles = [&](double t) {
    const double h = ceil(m / t), w = ceil(n / t);
    return count * (square ? h * (h + 1) / 2 : h * w);
  };
  const int64_t all = int64_t(tiles(256.0)), rest = all % 256;
  const double steps = (what == BatchProduct::kOfRows ? n : m) / 64;
  const double share = double(rest) / double(all), kLaunch = 4.0;
  const double bytes = 2.0 * count * m * (what == BatchProduct::kOfRows      ? n + m
                                          : what == BatchProduct::kOfSquares ? 2.0 * m
                                                                             : m + 2.0 * n);
  const double whole = us_of_tiles<256>(double(all - rest), steps, bytes) + kLaunch;
  const double us[5] = {us_of_tiles<64>(tiles(64.0), steps, bytes),
                        us_of_tiles<128>(tiles(128.0), steps, bytes),
                        us_of_tiles<256>(double(all), steps, bytes),
                        whole + us_of_tiles<64>(share * tiles(64.0), steps, bytes),
                        whole + us_of_tiles<128>(share * tiles(128.0), steps, bytes)};
  const int best = int(std::min_element(us, us + (rest < all && rest > 0 ? 5 : 3)) - us);
  return BatchLaunch{all, best < 2 ? 0 : best == 2 ? all : all - rest,
                     best == 2 ? 0 : best == 0 || best == 3 ? 64 : 128};
}

// Tiles of kT rows that `rows` rows in g.num groups (and the rest) can make at most.
inline int64_t most_row_tiles(const GroupArgs& g, int kT) {
  if (g.offsets == nullptr) return (int64_t(g.rows) + kT - 1) / kT;
  return g.rows / kT + std::min<int64_t>(int64_t(g.num) + 1, g.rows);
}

// The launches of a product of grouped rows and N columns.
struct RowLaunch {
  int tile;       // edge
  int tiles_n;    // tiles side by side
  int64_t most;   // tiles, at most
  bool split;     // of 256 tiles only those of whole rounds, and a launch of the rest in quarters
};
inline RowLaunch row_launch(const GroupArgs& g, int N, int K, int weight, double beside = 0.0) {
  RowLaunch r{grouped_tile(g, N, K, weight, beside), 0, 0, false};
  r.tiles_n = (N + r.tile - 1) / r.tile;
  r.most = most_row_tiles(g, r.tile) * r.tiles_n;
  if (r.tile < 256) return r;
  // (without offsets the tiles are known here)
  r.split = int64_t(K) * weight >= 128 * kSplitSteps &&
            (g.offsets != nullptr || whole_rounds(int(r.most)) < r.most);
  return r;
}

// Bytes that a value of the gated gradient's product costs beside its own: two of p are read, and two written.
constexpr double kGatedDgradBeside = 6.0;
inline bool gated_dgrad_streams(const GroupArgs& g, int H, int K) {
  return streams(g, H, K, kGatedDgradBeside, kGatedDgradBeside + 2.0);
}

// Whether a gated block's 64 tiles, which then mostly have a group's rows in one, read its weights
// past the caches.  us through and past the caches, of weights that these do not hold from one call to the
// next: 64 experts 2048 x 1408, 48 rows 80 and 74, 1,536 rows 169 and 136; 8 of 4096 x 11008, 64 rows 242 and
// 215; 16 rows of one matrix of several by turns, 2 x 11008 x 4096 41.8 and 39.0, 2 x 13824 x 5120 57.8 and
// 54.5, 2 x 5504 x 2048 14.5 and 14.2.  The same matrix in every call, as in a model of less than 256 MB in all,
// would be there yet: 29.9 and 34.9, 48.1 and 52.1, 9.8 and 13.3; a call cannot tell.
inline bool gated_weights_once(const GroupArgs& g) { return g.rows <= 64 * int64_t(g.num); }

// (Weights that are read once: tiles of 64.  4,096 rows in 64 groups, 2048 to 2 x 1408, us: 163 in them
// and 176 one after the other; 2,048 rows 156 and 177.)
//
// h alone leaves little at a tile's end, so that it gains less from tiles one after the other: there a step
// counts as 0.78 us, and the tiles' ends as two bytes less than those of a whole product.  Fitted to 143
// shapes (209 to 65,536 rows, K 256 to 8192): for 4 the slower way is taken by 5 to 10%, for one by 17%; 0.6%
// is lost on average (1.9% counted as the others, 2.9% in tiles alone).  us one after the other, and in tiles:
// 8,192 rows, 4096 to 2 x 11008, 1,161 and 1,086; 5120 to 2 x 13824, 2,008 and 1,791; 32,768 rows in 16 groups,
// 2048 to 2 x 1408, 351 and 334, but 24,640 rows in 64 groups 320 and 344.
constexpr double kAloneStep = 0.78, kAloneBeside = -2.0, kAloneBytes = 2.0;
inline bool gated_linear_streams(const GroupArgs& g, int H, int K, bool keep) {
  if (gated_weights_once(g)) return false;
  return keep ? streams(g, 2 * H, K, 1.0, 3.0)
              : streams(g, 2 * H, K, kAloneBeside, kAloneBytes, kAloneStep);
}

// Makes them: launch(edge, share, workgroups), with *tiles_n set.
template <class Launch>
void launch_row_tiles(const GroupArgs& g, int N, int K, int weight, int32_t* tiles_n,
                      Launch&& launch, double beside = 0.0) {
  using std::integral_constant;
  const RowLaunch r = row_launch(g, N, K, weight, beside);
  *tiles_n = r.tiles_n;
  const integral_constant<Share, kAll> all;
  if (r.tile == 64) return launch(integral_constant<int, 64>{}, all, r.most);
  if (r.tile == 128) return launch(integral_constant<int, 128>{}, all, r.most);
  if (!r.split) return launch(integral_constant<int, 256>{}, all, r.most);
  launch(integral_constant<int, 256>{}, integral_constant<Share, kRounds>{}, r.most);
  launch(integral_constant<int, 128>{}, integral_constant<Share, kRest>{},
         std::min<int64_t>(4 * r.most, 512));
}

// Tile *v of group *e for workgroup w, of `num` groups with `per` tiles each.  Where a group has
// tiles enough, every XCD (workgroups w, w + 8, ... run on one) takes an eighth of each group's, so
// that groups of many rows keep all of them busy; false where its eighth is a tile shorter.  64
// experts 2048 x 1408 (176 tiles each), fp32, over two micro-batches of uneven load: with whole
// groups to an XCD 733 us, with eighths 672; one call of even load 201 and 218.  Four experts of 80 x
// 136 (2 tiles each) 15.3 and 19.0.
constexpr int kSharedTiles = 64;
__host__ __device__ constexpr int slots_of(int num, int per) {
  constexpr int kXcds = kNumXcd;
  return num == 1 || per < kSharedTiles ? per : (per + kXcds - 1) / kXcds * kXcds;
}
__host__ __device__ inline bool share_of(int w, int num, int per, int* v, int* e) {
  if (num == 1 || per < kSharedTiles) {
    const int at = xcd_order(w, num * per);
    *e = at / per;
    *v = at % per;
    return true;
  }
  constexpr int kXcds = kNumXcd;
  const int slots = slots_of(num, per) / kXcds, i = w / kXcds, at = i % slots;
  *e = i / slots;
  const int xcd = (w + *e) % kXcds, q = per / kXcds, r = per % kXcds;
  *v = xcd * q + (xcd < r ? xcd : r) + at;
  return at < q + (xcd < r ? 1 : 0);
}

// The tile edge of the gradients of M x N matrices.
inline int wgrad_tile(const GroupArgs& g, int M, int N) {
  // 256 tiles where experts have rows enough to outweigh what a tile takes beside its
  // steps, and tiles enough for the chip.  us in 128 and 256 tiles, bf16 and accumulating (all
  // through the caches; past them the first are 178, 714 and 931 as chosen): 64
  // experts 2048 x 1408 of 384 rows 269 and 282, 319 and 621; 8 of 4096 x 11008 of 1,024
  // rows 861 and 855, 980 and 1,543; one of 5120 x 13824 of 8,192 rows 1,524 and 951, 1,483 and
  // 1,096; one of 4096 x 4096 of 4,096 rows 130 and 109, 142 and 133.
  const int64_t tiles = int64_t(g.num) * ((M + 255) / 256) * ((N + 255) / 256);
  return g.rows / g.num >= 2048 && tiles >= 192 ? 256 : 128;
}

}  // namespace gnmr
