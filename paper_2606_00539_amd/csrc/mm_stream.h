// Tiles of matrix products one after the other on the same compute unit: while a tile's results leave,
// the first two K steps of the next one are on their way, and what has been stored is not waited for
// before the next tile's second step.  (A workgroup for every tile pays for its start, its search for
// the tile, its first loads and the end of its stores; with one workgroup to a CU nothing covers them.)
//
// Tiles are 128 x 256, K steps 128 bytes, three of them in LDS (144 KB, one workgroup to a CU).  For a
// product, wavefronts of 64 x 128 have 1.5 times the LDS traffic of a 256 tile's and 0.75 times a 128
// tile's; groups of some hundred rows fill 128 high tiles better than 256 high ones.  The same with 256
// tiles, of two steps each in LDS, takes as long as a workgroup to a tile where groups are large (the
// chip's power bounds both), and longer where they are ragged: 24,576 rows in 64 groups, 2048 to 2 x
// 1408, us: 128 tiles 402, 256 tiles 409, 128 x 256 ones like this 360, 256 ones like this 462.
//
// What bounds them: where groups are many, weights that come from memory while two steps (96 KB a CU) are
// under way (as many rows in 64 groups take 302 us, in 8 groups 230, h alone); there is no LDS for more. A
// tile's results sent out piece by piece during the next one's first steps change nothing (317 and 316 us h
// alone; with the products the registers do not hold both).
#pragma once

#include "groups.h"
#include "mm_tile.h"

namespace gnmr {
namespace mm {

constexpr int kStreamWorkgroups = 256;

// The tiles of all groups in one order, found by ballots alone: the groups' boundaries are read
// once, those of the first 128 (a lane to a group, two sets) are kept.
class Tiles {
 public:
  __device__ __forceinline__ Tiles(const GroupArgs& groups, int tiles_n, int lane)
      : g(groups), per(tiles_n), lane_(lane) {
    if (g.offsets == nullptr) {
      total = group_wanted(g, 0) ? (g.rows + kStreamM - 1) / kStreamM * per : 0;
      return;
    }
    int sum = 0;
    for (int e0 = 0; e0 <= g.num; e0 += 64) {
      const Set s = read(e0, sum);
      if (e0 == 0) first = s;
      else if (e0 == 64) second = s;
      // (offsets in order leave no more tiles than this; others would let the sum overflow)
      sum = min(s.before + int(lane_of(uint32_t(s.upto), 63)), most());
    }
    total = sum * per;
  }

  // Tile v, 0 <= v < total.
  __device__ __forceinline__ RowTile at(int v) const {
    RowTile t{};
    int tm;
    if (g.offsets == nullptr) {
      walk<8>(v, total / per, per, &tm, &t.tn);
      t.row = tm * kStreamM;
      t.rows = g.rows - t.row;
      return t;
    }
    const int vm = v / per;
    int sum = 0;
    for (int e0 = 0; e0 <= g.num; e0 += 64) {
      const Set s = e0 == 0 ? first : e0 == 64 ? second : read(e0, sum);
      const int above = s.before + s.upto;
      const uint64_t here = __ballot(above - s.n <= vm && vm < above);
      if (here != 0) {
        const int src = __ffsll((unsigned long long)here) - 1;
        const int tiles_m = int(lane_of(uint32_t(s.n), src));
        const int start = (int(lane_of(uint32_t(above), src)) - tiles_m) * per;
        walk<8>(v - start, tiles_m, per, &tm, &t.tn);
        t.group = e0 + src;
        t.row = int(lane_of(uint32_t(s.begin), src)) + tm * kStreamM;
        t.rows = int(lane_of(uint32_t(s.end), src)) - t.row;
        return t;
      }
      sum = min(s.before + int(lane_of(uint32_t(s.upto), 63)), most());
    }
    return t;
  }

  int total;

 private:
  struct Set {
    int begin, end, n, upto, before;  // of this lane's group; tiles of the sets before
  };
  __device__ __forceinline__ Set read(int e0, int before) const {
    const int e = e0 + lane_;
    Set s{0, 0, 0, 0, before};
    if (e <= g.num && (e == g.num || group_wanted(g, e))) group_rows(g, e, &s.begin, &s.end);
    s.n = (s.end - s.begin + kStreamM - 1) / kStreamM;
    s.upto = int(wave_prefix(uint32_t(s.n)));
    return s;
  }

  __device__ __forceinline__ int most() const { return g.rows / kStreamM + g.num + 1; }

  const GroupArgs& g;
  int per, lane_;
  Set first{}, second{};
};

// 16 bytes to p + offset, or nowhere where `there` is false: the instruction is issued either way.
template <bool kPast>
__device__ __forceinline__ void store_if(void* p, bool there, uint32_t offset, const u32x4& v) {
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(p, 0, 0x7FFFFFFF, kBufferWord3);
  __builtin_amdgcn_raw_buffer_store_b128(v, r, there ? offset : 0x80000000u, 0, kPast ? 2 : 0);
}

// All tiles of a workgroup, K values each: whole steps, more than three.
//   place(tile, &om, &on) sets the operands of a tile; false: its products are 0
//   ahead(tile)           is called some steps before a tile's end
//   out(acc, tile, lds)   sends a tile's products out, through 12 KB of LDS for this wavefront, with
//                         exactly kStores vector memory stores and with loads that it has waited for
template <class T, int kStores, class Place, class Ahead, class Out>
__device__ __forceinline__ void stream(const GroupArgs& g, int tiles_n, int K, int wave, int lane,
                                       Place&& place, Ahead&& ahead, Out&& out) {
  static_assert(T::kSlots == 4 && T::kStages == 3, "three steps of 128 bytes");
  typedef typename T::Frag Frag;
  constexpr int kLoads = T::kLoads, kFirst = T::kFirst, kSecond = T::kSecond;
  // Memory operations end in order.  When a tile's second step has to have landed, there may be under
  // way: its third step, requested behind the stores, and the stores.
  constexpr int kWait = kLoads + kStores;
  static_assert(kWait < 64, "what the counter of memory operations holds");
  const Tiles tiles(g, tiles_n, lane);
  const int wg = blockIdx.x;
  // the workgroup's i-th tile: a round over the chip is consecutive tiles, an eighth to each XCD
  auto position = [&](int i) {
    const int left = tiles.total - i * kStreamWorkgroups;
    const int most = left < kStreamWorkgroups ? left : kStreamWorkgroups;
    return wg < most ? i * kStreamWorkgroups + xcd_order(wg, most) : -1;
  };
  int at = position(0);
  if (at < 0) return;
  const int nk = K / T::kStepK, padded = (nk + 2) / 3 * 3;

  typename T::Acc acc[T::kBM][T::kBN];
  typename T::ReadM rm;
  typename T::ReadN rn;
  rm.at((wave / T::kWN) * T::kWaveM, lane);
  rn.at((wave % T::kWN) * T::kWaveN, lane);
  Frag fm[2][T::kBM], fn[2][T::kBN];
  auto read = [&](int set, const char* st, int kk) {
#pragma unroll
    for (int b = 0; b < T::kBM; ++b) fm[set][b] = rm.get(st, kk, b);
#pragma unroll
    for (int b = 0; b < T::kBN; ++b) fn[set][b] = rn.get(st + T::OpM::kBytes, kk, b);
  };
  auto mfma = [&](int set) {
#pragma unroll
    for (int i = 0; i < T::kBM; ++i)
#pragma unroll
      for (int j = 0; j < T::kBN; ++j) acc[i][j] = T::mfma(fn[set][j], fm[set][i], acc[i][j]);
  };
  auto order = [](auto loads) {
    constexpr int kL = decltype(loads)::value, kMfma = T::kBM * T::kBN;
    constexpr int kPer = (kL + kMfma - 1) / kMfma;
#pragma unroll
    for (int i = 0; i < kMfma; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                          // MFMA
      if (i * T::kReadsEach < T::kReads)
        __builtin_amdgcn_sched_group_barrier(0x100, T::kReadsEach, 0);            // LDS read
      if (i * kPer < kL) __builtin_amdgcn_sched_group_barrier(0x020, kPer, 0);     // load
    }
  };
  using std::integral_constant;
  struct Operands {
    typename T::OpM m;
    typename T::OpN n;
    int steps;      // that are there: nk, or 0
  };
  Operands now, next;
  auto request = [&](const Operands& o, char* st, int s, int lo, int hi) {
    constexpr int kM = T::OpM::kLoads;
    if (lo < kM) o.m.request(st, s, s < o.steps, wave, lo, hi < kM ? hi : kM);
    if (hi > kM)
      o.n.request(st + T::OpM::kBytes, s, s < o.steps, wave, lo > kM ? lo - kM : 0, hi - kM);
  };

  RowTile tile = tiles.at(at);
  now.steps = place(tile, &now.m, &now.n) ? nk : 0;
  request(now, T::template stage<0>(), 0, 0, kLoads);
  request(now, T::template stage<1>(), 1, 0, kLoads);
  request(now, T::template stage<2>(), 2, 0, kFirst);
  // (both of the first steps: what the first wait inside allows for stores is then harmless)
  wait_loads<kFirst>();
  meet();
  read(0, T::template stage<0>(), 0);

  // Step s of a tile in stage u.  The steps behind a tile's last are the next one's first.
  auto one = [&](int s, auto u, auto is_first, auto is_last) {
    constexpr int U = decltype(u)::value;
    constexpr bool kFirstStep = decltype(is_first)::value && U == 0;
    constexpr bool kLastRound = decltype(is_last)::value, kLastStep = kLastRound && U == 2;
    char* const cur = T::template stage<U>();
    char* const nxt = T::template stage<(U + 1) % 3>();
    char* const old = T::template stage<(U + 2) % 3>();
    auto behind = [&](char* st, auto by, int lo, int hi) {   // parts of step s + by
      constexpr int kBy = decltype(by)::value;
      if constexpr (kLastRound && U + kBy >= 3) request(next, st, U + kBy - 3, lo, hi);
      else request(now, st, s + kBy, lo, hi);
    };
    const integral_constant<int, 2> ahead_two;
#pragma unroll
    for (int kk = 0; kk < 3; ++kk) {
      read((kk + 1) & 1, cur, kk + 1);
      if (kk == 0) behind(old, ahead_two, kFirst, kSecond);
      if (kk == 1) behind(old, ahead_two, kSecond, kLoads);
      mfma(kk & 1);
      if (kk == 0) order(integral_constant<int, kSecond - kFirst>{});
      else if (kk == 1) order(integral_constant<int, kLoads - kSecond>{});
      else order(integral_constant<int, 0>{});
    }
    __builtin_amdgcn_sched_barrier(0);
    // step s + 1 has landed; what is behind it, and at first what the tile before stored, need not
    if constexpr (kFirstStep) wait_loads<kWait>();
    else wait_loads<kLoads>();
    meet();
    __builtin_amdgcn_sched_barrier(0);
    // (at a tile's end the stage is needed for its results first)
    if constexpr (!kLastStep) behind(cur, integral_constant<int, 3>{}, 0, kFirst);
    read(0, nxt, 0);
    mfma(1);
    order(integral_constant<int, kLastStep ? 0 : kFirst>{});
  };
  auto round = [&](int s, auto is_first, auto is_last) {
    one(s, integral_constant<int, 0>{}, is_first, is_last);
    one(s + 1, integral_constant<int, 1>{}, is_first, is_last);
    one(s + 2, integral_constant<int, 2>{}, is_first, is_last);
  };
  const std::true_type yes;
  const std::false_type no;
#pragma unroll 1
  for (int i = 1;; ++i) {
#pragma unroll
    for (int m = 0; m < T::kBM; ++m)
#pragma unroll
      for (int n = 0; n < T::kBN; ++n) acc[m][n] = typename T::Acc{};
    const int then = position(i);
    RowTile coming{};
    next.steps = 0;
    if (then >= 0) {
      coming = tiles.at(then);
      next.steps = place(coming, &next.m, &next.n) ? nk : 0;
    } else {
      next.m = now.m;
      next.n = now.n;
    }
    round(0, yes, no);
#pragma unroll 1
    for (int s = 3; s < padded - 3; s += 3) round(s, no, no);
    ahead(tile);
    round(padded - 3, no, yes);
    out(acc, tile, T::template stage<2>() + wave * (T::kStage / kWaves));
    if (then < 0) break;
    meet();     // all have read their results
    tile = coming;
    now = next;
    request(now, T::template stage<2>(), 2, 0, kFirst);
  }
  wait_loads<0>();  // requests behind the last step still write to LDS
}

}  // namespace mm
}  // namespace gnmr
