// K6: the products of a mixture-of-experts linear layer.  Rows (tokens) lie sorted
// by expert, expert e's in [offsets[e], offsets[e+1]):
//
//   linear   y[t][o]  = sum_i x[t][i]  W_e[o][i]
//   dgrad    dx[t][i] = sum_o dy[t][o] W_e[o][i]
//   wgrad    dW_e[o][i] (+)= sum over e's rows t of dy[t][o] x[t][i], with the sums of
//            squares of dW_e over 128 x 128 blocks, of which the controller forms
//            the expert's norm (Sec. 2; Alg. 1) without reading dW_e again
//
// bf16 operands, fp32 accumulation, one rounding to bf16 (or none: fp32 dW).
#include <type_traits>

#include "gnmr_internal.h"
#include "groups.h"
#include "lane_ops.h"
#include "mm_tile.h"

namespace gnmr {
namespace {

using mm::Bf16;
using mm::f32x4;
using mm::u32x2;
using mm::u32x4;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// linear (kDgrad false) and dgrad: out[t][n] = sum_k in[t][k] * W_e(n, k).
template <bool kDgrad, int kT, Share kShare>
__global__ __launch_bounds__(mm::kThreads, (mm::Depth<false, kDgrad, kT>::kPerCu)) void k6_rows(const GroupedRows a) {
  using D = mm::Depth<false, kDgrad, kT>;
  using T = mm::Tile<Bf16, false, kDgrad, kT, kT, 2, D::kStep, D::kStages>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_row_tile<kT, kShare>(a.g, a.tiles_n, blockIdx.x, lane, &t)) return;
  const int n0 = t.tn * kT;
  if (kShare == kRest && n0 >= a.N) return;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(a.in + int64_t(t.row) * a.in_stride, a.in_stride * 2, t.rows, wave, lane);
  const uint16_t* w = a.w + (t.group < a.g.num ? int64_t(t.group) * a.N * a.K : 0);
  on.at(kDgrad ? w + n0 : w + int64_t(n0) * a.K, int64_t(kDgrad ? a.N : a.K) * 2, a.N - n0, wave,
        lane);
  T::product(acc, om, on, t.group < a.g.num ? a.K : 0, wave, lane);
  T::out16(
      acc, wave, lane,
      [](int, int, float a0, float a1, float a2, float a3) {
        return u32x2{pack(a0, a1), pack(a2, a3)};
      },
      [&](int m, int n, const u32x4& v) {
        if (m < t.rows && n0 + n < a.N)
          put(reinterpret_cast<u32x4*>(a.out + int64_t(t.row + m) * a.out_stride + n0 + n), v, a.past);
      });
}

// The 128 tile's three stages leave room for three workgroups on a CU; where it holds fp32 values
// to add to, their registers allow two, and there is room for four stages.  64 experts 2048 x
// 1408, 24,576 rows, three and two on a CU (all through the caches): bf16 269 and 289 us, accumulating 319 and 347, fp32
// 334 and 365, accumulating 536 and 431.
template <bool kF32, bool kAcc, int kT>
struct WgradTile {
  static constexpr int kPerCu = kT == 256 ? 1 : kAcc ? 2 : 3;
  using T = mm::Tile<Bf16, true, true, kT, kT, 2, 64, kPerCu == 3 ? 3 : 4>;
};

template <bool kF32, bool kAcc, int kT>
__global__ __launch_bounds__(mm::kThreads, (WgradTile<kF32, kAcc, kT>::kPerCu)) void k6_wgrad(
    const GroupedWgrad a) {
  using T = typename WgradTile<kF32, kAcc, kT>::T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int v, e;
  if (!share_of(blockIdx.x, a.g.num, a.tiles_m * a.tiles_n, &v, &e) || !group_wanted(a.g, e)) return;
  int tm, tn, begin, end;
  walk<8>(v, a.tiles_m, a.tiles_n, &tm, &tn);
  group_rows(a.g, e, &begin, &end);
  const int m0 = tm * kT, n0 = tn * kT;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(a.dy + int64_t(begin) * a.dy_stride + m0, a.dy_stride * 2, a.M - m0, wave, lane);
  on.at(a.x + int64_t(begin) * a.x_stride + n0, a.x_stride * 2, a.N - n0, wave, lane);
  const int64_t base = (int64_t(e) * a.M + m0) * a.N + n0;
  // Accumulating in 128 tiles, the stored values are on their way while the product runs
  // (a 256 tile has no registers for them).
  typedef typename std::conditional<kF32, f32x4, u32x2>::type Old;
  constexpr bool kEarly = kAcc && kT == 128;
  Old old[kEarly ? T::kPieces : 1];
  const int col = T::col(wave, lane);
  auto there = [&](int row) { return m0 + row < a.M && n0 + col < a.N; };
  // (rows and columns past the last ones read those)
  const int last = a.M - 1 - m0, edge = min(col, a.N - n0 - 4);
  auto stored = [&](int row) {
    return static_cast<char*>(a.dw) + (base + int64_t(min(row, last)) * a.N + edge) * (kF32 ? 4 : 2);
  };
  if constexpr (kEarly) {
#pragma unroll
    for (int q = 0; q < T::kPieces; ++q) {
      old[q] = *reinterpret_cast<const Old*>(stored(T::row(q, wave, lane)));
    }
  }
  T::product(acc, om, on, end - begin, wave, lane);
  float ss = 0.0f;
  auto square = [&](float q) { ss = fmaf(q, q, ss); };
  if constexpr (!kF32 && !kAcc) {
    T::out16(
        acc, wave, lane,
        [](int, int, float a0, float a1, float a2, float a3) {
          return u32x2{pack(a0, a1), pack(a2, a3)};
        },
        // Gradients that nothing was added to go past the caches: what they would drive out is dy and
        // x.  64 and 24 experts 2048 x 1408 of 384 rows, us through and past them: fp32 313 and 201, 110
        // and 74, bf16 227 and 163, 67 and 65; with a pass that reads the gradient behind it fp32 554
        // and 522.  (Experts of a row or two are up to 13%
        // slower so.)  Accumulated ones do not gain.
        [&](int m, int n, const u32x4& v) {
          if (m0 + m < a.M && n0 + n < a.N) {
            __builtin_nontemporal_store(
                v, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.dw) + base + int64_t(m) * a.N + n));
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              square(low(v[k]));
              square(high(v[k]));
            }
          }
        });
  } else {
    T::out32(
        acc, wave, lane,
        [&](int q) {
          if constexpr (kAcc && !kEarly)
            return *reinterpret_cast<const Old*>(stored(T::row(q, wave, lane)));
          else return Old{};
        },
        [&](int q, f32x4 v, Old was) {
          const int row = T::row(q, wave, lane);
          if (!there(row)) return;
          Old* p = reinterpret_cast<Old*>(stored(row));
          if constexpr (kEarly) was = old[q];
          if constexpr (kF32) {
            if constexpr (kAcc) v += was;
            if constexpr (kAcc) *p = v;
            else __builtin_nontemporal_store(v, p);
          } else {
            const u32x2 r{pack(v[0] + low(was.x), v[1] + high(was.x)),
                          pack(v[2] + low(was.y), v[3] + high(was.y))};
            *p = r;
            v = f32x4{low(r.x), high(r.x), low(r.y), high(r.y)};
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) square(v[k]);
        });
  }
  ss = wave_sum(ss);
  const int blocks_n = (a.N + kGroupedBlock - 1) / kGroupedBlock;
  const int64_t blocks = int64_t((a.M + kGroupedBlock - 1) / kGroupedBlock) * blocks_n;
  if constexpr (kT == 256) {
    const int bm = 2 * tm + (wave >> 1), bn = 2 * tn + (wave & 1);
    if (lane == 0 && bm * kGroupedBlock < a.M && bn < blocks_n)
      a.partials[e * blocks + int64_t(bm) * blocks_n + bn] = ss;
  } else {
    __shared__ float red[mm::kWaves];
    if (lane == 0) red[wave] = ss;
    __syncthreads();
    if (threadIdx.x == 0)
      a.partials[e * blocks + int64_t(tm) * blocks_n + tn] = ((red[0] + red[1]) + red[2]) + red[3];
  }
}

template <bool kDgrad>
void launch_rows(GroupedRows a, hipStream_t s) {
  a.past = past_caches(a.g.rows, a.N);
  auto launch = [&](auto edge, auto share, int64_t wgs) {
    hipLaunchKernelGGL((k6_rows<kDgrad, decltype(edge)::value, decltype(share)::value>),
                       dim3(unsigned(wgs)), dim3(mm::kThreads), 0, s, a);
  };
  launch_row_tiles(a.g, a.N, a.K, 2, &a.tiles_n, launch);
}

template <bool kF32, bool kAcc>
void launch_wgrad_of(GroupedWgrad a, hipStream_t s) {
  auto launch = [&](auto edge) {
    constexpr int kT = decltype(edge)::value;
    a.tiles_m = (a.M + kT - 1) / kT;
    a.tiles_n = (a.N + kT - 1) / kT;
    hipLaunchKernelGGL((k6_wgrad<kF32, kAcc, kT>),
                       dim3(unsigned(int64_t(a.g.num) * slots_of(a.g.num, a.tiles_m * a.tiles_n))),
                       dim3(mm::kThreads), 0, s, a);
  };
  if (wgrad_tile(a.g, a.M, a.N) == 256) launch(std::integral_constant<int, 256>{});
  else launch(std::integral_constant<int, 128>{});
}

}  // namespace

int64_t grouped_rows_workgroups(const GroupedRows& a) {
  return most_row_tiles(a.g, 64) * ((a.N + 63) / 64);
}

hipError_t launch_grouped_rows(const GroupedRows& a, bool dgrad, hipStream_t s) {
  if (dgrad) launch_rows<true>(a, s);
  else launch_rows<false>(a, s);
  return hipGetLastError();
}

hipError_t launch_grouped_wgrad(const GroupedWgrad& a, bool f32, bool accumulate, hipStream_t s) {
  if (f32 && accumulate) launch_wgrad_of<true, true>(a, s);
  else if (f32) launch_wgrad_of<true, false>(a, s);
  else if (accumulate) launch_wgrad_of<false, true>(a, s);
  else launch_wgrad_of<false, false>(a, s);
  return hipGetLastError();
}

}  // namespace gnmr
