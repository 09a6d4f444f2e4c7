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
using mm::u32x2;
using mm::u32x4;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

// linear (kDgrad false) and dgrad: out[t][n] = sum_k in[t][k] * W_e(n, k).
template <bool kDgrad, int kTM, int kTN, int kWM, int kStages, int kPerCu>
__global__ __launch_bounds__(mm::kThreads, kPerCu) void k6_rows(const GroupedRows a) {
  using T = mm::Tile<Bf16, false, kDgrad, kTM, kTN, kWM, kStages>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_row_tile<kTM>(a.g, a.tiles_n, blockIdx.x, lane, &t)) return;
  const int n0 = t.tn * kTN;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(a.in + int64_t(t.row) * a.in_stride, a.in_stride * 2, t.rows, wave, lane);
  const uint16_t* w = a.w + (t.group < a.g.num ? int64_t(t.group) * a.N * a.K : 0);
  on.at(kDgrad ? w + n0 : w + int64_t(n0) * a.K, int64_t(kDgrad ? a.N : a.K) * 2, a.N - n0, wave,
        lane);
  T::product(acc, om, on, t.group < a.g.num ? a.K : 0, wave, lane);
  T::each(wave, lane, [&](int i, int j, int g, int m, int n) {
    if (m < t.rows && n0 + n < a.N) {
      const auto& c = acc[i][j];
      *reinterpret_cast<u32x2*>(a.out + int64_t(t.row + m) * a.out_stride + n0 + n) =
          u32x2{pack(c[4 * g], c[4 * g + 1]), pack(c[4 * g + 2], c[4 * g + 3])};
    }
  });
}

template <bool kF32, bool kAcc, int kT, int kStages, int kPerCu>
__global__ __launch_bounds__(mm::kThreads, kPerCu) void k6_wgrad(const GroupedWgrad a) {
  using T = mm::Tile<Bf16, true, true, kT, kT, 2, kStages>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = a.tiles_m * a.tiles_n, v = xcd_order(blockIdx.x, a.g.num * per);
  const int e = v / per;
  if (!group_wanted(a.g, e)) return;
  int tm, tn, begin, end;
  walk<8>(v % per, a.tiles_m, a.tiles_n, &tm, &tn);
  group_rows(a.g, e, &begin, &end);
  const int m0 = tm * kT, n0 = tn * kT;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(a.dy + int64_t(begin) * a.dy_stride + m0, a.dy_stride * 2, a.M - m0, wave, lane);
  on.at(a.x + int64_t(begin) * a.x_stride + n0, a.x_stride * 2, a.N - n0, wave, lane);
  T::product(acc, om, on, end - begin, wave, lane);
  float ss = 0.0f;
  const int64_t base = int64_t(e) * a.M * a.N;
  T::each(wave, lane, [&](int i, int j, int g, int m, int n) {
    if (m0 + m < a.M && n0 + n < a.N) {
      const auto& c = acc[i][j];
      const int64_t at = base + int64_t(m0 + m) * a.N + n0 + n;
      float q[4] = {c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
      if constexpr (kF32) {
        f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(a.dw) + at);
        if constexpr (kAcc) {
          const f32x4 old = *p;
#pragma unroll
          for (int k = 0; k < 4; ++k) q[k] += old[k];
        }
        *p = f32x4{q[0], q[1], q[2], q[3]};
      } else {
        u32x2* p = reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.dw) + at);
        if constexpr (kAcc) {
          const u32x2 old = *p;
          q[0] += low(old.x);
          q[1] += high(old.x);
          q[2] += low(old.y);
          q[3] += high(old.y);
        }
        const u32x2 r{pack(q[0], q[1]), pack(q[2], q[3])};
        *p = r;
        q[0] = low(r.x);
        q[1] = high(r.x);
        q[2] = low(r.y);
        q[3] = high(r.y);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) ss = fmaf(q[k], q[k], ss);
    }
  });
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

template <bool kDgrad, int kTM, int kTN, int kWM, int kStages, int kPerCu>
void launch_rows(GroupedRows a, hipStream_t s) {
  a.tiles_n = (a.N + kTN - 1) / kTN;
  const int64_t wgs = most_row_tiles(a.g, kTM) * a.tiles_n;
  hipLaunchKernelGGL((k6_rows<kDgrad, kTM, kTN, kWM, kStages, kPerCu>), dim3(unsigned(wgs)),
                     dim3(mm::kThreads), 0, s, a);
}

template <bool kF32, bool kAcc>
void launch_wgrad_of(GroupedWgrad a, hipStream_t s) {
  constexpr int kT = 128;
  a.tiles_m = (a.M + kT - 1) / kT;
  a.tiles_n = (a.N + kT - 1) / kT;
  hipLaunchKernelGGL((k6_wgrad<kF32, kAcc, kT, 2, 2>),
                     dim3(unsigned(int64_t(a.g.num) * a.tiles_m * a.tiles_n)), dim3(mm::kThreads),
                     0, s, a);
}

}  // namespace

int64_t grouped_rows_workgroups(const GroupedRows& a) {
  return most_row_tiles(a.g, 128) * ((a.N + 127) / 128);
}

hipError_t launch_grouped_rows(const GroupedRows& a, bool dgrad, hipStream_t s) {
  if (dgrad) launch_rows<true, 128, 128, 2, 2, 2>(a, s);
  else launch_rows<false, 128, 128, 2, 2, 2>(a, s);
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
