// K7: the INT8 low-cost path of a linear layer (Sec. 5.3, App. E.3) as a real 8-bit
// product instead of a simulated one:
//
//   inv_t = 127 / amax_t, q[t][i] = rint(x[t][i] * inv_t), sx_t = amax_t / 127
//   y[t][o] = bf16_rne( (sum_i q[t][i] c[o][i]) * (sx_t * sw_o) )
//
// with the weights held as codes c and a scale sw for each output channel.  The sum
// is a whole number below 2^31 (in_features < 2^17), so it is exact in any order.
#include "gnmr_internal.h"
#include "groups.h"
#include "lane_ops.h"
#include "mm_tile.h"

namespace gnmr {
namespace {

using mm::f32x4;
using mm::Int8;
using mm::u32x2;
using mm::u32x4;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

struct Eight {
  float v[8];
};
template <bool kF32>
__device__ __forceinline__ Eight eight(const void* row, int i) {
  Eight e;
  if constexpr (kF32) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(row) + i);
    const f32x4 b = *reinterpret_cast<const f32x4*>(static_cast<const float*>(row) + i + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      e.v[k] = a[k];
      e.v[4 + k] = b[k];
    }
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(row) + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      e.v[2 * k] = __uint_as_float(a[k] << 16);
      e.v[2 * k + 1] = __uint_as_float(a[k] & 0xFFFF0000u);
    }
  }
  return e;
}

// The bits of the largest magnitude: a NaN's are above infinity's.
__device__ __forceinline__ uint32_t largest(const Eight& e, uint32_t m) {
#pragma unroll
  for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(e.v[k]) & 0x7FFFFFFFu);
  return m;
}

// A row whose largest magnitude is below 2^-100 counts as zero (127 / amax has to be
// finite); one with an infinity or a NaN gets the scale NaN and codes 0, so that every
// output of it is NaN.
__device__ __forceinline__ void row_scale(uint32_t bits, float* inv, float* scale) {
  const float amax = __uint_as_float(bits);
  if (bits >= 0x7F800000u) {
    *inv = 0.0f;
    *scale = __uint_as_float(0x7FC00000u);
  } else {
    *inv = amax < 0x1p-100f ? 0.0f : 127.0f / amax;
    *scale = amax < 0x1p-100f ? 0.0f : amax / 127.0f;
  }
}

__device__ __forceinline__ u32x2 codes(const Eight& e, float inv) {
  uint32_t r[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int q = inv == 0.0f ? 0 : int(rintf(e.v[k] * inv));
    r[k >> 2] |= uint32_t(q & 0xFF) << (8 * (k & 3));
  }
  return u32x2{r[0], r[1]};
}

// One workgroup per row.
template <bool kF32>
__global__ __launch_bounds__(256) void k7_quantize(const QuantizeRows a) {
  __shared__ uint32_t red[4];
  const int64_t row = blockIdx.x;
  const void* x = static_cast<const char*>(a.x) + row * a.x_stride * (kF32 ? 4 : 2);
  uint32_t m = 0;
  for (int i = 8 * threadIdx.x; i < a.cols; i += 8 * 256) m = largest(eight<kF32>(x, i), m);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), d)));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(max(red[0], red[1]), max(red[2], red[3]));
  float inv, scale;
  row_scale(m, &inv, &scale);
  if (threadIdx.x == 0) a.scale[row] = scale;
  int8_t* q = a.codes + row * a.codes_stride;
  for (int i = 8 * threadIdx.x; i < a.cols; i += 8 * 256)
    *reinterpret_cast<u32x2*>(q + i) = codes(eight<kF32>(x, i), inv);
}

template <int kT>
__global__ __launch_bounds__(mm::kThreads, (mm::Depth<false, false, kT>::kPerCu)) void k7_linear(const QuantizedLinear a) {
  using D = mm::Depth<false, false, kT>;
  using T = mm::Tile<Int8, false, false, kT, kT, 2, D::kStep, D::kStages>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_row_tile<kT>(a.g, a.tiles_n, blockIdx.x, lane, &t)) return;
  const int n0 = t.tn * kT, e = t.group < a.g.num ? t.group : 0;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(a.q + int64_t(t.row) * a.q_stride, a.q_stride, t.rows, wave, lane);
  on.at(a.w + (int64_t(e) * a.N + n0) * a.K, a.K, a.N - n0, wave, lane);
  T::product(acc, om, on, t.group < a.g.num ? a.K : 0, wave, lane);
  const bool none = t.group >= a.g.num;
  const float* sw = a.w_scale + int64_t(e) * a.N + n0;
  const float* sx = a.q_scale + t.row;
  T::out16(
      acc, wave, lane,
      [&](int m, int n, int a0, int a1, int a2, int a3) {
        // rows and channels past the last ones read those: nothing of theirs is stored
        const float s = none ? 0.0f : sx[min(m, t.rows - 1)];
        const f32x4 w = *reinterpret_cast<const f32x4*>(sw + min(n, a.N - n0 - 4));
        return none ? u32x2{0, 0}
                    : u32x2{pack(float(a0) * (s * w[0]), float(a1) * (s * w[1])),
                            pack(float(a2) * (s * w[2]), float(a3) * (s * w[3]))};
      },
      [&](int m, int n, const u32x4& v) {
        if (m < t.rows && n0 + n < a.N)
          *reinterpret_cast<u32x4*>(a.y + int64_t(t.row + m) * a.y_stride + n0 + n) = v;
      });
}

}  // namespace

// Rows of codes in the workspace start 16-byte aligned.
int64_t quantized_codes_stride(int32_t in_features) { return (int64_t(in_features) + 15) / 16 * 16; }

int64_t quantized_linear_workgroups(const GroupArgs& g, int32_t out_features) {
  return most_row_tiles(g, 64) * ((out_features + 63) / 64);
}

hipError_t launch_quantize_rows(const QuantizeRows& a, bool f32, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (f32) hipLaunchKernelGGL(k7_quantize<true>, dim3(unsigned(a.rows)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k7_quantize<false>, dim3(unsigned(a.rows)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_quantized_linear(QuantizedLinear a, hipStream_t s) {
  auto launch = [&](auto edge) {
    constexpr int kT = decltype(edge)::value;
    a.tiles_n = (a.N + kT - 1) / kT;
    hipLaunchKernelGGL((k7_linear<kT>),
                       dim3(unsigned(most_row_tiles(a.g, kT) * a.tiles_n)), dim3(mm::kThreads), 0,
                       s, a);
  };
  const int tile = grouped_tile(a.g, a.N, a.K, 1);
  if (tile == 64) launch(std::integral_constant<int, 64>{});
  else if (tile == 128) launch(std::integral_constant<int, 128>{});
  else launch(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

}  // namespace gnmr
