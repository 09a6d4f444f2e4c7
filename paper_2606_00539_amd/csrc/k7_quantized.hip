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
using mm::i32x4;
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

// kLanes lanes to a row: a wavefront (rows of up to 2,048 values, four to a workgroup) or the
// workgroup.  The second pass over a row meets it in the L1 or L2.
template <bool kF32, int kLanes>
__global__ __launch_bounds__(256) void k7_quantize(const QuantizeRows a) {
  __shared__ uint32_t red[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x % kLanes;
  const int64_t row = int64_t(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
  if (kLanes == 64 && row >= a.rows) return;
  const void* x = static_cast<const char*>(a.x) + row * a.x_stride * (kF32 ? 4 : 2);
  uint32_t m = 0;
#pragma unroll 4
  for (int i = 8 * lane; i < a.cols; i += 8 * kLanes) m = largest(eight<kF32>(x, i), m);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), d)));
  if constexpr (kLanes == 256) {
    if ((threadIdx.x & 63) == 0) red[wave] = m;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
  }
  float inv, scale;
  row_scale(m, &inv, &scale);
  if (lane == 0) a.scale[row] = scale;
  int8_t* q = a.codes + row * a.codes_stride;
#pragma unroll 4
  for (int i = 8 * lane; i < a.cols; i += 8 * kLanes)
    *reinterpret_cast<u32x2*>(q + i) = codes(eight<kF32>(x, i), inv);
}

// One row (a decoding step of one sequence), quantised on the way: a workgroup forms its
// codes in LDS, reading it from the L2 (10 KiB at 5,120 features), while its first weights
// are on their way; then its wavefronts take kChannels output channels each, a lane 16 bytes of
// each channel at a time, four products to an instruction.  The weights' bytes bound it: 5,120 to
// 13,824 features 14.3 us (5 TB/s), in tiles of 64 behind a launch for the codes 16.9; 13,824 to
// 5,120 16.5 and 26.6.  (Two and four rows took 18.3 and 24.5 so, 17.2 in tiles.)
constexpr int kChannels = 4, kAhead = 2;  // chunks of each channel on their way at a time

__device__ __forceinline__ int dot16(const i32x4& a, const i32x4& b, int c) {
#pragma unroll
  for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_sdot4(a[k], b[k], c, false);
  return c;
}

// 16 weights from p, of which `left` exist (a multiple of 8)
__device__ __forceinline__ i32x4 weights16(const int8_t* p, int left) {
  if (left >= 16) return *reinterpret_cast<const i32x4*>(p);
  if (left <= 0) return i32x4{0, 0, 0, 0};
  const u32x2 h = *reinterpret_cast<const u32x2*>(p);
  return i32x4{int(h.x), int(h.y), 0, 0};
}

__global__ __launch_bounds__(256) void k7_token(const QuantizedToken a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];  // the row, then its codes
  __shared__ uint32_t red[4];
  if (a.mask != nullptr && int(a.mask[0] != 0) != a.mask_value) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n0 = (blockIdx.x * 4 + wave) * kChannels;
  const int chunks = (a.K + 15) / 16;
  auto fetch = [&](i32x4 (&w)[kAhead][kChannels], int j0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int c = 0; c < kChannels; ++c) {
        const int j = j0 + 64 * k, n = min(n0 + c, a.N - 1);
        w[k][c] = weights16(a.w + int64_t(n) * a.K + 16 * j, a.K - 16 * j);
      }
  };
  i32x4 next[kAhead][kChannels];
  fetch(next, lane);
  u32x4* const row = reinterpret_cast<u32x4*>(lds);
  char* const q = lds + 32 * chunks;
  uint32_t m = 0;
  for (int i = tid; i < 2 * chunks; i += 256) {
    const u32x4 v = 8 * i < a.K ? reinterpret_cast<const u32x4*>(a.x)[i] : u32x4{0, 0, 0, 0};
    row[i] = v;
    m = largest(eight<false>(&v, 0), m);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), d)));
  if (lane == 0) red[wave] = m;
  __syncthreads();
  float inv, sx;
  row_scale(max(max(red[0], red[1]), max(red[2], red[3])), &inv, &sx);
  for (int i = tid; i < 2 * chunks; i += 256)
    *reinterpret_cast<u32x2*>(q + 8 * i) = codes(eight<false>(row + i, 0), inv);
  __syncthreads();
  int acc[kChannels] = {};
  for (int j0 = lane; j0 < chunks; j0 += 64 * kAhead) {
    i32x4 w[kAhead][kChannels];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int c = 0; c < kChannels; ++c) w[k][c] = next[k][c];
    fetch(next, j0 + 64 * kAhead);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      // (weights past the last chunk are zero: any code does)
      const i32x4 x = *reinterpret_cast<const i32x4*>(q + 16 * min(j0 + 64 * k, chunks - 1));
#pragma unroll
      for (int c = 0; c < kChannels; ++c) acc[c] = dot16(x, w[k][c], acc[c]);
    }
  }
#pragma unroll
  for (int c = 0; c < kChannels; ++c)
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) acc[c] += __shfl_xor(acc[c], d);
  if (lane == 0 && n0 < a.N) {  // (N is a multiple of 8: all kChannels exist)
    float v[kChannels];
#pragma unroll
    for (int c = 0; c < kChannels; ++c) v[c] = float(acc[c]) * (sx * a.w_scale[n0 + c]);
    *reinterpret_cast<u32x2*>(a.y + n0) = u32x2{pack(v[0], v[1]), pack(v[2], v[3])};
  }
}

template <int kT, Share kShare>
__global__ __launch_bounds__(mm::kThreads, (mm::Depth<false, false, kT>::kPerCu)) void k7_linear(const QuantizedLinear a) {
  using D = mm::Depth<false, false, kT>;
  using T = mm::Tile<Int8, false, false, kT, kT, 2, D::kStep, D::kStages>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_row_tile<kT, kShare>(a.g, a.tiles_n, blockIdx.x, lane, &t)) return;
  const int n0 = t.tn * kT, e = t.group < a.g.num ? t.group : 0;
  if (kShare == kRest && n0 >= a.N) return;
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
          put(reinterpret_cast<u32x4*>(a.y + int64_t(t.row + m) * a.y_stride + n0 + n), v, a.past);
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
  if (a.cols <= 2048) {
    const dim3 wgs(unsigned((int64_t(a.rows) + 3) / 4));
    if (f32) hipLaunchKernelGGL((k7_quantize<true, 64>), wgs, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k7_quantize<false, 64>), wgs, dim3(256), 0, s, a);
  } else {
    const dim3 wgs(unsigned(a.rows));
    if (f32) hipLaunchKernelGGL((k7_quantize<true, 256>), wgs, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k7_quantize<false, 256>), wgs, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

bool quantized_token(const GroupArgs& g, int32_t in_features) {
  // row and codes take three bytes a feature of the LDS
  return g.offsets == nullptr && g.rows == 1 && in_features <= 16384;
}

hipError_t launch_quantized_token(const QuantizedToken& a, hipStream_t s) {
  hipLaunchKernelGGL(k7_token, dim3(unsigned((a.N + 4 * kChannels - 1) / (4 * kChannels))),
                     dim3(256), size_t(48) * ((a.K + 15) / 16), s, a);
  return hipGetLastError();
}

hipError_t launch_quantized_linear(QuantizedLinear a, hipStream_t s) {
  a.past = past_caches(a.g.rows, a.N);
  auto launch = [&](auto edge, auto share, int64_t wgs) {
    hipLaunchKernelGGL((k7_linear<decltype(edge)::value, decltype(share)::value>),
                       dim3(unsigned(wgs)), dim3(mm::kThreads), 0, s, a);
  };
  launch_row_tiles(a.g, a.N, a.K, 1, &a.tiles_n, launch);
  return hipGetLastError();
}

}  // namespace gnmr
