// K10: layer norm of rows and its gradients, in fp32:
//
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), y = (x - m) r w + b
//   g = dy w, z = (x - m) r:  dx = r (g - mean(g) - z mean(g z)),
//   dw = sum over rows of dy z,  db = sum over rows of dy
//
// A row is held in registers by 8 to 64 lanes, or by a workgroup: it is read once.  Its mean
// is first taken in fp32 and then corrected by the mean of what is left, since where the mean is
// much larger than the deviations its rounding alone would show in x - m; the gradients' kernel does
// the same with the mean that it is given.
#include "gnmr_internal.h"
#include "lane_ops.h"
#include "values.h"

namespace gnmr {
namespace {

constexpr int kThreads = 256;

// Sums of N values over the kLanes lanes of a row, in each of them; kLanes = kThreads is the
// workgroup.  `red` is that row's memory, used by every second sum: between two uses of it lies a
// barrier of the other's.
template <int kLanes, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[4]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float s = v[n];
    if constexpr (kLanes >= 64) s = add_other<32>(s);
    if constexpr (kLanes >= 32) s = add_other<16>(s);
    if constexpr (kLanes >= 16) {
      s = add_other<8>(s);
      s = add_other<4>(s);
    } else {
      // eight lanes, mirrored: the quads then hold the same four sums
      s += __uint_as_float(uint32_t(
          __builtin_amdgcn_update_dpp(0, int(__float_as_uint(s)), 0x141, 0xF, 0xF, false)));
    }
    s = add_other<2>(s);
    v[n] = add_other<1>(s);
  }
  if constexpr (kLanes > 64) {
    static_assert(kLanes == kThreads, "lanes of a wavefront or a workgroup");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (lane == 0) red[n][wave] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = (red[n][0] + red[n][1]) + (red[n][2] + red[n][3]);
  }
}

// eight weights, of either type
__device__ __forceinline__ Eight weights(const void* w, bool f32, int col, int count) {
  return f32 ? load_some<true>(w, col, count) : load_some<false>(w, col, count);
}

template <bool kF32, int kLanes, int kVec>
__global__ __launch_bounds__(kThreads) void k10_forward(const LayerNorm a) {
  __shared__ float red[2][2][4];
  const int at = threadIdx.x % kLanes;
  const int64_t row = int64_t(blockIdx.x) * (kThreads / kLanes) + threadIdx.x / kLanes;
  const bool there = row < a.rows;    // (of a workgroup's row the same for all)
  const char* x = static_cast<const char*>(a.x) + (there ? row : 0) * a.x_stride * (kF32 ? 4 : 2);
  Eight v[kVec];
  float s[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int col = 8 * (at + i * kLanes);
    v[i] = load_some<kF32>(x, col, there ? a.cols - col : 0);
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) s[0] += v[i].v[k];
  row_sums<kLanes, 1>(s, red[0]);
  const float n = float(a.cols), mean = s[0] / n;
  float d[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kVec; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[i].v[k] = 8 * (at + i * kLanes) + k < a.cols ? v[i].v[k] - mean : 0.0f;
      d[0] += v[i].v[k];
      d[1] = fmaf(v[i].v[k], v[i].v[k], d[1]);
    }
  row_sums<kLanes, 2>(d, red[1]);
  const float left = d[0] / n, var = d[1] / n - left * left;
  const float rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + a.eps);
  if (!there) return;
  if (at == 0) {
    if (a.mean != nullptr) a.mean[row] = mean + left;
    if (a.rstd != nullptr) a.rstd[row] = rstd;
  }
  char* y = static_cast<char*>(a.y) + row * a.y_stride * (kF32 ? 4 : 2);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int col = 8 * (at + i * kLanes), count = a.cols - col;
    if (count <= 0) continue;
    Eight w, b;
    if (a.weight != nullptr) w = weights(a.weight, a.weight_f32, col, count);
    if (a.bias != nullptr) b = weights(a.bias, a.weight_f32, col, count);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float z = (v[i].v[k] - left) * rstd;
      if (a.weight != nullptr) z *= w.v[k];
      if (a.bias != nullptr) z += b.v[k];
      v[i].v[k] = z;
    }
    store_some<kF32>(y, col, count, v[i]);
  }
}

// Workgroups take rows by turns and keep their columns' sums over them in registers; what each
// has in the end goes to `parts`, [workgroup][dw, db][cols].
template <bool kF32, int kLanes, int kVec>
__global__ __launch_bounds__(kThreads) void k10_backward(const LayerNormBackward a) {
  constexpr int kSlots = kThreads / kLanes;
  __shared__ float red[2][3][4];
  __shared__ float sums[kSlots > 1 ? kSlots * kLanes * 8 : 1];
  const int at = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  const float n = float(a.cols);
  Eight w[kVec], dw[kVec], db[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int col = 8 * (at + i * kLanes);
    if (a.weight != nullptr) w[i] = weights(a.weight, a.weight_f32, col, a.cols - col);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      dw[i].v[k] = db[i].v[k] = 0.0f;
      if (a.weight == nullptr) w[i].v[k] = 1.0f;
    }
  }
  int turn = 0;
  for (int64_t first = int64_t(blockIdx.x) * kSlots; first < a.rows;
       first += int64_t(gridDim.x) * kSlots) {
    const int64_t row = first + slot;
    const bool there = row < a.rows;
    const int64_t r = there ? row : first;
    const char* x = static_cast<const char*>(a.x) + r * a.x_stride * (kF32 ? 4 : 2);
    const char* dy = static_cast<const char*>(a.dy) + r * a.dy_stride * (kF32 ? 4 : 2);
    const float mean = a.mean[r], rstd = a.rstd[r];
    Eight v[kVec], g[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int col = 8 * (at + i * kLanes), count = there ? a.cols - col : 0;
      v[i] = load_some<kF32>(x, col, count);
      g[i] = load_some<kF32>(dy, col, count);
    }
    float s[3] = {0.0f, 0.0f, 0.0f};    // of x - mean, g, g (x - mean)
#pragma unroll
    for (int i = 0; i < kVec; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float d = 8 * (at + i * kLanes) + k < a.cols ? v[i].v[k] - mean : 0.0f;
        const float q = g[i].v[k] * w[i].v[k];
        v[i].v[k] = d;
        s[0] += d;
        s[1] += q;
        s[2] = fmaf(q, d, s[2]);
      }
    row_sums<kLanes, 3>(s, red[turn]);
    turn ^= 1;
    if (!there) continue;
    const float left = s[0] / n, g1 = s[1] / n, gz = rstd * (s[2] / n - left * g1);
    char* dx = static_cast<char*>(a.dx) + row * a.dx_stride * (kF32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int col = 8 * (at + i * kLanes), count = a.cols - col;
      if (count <= 0) continue;
      Eight out;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float z = (v[i].v[k] - left) * rstd, q = g[i].v[k];
        out.v[k] = rstd * (q * w[i].v[k] - g1 - z * gz);
        dw[i].v[k] = fmaf(q, z, dw[i].v[k]);
        db[i].v[k] += q;
      }
      if (a.dx != nullptr) store_some<kF32>(dx, col, count, out);
    }
  }
  if (a.parts == nullptr) return;
  float* to = a.parts + int64_t(blockIdx.x) * 2 * a.cols;
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      Eight e = which == 0 ? dw[i] : db[i];
      const int col = 8 * (at + i * kLanes), count = a.cols - col;
      if constexpr (kSlots > 1) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) sums[(slot * 8 + k) * kLanes + at] = e.v[k];
        __syncthreads();
        if (slot == 0) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            e.v[k] = 0.0f;
#pragma unroll
            for (int q = 0; q < kSlots; ++q) e.v[k] += sums[(q * 8 + k) * kLanes + at];
          }
        }
      }
      if (slot == 0 && count > 0) store_some<true>(to + which * a.cols, col, count, e);
    }
}

// dw and db from the workgroups' sums: 64 columns to a workgroup, whose wavefronts take a
// share of the sums each, in order.
__global__ __launch_bounds__(kThreads) void k10_reduce(const LayerNormBackward a) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (a.cols + 63) / 64, which = blockIdx.x / blocks;
  void* out = which == 0 ? a.dweight : a.dbias;
  if (out == nullptr) return;
  const int col = (blockIdx.x % blocks) * 64 + lane;
  const int share = (a.num_parts + 3) / 4, lo = wave * share, hi = min(lo + share, a.num_parts);
  float s = 0.0f;
  if (col < a.cols) {
    const float* p = a.parts + which * a.cols + col;
#pragma unroll 8
    for (int k = lo; k < hi; ++k) s += p[int64_t(k) * 2 * a.cols];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || col >= a.cols) return;
  s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
  if (a.weight_f32) store_one<true>(out, col, s);
  else store_one<false>(out, col, s);
}

// launch(lanes, vectors): who holds a row of that many columns.
template <class Launch>
void by_width(int cols, Launch&& launch) {
  using std::integral_constant;
  auto of = [&](auto lanes, auto vec) { launch(lanes, vec); };
  if (cols <= 64) return of(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  if (cols <= 128) return of(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (cols <= 256) return of(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (cols <= 512) return of(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (cols <= 1024) return of(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (cols <= 2048) return of(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (cols <= 4096) return of(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (cols <= 8192) return of(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  of(integral_constant<int, 256>{}, integral_constant<int, 8>{});
}

}  // namespace

int layer_norm_lanes(int cols) {
  int lanes = 0;
  by_width(cols, [&](auto l, auto) { lanes = decltype(l)::value; });
  return lanes;
}

int layer_norm_parts(int64_t rows, int cols) {
  const int64_t slots = kThreads / layer_norm_lanes(cols), turns = (rows + slots - 1) / slots;
  return int(turns < 512 ? turns : 512);
}

hipError_t launch_layer_norm(const LayerNorm& a, bool f32, hipStream_t s) {
  by_width(a.cols, [&](auto lanes, auto vec) {
    constexpr int L = decltype(lanes)::value, V = decltype(vec)::value, R = kThreads / L;
    const dim3 grid(unsigned((a.rows + R - 1) / R));
    if (f32) hipLaunchKernelGGL((k10_forward<true, L, V>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k10_forward<false, L, V>), grid, dim3(kThreads), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_layer_norm_backward(LayerNormBackward a, bool f32, hipStream_t s) {
  a.num_parts = layer_norm_parts(a.rows, a.cols);
  by_width(a.cols, [&](auto lanes, auto vec) {
    constexpr int L = decltype(lanes)::value, V = decltype(vec)::value;
    const dim3 grid{unsigned(a.num_parts)};
    if (a.rows == 0) return;
    if (f32) hipLaunchKernelGGL((k10_backward<true, L, V>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k10_backward<false, L, V>), grid, dim3(kThreads), 0, s, a);
  });
  if (a.dweight != nullptr || a.dbias != nullptr)
    hipLaunchKernelGGL(k10_reduce, dim3(unsigned(2 * ((a.cols + 63) / 64))), dim3(kThreads), 0, s,
                       a);
  return hipGetLastError();
}

}  // namespace gnmr
