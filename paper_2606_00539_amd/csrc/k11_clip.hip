// K11: the global norm of a set of gradients, and the gradients scaled to at most max_norm:
//
//   n = sqrt( sum over tensors of |g|^2 + sum over u of norm_u^2 ),
//   c = max_norm / (n + eps) where n + eps > max_norm, else 1 (NaN where n is NaN);  out = c g
//
// norm_u are norms that are known (the controller's): their tensors need no reading for n.  Sums
// and products are in float64, so that no gradient's square overflows or vanishes; the rate of
// float64 on this chip is far above that of memory.  A workgroup sums the chunks w, w + G, ... of all
// tensors; the sums are added in one order by whoever needs them, so all workgroups have the same c.
#include <type_traits>

#include "gnmr_internal.h"
#include "lane_ops.h"
#include "values.h"

namespace gnmr {
namespace {

constexpr int kThreads = 256;
// The tensor of chunk c, by a lane to a tensor: first[] rises, and a tensor without values
// has the next one's first chunk.
template <class T>
__device__ __forceinline__ int tensor_of(const T& t, int c, int lane) {
  int k = -1;
#pragma unroll
  for (int base = 0; base < T::kMost; base += 64) {
    const int i = base + lane;
    k += __popcll(__ballot(i < t.num && t.t[i < T::kMost ? i : 0].first <= c));
  }
  return k;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// each(i, count) for the runs of up to N values that this thread has of [lo, hi); whole runs
// kAhead at a time, runs(i), N * kThreads apart: their loads are on their way together.
template <int N, int kAhead, class Runs, class Each>
__device__ __forceinline__ void sweep(int64_t lo, int64_t hi, Runs&& runs, Each&& each) {
  constexpr int kStride = N * kThreads;
  int64_t i = lo + N * threadIdx.x;
  for (; i + (kAhead - 1) * kStride + N <= hi; i += kAhead * kStride) runs(i);
  for (; i < hi; i += kStride) each(i, hi - i < N ? int(hi - i) : N);
}

template <bool kF32>
__device__ __forceinline__ double squares(const void* p, int64_t lo, int64_t hi) {
  constexpr int N = kF32 ? 4 : 8, kAhead = 4;
  double s[2] = {0.0, 0.0};
  auto add = [&](const Run<N>& e) {
#pragma unroll
    for (int k = 0; k < N; ++k) s[k & 1] = fma(double(e.v[k]), double(e.v[k]), s[k & 1]);
  };
  sweep<N, kAhead>(
      lo, hi,
      [&](int64_t i) {
        Run<N> e[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) e[q] = load_run<kF32, N>(p, i + q * N * kThreads);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) add(e[q]);
      },
      [&](int64_t i, int count) { add(load_some<kF32, N>(p, i, count)); });
  return s[0] + s[1];
}

template <class T>
__global__ __launch_bounds__(kThreads) void k11_squares(const T t, double* parts) {
  __shared__ double red[4];
  const int lane = threadIdx.x & 63;
  double s = 0.0;
  for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const ClipTensor& k = t.t[__builtin_amdgcn_readfirstlane(tensor_of(t, c, lane))];
    const int64_t lo = int64_t(c - k.first) * t.chunk, hi = min(lo + t.chunk, k.numel);
    s += k.in_f32 ? squares<true>(k.in, lo, hi) : squares<false>(k.in, lo, hi);
  }
  s = block_sum(s, red);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// Whether f lies in the middle of two bf16 values: only there can rounding a product to fp32 first make
// another bf16 value of it.
__device__ __forceinline__ bool in_the_middle(float f) {
  return (__float_as_uint(f) & 0xFFFFu) == 0x8000u;
}
// d as an fp32 value that rounds to bf16 as d itself does: d, or that one of its fp32 neighbours whose
// last bit is 1.
__device__ __forceinline__ float before_bf16(double d) {
  const float f = float(d);
  const uint32_t bits = __float_as_uint(f);
  const double near = fabs(double(f)), of = fabs(d);
  return __uint_as_float(near < of ? bits | 1u : near > of ? (bits - 1u) | 1u : bits);
}

// Lanes side by side take and leave contiguous memory: eight values a lane only of bf16 to bf16.
// What is read is not read again; what is written goes past the caches too where they cannot hold it.
// 317M values of bf16 to fp32, with the pass before, us: 430, all through the caches 454; 553M of fp32
// to fp32 816 (5.4 TB/s) and 854; eight fp32 values to a lane, 32 bytes apart, 866.
template <bool kIn, bool kOut, bool kPast>
__device__ __forceinline__ void scale(const void* in, void* out, int64_t lo, int64_t hi, double c) {
  constexpr int N = kIn || kOut ? 4 : 8, kAhead = 4;
  auto by = [&](Run<N>& e) {
    Run<N> was;
    bool middle = false;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      was.v[k] = e.v[k];
      e.v[k] = float(double(e.v[k]) * c);
      middle |= in_the_middle(e.v[k]);
    }
    if (!kOut && middle) {
#pragma unroll
      for (int k = 0; k < N; ++k) e.v[k] = before_bf16(double(was.v[k]) * c);
    }
  };
  sweep<N, kAhead>(
      lo, hi,
      [&](int64_t i) {
        Run<N> e[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) e[q] = load_run<kIn, N, true>(in, i + q * N * kThreads);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          by(e[q]);
          store_run<kOut, N, kPast>(out, i + q * N * kThreads, e[q]);
        }
      },
      [&](int64_t i, int count) {
        Run<N> e = load_some<kIn, N>(in, i, count);
        by(e);
        store_some<kOut, N>(out, i, count, e);
      });
}

// This thread's share of what `threads` of them add: the parts, then the squares of the norms.
__device__ __forceinline__ double share(const ClipScale& a, int threads) {
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < a.num_parts; i += threads) s += a.parts[i];
  for (int64_t i = threadIdx.x; i < a.num_norms; i += threads) s = fma(a.norms[i], a.norms[i], s);
  return s;
}

constexpr int kTotalThreads = 1024;
__global__ __launch_bounds__(kTotalThreads) void k11_total(const ClipScale a, double* total) {
  __shared__ double red[kTotalThreads / 64];
  const double s = wave_sum(share(a, kTotalThreads));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  double t = 0.0;
#pragma unroll
  for (int i = 0; i < kTotalThreads / 64; ++i) t += red[i];
  *total = t;
}

// Four wavefronts to a SIMD though registers leave room for eight, whose accesses get in each other's way.
// 300M values, us with four, six and eight: bf16 to bf16 202, 207, 215; fp32 to bf16 304, 314, 323; bf16
// to fp32 328, 331, 339.
template <bool kPast, class T>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4, 4))) void k11_scale(
    const T t, const ClipScale a) {
  __shared__ double red[4];
  const int lane = threadIdx.x & 63;
  const double n = sqrt(block_sum(share(a, kThreads), red)), sum = n + a.eps;
  const double c = sum > a.max_norm ? a.max_norm / sum : n != n ? n : 1.0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = n;
  for (int i = blockIdx.x; i < t.chunks; i += gridDim.x) {
    // backwards: of a set that the caches do not hold, its end was read last and lies there yet
    const int w = t.chunks - 1 - i;
    const ClipTensor& k = t.t[__builtin_amdgcn_readfirstlane(tensor_of(t, w, lane))];
    if (c == 1.0 && k.in == k.out) continue;
    const int64_t lo = int64_t(w - k.first) * t.chunk, hi = min(lo + t.chunk, k.numel);
    if (k.in_f32) {
      if (k.out_f32) scale<true, true, kPast>(k.in, k.out, lo, hi, c);
      else scale<true, false, kPast>(k.in, k.out, lo, hi, c);
    } else {
      if (k.out_f32) scale<false, true, kPast>(k.in, k.out, lo, hi, c);
      else scale<false, false, kPast>(k.in, k.out, lo, hi, c);
    }
  }
}

// launch(the tensors, in an argument of 1 KB where they fit one): the host copies it whole.  Calls with
// tensors of 4,096 values, us, medians of three runs in turn with it and with the long one alone: 28 tensors
// 21.3 and 21.5, 30 21.4 and 21.8, 8 the same.
template <class Launch>
void with_few(const ClipTensors& t, Launch&& launch) {
  if (t.num > kClipFew) return launch(t);
  ClipTensorsOf<kClipFew> few;
  few.num = t.num;
  few.chunks = t.chunks;
  few.chunk = t.chunk;
  for (int i = 0; i < kClipFew; ++i) few.t[i] = t.t[i];
  launch(few);
}

}  // namespace

hipError_t launch_clip_squares(const ClipTensors& t, int workgroups, double* parts, hipStream_t s) {
  with_few(t, [&](const auto& some) {
    hipLaunchKernelGGL((k11_squares<std::decay_t<decltype(some)>>), dim3(unsigned(workgroups)),
                       dim3(kThreads), 0, s, some, parts);
  });
  return hipGetLastError();
}

hipError_t launch_clip_total(const ClipScale& a, double* total, hipStream_t s) {
  hipLaunchKernelGGL(k11_total, dim3(1), dim3(kTotalThreads), 0, s, a, total);
  return hipGetLastError();
}

hipError_t launch_clip_scale(const ClipTensors& t, const ClipScale& a, bool past, hipStream_t s) {
  const int most = 2 * kClipWorkgroups, wgs = t.chunks < 1 ? 1 : t.chunks < most ? t.chunks : most;
  with_few(t, [&](const auto& some) {
    typedef std::decay_t<decltype(some)> T;
    const dim3 grid{unsigned(wgs)}, block(kThreads);
    if (past) hipLaunchKernelGGL((k11_scale<true, T>), grid, block, 0, s, some, a);
    else hipLaunchKernelGGL((k11_scale<false, T>), grid, block, 0, s, some, a);
  });
  return hipGetLastError();
}

}  // namespace gnmr
