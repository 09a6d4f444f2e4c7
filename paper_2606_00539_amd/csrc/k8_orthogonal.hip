// K8: Newton-Schulz orthogonalisation of updates G (m x n, m <= n after a transposition
// where needed), many of one shape at a time:
//
//   X = G / (||G||_F + eps)
//   repeat `steps` times:  A = X X^T,  B = b A + c A A,  X = a X + B X
//   out = scale * X
//
// drives every singular value of G towards 1 and keeps its singular vectors.
//
// The iterates are held in fp16 between the products, scaled by 2^12: |X| <= its
// largest singular value, which the usual coefficients keep below 1.3, so the range
// holds values from 2^-26 (with all 11 bits) to 16, and each product's rounding is
// 2^-12 relative, an eighth of bf16's at the same matrix-core rate.  Products
// accumulate in fp32 and a X is added in fp32.  The first X is G times a power of
// two, exact for bf16 input; what is left of the norm goes into the first
// iteration's factors.  The norm is summed in float64.
#include "gnmr_internal.h"
#include "groups.h"
#include "lane_ops.h"
#include "mm_tile.h"

namespace gnmr {
namespace {

using mm::F16;
using mm::u32x2;
using mm::u32x4;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kHeld = 0x1p12f;       // what X, A and B are multiplied by in fp16
constexpr float kUnheld = 0x1p-12f;
constexpr int kNormBlocks = 64;        // partial sums of squares of one matrix

__device__ __forceinline__ float value(const void* p, int64_t i, bool f32) {
  return f32 ? static_cast<const float*>(p)[i]
             : __uint_as_float(uint32_t(static_cast<const uint16_t*>(p)[i]) << 16);
}

__global__ __launch_bounds__(256) void k8_norm(const Orthogonal a) {
  __shared__ double red[4];
  const int64_t size = int64_t(a.rows) * a.cols, at = int64_t(blockIdx.y) * size;
  double ss = 0.0;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < size; i += kNormBlocks * 256) {
    const double v = value(a.in, at + i, a.f32);
    ss = fma(v, v, ss);
  }
  ss = wave_sum(ss);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  if (threadIdx.x == 0)
    a.sums[int64_t(blockIdx.y) * kNormBlocks + blockIdx.x] = ((red[0] + red[1]) + red[2]) + red[3];
}

// X (and zeros around it) from G: 64 x 64 elements to a workgroup.
__global__ __launch_bounds__(256) void k8_load(const Orthogonal a) {
  __shared__ float tile[64][65];
  const int64_t size = int64_t(a.rows) * a.cols;
  const int mat = blockIdx.z, m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  double ss = a.sums[int64_t(mat) * kNormBlocks + (threadIdx.x & 63)];
  ss = wave_sum(ss);
  const double norm = sqrt(ss) + double(a.eps);
  int k = 0;
  (void)frexp(norm, &k);            // norm = f * 2^k, f in [0.5, 1)
  const int up = 12 - k;            // |G| * 2^up <= 2^12
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
    a.factor[mat] = norm == 0.0 ? 0.0f : float(1.0 / ldexp(norm, up));
  const char* in = static_cast<const char*>(a.in) + int64_t(mat) * size * (a.f32 ? 4 : 2);
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  for (int i = ty; i < 64; i += 4) {
    // reads go along the rows of G
    const int r = a.flip ? n0 + i : m0 + i, c = a.flip ? m0 + tx : n0 + tx;
    float v = 0.0f;
    if (r < a.rows && c < a.cols) v = value(in, int64_t(r) * a.cols + c, a.f32);
    if (a.flip) tile[tx][i] = v;
    else tile[i][tx] = v;
  }
  __syncthreads();
  _Float16* x = a.x[0] + int64_t(mat) * a.mp * a.np;
  for (int i = ty; i < 64; i += 4)
    x[int64_t(m0 + i) * a.np + n0 + tx] = _Float16(ldexpf(tile[i][tx], up));
}

enum { kGram, kPoly, kApply, kLast };

// One product of an iteration: A = X X^T; B = b A + c A A; X = a X + B X; the last X.
template <int kWhat, bool kFlip, int kT, int kStages, int kPerCu>
__global__ __launch_bounds__(mm::kThreads, kPerCu) void k8_product(const Orthogonal a) {
  constexpr bool kIntoX = kWhat == kApply || kWhat == kLast;
  using T = mm::Tile<F16, false, kIntoX, kT, kT, 2, kStages>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = a.tiles_m * a.tiles_n, v = xcd_order(blockIdx.x, a.count * per);
  const int mat = v / per;
  int tm, tn;
  walk<8>(v % per, a.tiles_m, a.tiles_n, &tm, &tn);
  const int m0 = tm * kT, n0 = tn * kT;
  const int N = kIntoX ? a.np : a.mp, K = kWhat == kGram ? a.np : a.mp;
  const _Float16* x = a.x[a.now] + int64_t(mat) * a.mp * a.np;
  _Float16* A = a.A + int64_t(mat) * a.mp * a.mp;
  _Float16* B = a.B + int64_t(mat) * a.mp * a.mp;
  const _Float16* left = kWhat == kGram ? x : kWhat == kPoly ? A : B;
  const _Float16* right = kWhat == kPoly ? A : x;
  const int ld = kWhat == kGram ? a.np : a.mp;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(left + int64_t(m0) * ld, int64_t(ld) * 2, a.mp - m0, wave, lane);
  if constexpr (kIntoX) on.at(right + n0, int64_t(a.np) * 2, a.np - n0, wave, lane);
  else on.at(right + int64_t(n0) * ld, int64_t(ld) * 2, a.mp - n0, wave, lane);
  T::template product<kFlip>(acc, om, on, K, wave, lane);
  const float f = a.first ? a.factor[mat] : kUnheld;   // X = f * what is held
  T::template each<kFlip>(wave, lane, [&](int i, int j, int g, int dm, int dn) {
    const int m = m0 + dm, n = n0 + dn;
    const auto& c = acc[i][j];
    if constexpr (kWhat == kGram) {
      if (m < a.mp && n < a.mp) {
        f16x4 h;
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = _Float16(c[4 * g + k] * (f * f * kHeld));
        *reinterpret_cast<f16x4*>(A + int64_t(m) * a.mp + n) = h;
      }
    } else if constexpr (kWhat == kPoly) {
      if (m < a.mp && n < a.mp) {
        const f16x4 old = *reinterpret_cast<const f16x4*>(A + int64_t(m) * a.mp + n);
        f16x4 h;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          h[k] = _Float16(a.cb * float(old[k]) + (a.cc * kUnheld) * c[4 * g + k]);
        *reinterpret_cast<f16x4*>(B + int64_t(m) * a.mp + n) = h;
      }
    } else if constexpr (kWhat == kApply) {
      if (m < a.mp && n < N) {
        const f16x4 old = *reinterpret_cast<const f16x4*>(x + int64_t(m) * a.np + n);
        f16x4 h;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          h[k] = _Float16((a.ca * float(old[k]) + kUnheld * c[4 * g + k]) * (f * kHeld));
        *reinterpret_cast<f16x4*>(a.x[a.now ^ 1] + int64_t(mat) * a.mp * a.np +
                                  int64_t(m) * a.np + n) = h;
      }
    } else {
      // four elements along m with kFlip, along n without
      __bf16* out = a.out + int64_t(mat) * a.m * a.n;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int mk = kFlip ? m + k : m, nk = kFlip ? n : n + k;
        if (mk < a.m && nk < a.n) {
          const float old = float(x[int64_t(mk) * a.np + nk]);
          const float r = (a.ca * old + kUnheld * c[4 * g + k]) * (f * a.scale);
          out[kFlip ? int64_t(nk) * a.m + mk : int64_t(mk) * a.n + nk] = __bf16(r);
        }
      }
    }
  });
}

template <int kWhat, bool kFlip>
void launch_product(Orthogonal a, hipStream_t s) {
  constexpr int kT = 128;
  a.tiles_m = (a.mp + kT - 1) / kT;
  a.tiles_n = ((kWhat == kGram || kWhat == kPoly ? a.mp : a.np) + kT - 1) / kT;
  hipLaunchKernelGGL((k8_product<kWhat, kFlip, kT, 2, 2>),
                     dim3(unsigned(int64_t(a.count) * a.tiles_m * a.tiles_n)), dim3(mm::kThreads),
                     0, s, a);
}

int pad(int x) { return (x + 63) / 64 * 64; }
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int64_t orthogonal_workgroups(const Orthogonal& a) {
  const int64_t mp = pad(std::min(a.rows, a.cols)), np = pad(std::max(a.rows, a.cols));
  return a.count * ((mp + 127) / 128) * ((np + 127) / 128);
}

int64_t orthogonal_workspace(int32_t rows, int32_t cols, int32_t count) {
  const int64_t mp = pad(std::min(rows, cols)), np = pad(std::max(rows, cols));
  return up256(int64_t(count) * kNormBlocks * 8) + up256(int64_t(count) * 4) +
         int64_t(count) * (2 * mp * np + 2 * mp * mp) * 2;
}

hipError_t launch_orthogonal(Orthogonal a, void* workspace, int steps, hipStream_t s) {
  a.flip = a.rows > a.cols;
  a.m = a.flip ? a.cols : a.rows;
  a.n = a.flip ? a.rows : a.cols;
  a.mp = pad(a.m);
  a.np = pad(a.n);
  char* w = static_cast<char*>(workspace);
  a.sums = reinterpret_cast<double*>(w);
  w += up256(int64_t(a.count) * kNormBlocks * 8);
  a.factor = reinterpret_cast<float*>(w);
  w += up256(int64_t(a.count) * 4);
  const int64_t xs = int64_t(a.count) * a.mp * a.np, as = int64_t(a.count) * a.mp * a.mp;
  a.x[0] = reinterpret_cast<_Float16*>(w);
  a.x[1] = a.x[0] + xs;
  a.A = a.x[1] + xs;
  a.B = a.A + as;
  hipLaunchKernelGGL(k8_norm, dim3(kNormBlocks, unsigned(a.count)), dim3(256), 0, s, a);
  hipLaunchKernelGGL(k8_load, dim3(unsigned(a.np / 64), unsigned(a.mp / 64), unsigned(a.count)),
                     dim3(256), 0, s, a);
  for (int i = 0; i < steps; ++i) {
    a.first = i == 0;
    a.now = i & 1;
    launch_product<kGram, false>(a, s);
    launch_product<kPoly, false>(a, s);
    if (i + 1 < steps) launch_product<kApply, false>(a, s);
    else if (a.flip) launch_product<kLast, true>(a, s);
    else launch_product<kLast, false>(a, s);
  }
  return hipGetLastError();
}

}  // namespace gnmr
