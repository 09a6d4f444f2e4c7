// K8: Newton-Schulz orthogonalisation of updates G (m x n, m <= n after a transposition
// where needed), many of one shape at a time:
//
//   X = G / (||G||_F + eps)
//   repeat `steps` times:  A = X X^T,  P = a I + b A + c A A,  X = P X
//   out = scale * X
//
// drives every singular value of G towards 1 and keeps its singular vectors.
//
// The iterates are held in fp16 between the products, X scaled by 2^12: |X| <= its
// largest singular value, so the range holds values from 2^-26 (with all 11 bits) to 15.99, and each
// rounding is at most 2^-11 relative, an eighth of bf16's at the same matrix-core rate.  |A| can
// reach the square of that value and |P| what the polynomial makes of it: their powers of two follow
// from the coefficients (k8_range.h), 2^12 too with the usual ones, whose |A| stays below 1.5
// and |P| below 4.  With lower ones their small values lose bits, but A and P act as wholes: what
// counts is the rounding beside their largest.  Products accumulate in fp32.
//
// The diagonals are kept whole, for they are the largest entries and, in an update much wider than
// high, nearly equal: their roundings went one way in every row and step, and made most of the
// error.  What rounding takes off A's diagonal (d) is put back into P's in fp32, as b d + 2 c A_ii d
// (off the diagonal it is as small as the entries' own rounding); and P is held as D P' with P'
// rounded and D, next to I, such that D P' has P's diagonal: D multiplies the rows of the product.
// Error in the 2-norm before and after, of which the last rounding to bf16 is 1.66e-3: 32 x 1673
// 3.2e-3 and 1.8e-3, 256 x 256 2.1e-3 and 1.9e-3, 1408 x 2048 1.89e-3 and 1.83e-3; 64 updates of 1408 x
// 2048 take 1% longer so, 16 of 256 x 256 2%.  (a X added to the product in fp32, instead of a in
// P's diagonal, costs a read of X for every product, 640 us instead of 540, and is no nearer.)
//
// The first X is G times a power of two, exact for bf16 input; what is left of the norm goes into
// the first iteration's factors.  The norm is summed in float64.
// Where eps is larger than the norm, X starts that much below 1 and is held as many powers of two
// higher, fewer by every step by what it may grow: it keeps its bits however small.
#include "gnmr_internal.h"
#include "groups.h"
#include "k8_range.h"
#include "lane_ops.h"
#include "mm_tile.h"

namespace gnmr {
namespace {

using mm::F16;
using mm::f32x4;
using mm::u32x2;
using mm::u32x4;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ u32x2 half4(float a, float b, float c, float d) {
  return __builtin_bit_cast(u32x2, f16x4{_Float16(a), _Float16(b), _Float16(c), _Float16(d)});
}

constexpr float kHeld = 0x1p12f;       // what X is multiplied by in fp16
constexpr float kUnheld = 0x1p-12f;
static_assert(kHeld == float(1 << kHeldX), "X is held as its range assumes");

// Eight values from p, which is aligned to 16 bytes.
template <bool kF32>
__device__ __forceinline__ void eight(const char* p, float* v) {
  if constexpr (kF32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 q = reinterpret_cast<const f32x4*>(p)[h];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[4 * h + k] = q[k];
    }
  } else {
    const u32x4 q = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(q[k] << 16);
      v[2 * k + 1] = __uint_as_float(q[k] & 0xFFFF0000u);
    }
  }
}
template <bool kF32>
__device__ __forceinline__ float one_value(const char* p) {
  if constexpr (kF32) return *reinterpret_cast<const float*>(p);
  else return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
}

// Partial sums of squares of each matrix, in float64: a.parts workgroups a matrix.
template <bool kF32>
__global__ __launch_bounds__(256) void k8_norm(const Orthogonal a) {
  constexpr int kSize = kF32 ? 4 : 2;
  __shared__ double red[4];
  const int64_t size = int64_t(a.rows) * a.cols;
  const char* p = static_cast<const char*>(a.in) + int64_t(blockIdx.y) * size * kSize;
  // up to the first 16-byte boundary one by one, then eight at a time
  const int64_t skew = (16 - reinterpret_cast<uintptr_t>(p) % 16) % 16 / kSize;
  const int64_t head = skew < size ? skew : size, body = (size - head) / 8;
  const int64_t first = int64_t(blockIdx.x) * 256 + threadIdx.x, all = int64_t(a.parts) * 256;
  double ss = 0.0;
  auto add = [&](float v) { ss = fma(double(v), double(v), ss); };
  const char* q = p + head * kSize;
#pragma unroll 4
  for (int64_t i = first; i < body; i += all) {
    float v[8];
    eight<kF32>(q + i * 8 * kSize, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) add(v[k]);
  }
  if (first < head) add(one_value<kF32>(p + first * kSize));
  const int64_t tail = head + 8 * body + first;
  if (tail < size) add(one_value<kF32>(p + tail * kSize));
  ss = wave_sum(ss);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  if (threadIdx.x == 0)
    a.sums[int64_t(blockIdx.y) * a.parts + blockIdx.x] = ((red[0] + red[1]) + red[2]) + red[3];
}

// X (and zeros around it) from G: 64 x 64 elements to a workgroup.  Reads go along the rows
// of G and writes along those of X, through LDS where X is the transpose.
template <bool kF32, bool kFlip>
__global__ __launch_bounds__(256) void k8_load(const Orthogonal a) {
  constexpr int kSize = kF32 ? 4 : 2;
  __shared__ double red[4];
  const int64_t size = int64_t(a.rows) * a.cols;
  const int mat = blockIdx.z, m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  double ss = 0.0;
  for (int i = threadIdx.x; i < a.parts; i += 256) ss += a.sums[int64_t(mat) * a.parts + i];
  ss = wave_sum(ss);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  const double length = sqrt(((red[0] + red[1]) + red[2]) + red[3]);
  const double norm = length + double(a.eps);
  int k = 0, extra = 0;
  (void)frexp(norm, &k);            // norm = f * 2^k, f in [0.5, 1)
  if (length > 0.0 && length < norm) {
    (void)frexp(norm / length, &extra);
    --extra;                        // length * 2^extra <= norm (0 where length is infinite)
  }
  const int up = 12 - k + extra;    // |G| * 2^up <= 2^12
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    // The factor is kept to 20 bits (X to 5e-7 of its scale): the last bit of a norm, which a
    // product with 2^20 that is off by as much changes, then leaves every bit of the result.
    const float f = norm == 0.0 ? 0.0f : float(1.0 / ldexp(norm, 12 - k));
    a.start[mat] = OrthogonalStart{__uint_as_float((__float_as_uint(f) + 8u) & ~15u), extra};
  }
  // eight consecutive elements of a row of G to a lane: rows r0 .. r0+63 from column c0
  const char* in = static_cast<const char*>(a.in) + int64_t(mat) * size * kSize;
  const int r0 = kFlip ? n0 : m0, c0 = kFlip ? m0 : n0;
  const bool vectors = a.cols % 8 == 0 && reinterpret_cast<uintptr_t>(a.in) % 16 == 0;
  _Float16* x = a.x[0] + int64_t(mat) * a.mp * a.np;
  __shared__ _Float16 tile[kFlip ? 64 : 1][72];
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    const int i = 32 * pass + (threadIdx.x >> 3), j = 8 * (threadIdx.x & 7);
    const int r = r0 + i, c = c0 + j;
    float v[8] = {};
    if (r < a.rows) {
      const char* p = in + (int64_t(r) * a.cols + c) * kSize;
      if (vectors) {
        if (c < a.cols) eight<kF32>(p, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < a.cols) v[e] = one_value<kF32>(p + e * kSize);
      }
    }
    _Float16 h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = _Float16(ldexpf(v[e], up));
    if constexpr (kFlip) {
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[j + e][i] = h[e];
    } else {
      *reinterpret_cast<u32x4*>(x + int64_t(m0 + i) * a.np + n0 + j) =
          *reinterpret_cast<const u32x4*>(h);
    }
  }
  if constexpr (kFlip) {
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      const int i = 32 * pass + (threadIdx.x >> 3), j = 8 * (threadIdx.x & 7);
      *reinterpret_cast<u32x4*>(x + int64_t(m0 + i) * a.np + n0 + j) =
          *reinterpret_cast<const u32x4*>(&tile[i][j]);
    }
  }
}

enum { kGram, kPoly, kApply, kLast };  // the products of an iteration; the last X

// One product: A = X X^T; P = a I + b A + c A A; X = P X, or the result from it.
// A and P are symmetric: their tiles above the diagonal are computed and leave twice.
template <int kWhat, bool kFlip, int kT>
__global__ __launch_bounds__(
    mm::kThreads, (mm::Depth<false, kWhat == kApply || kWhat == kLast, kT>::kPerCu)) void k8_product(const Orthogonal a) {
  constexpr bool kIntoX = kWhat == kApply || kWhat == kLast;
  using D = mm::Depth<false, kIntoX, kT>;
  using T = mm::Tile<F16, false, kIntoX, kT, kT, 2, D::kStep, D::kStages, kFlip>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int v = xcd_order(blockIdx.x, a.num_tiles), part = 0;
  constexpr int kSide = 256 / kT;
  if constexpr (kT < 256) {
    part = v % (kSide * kSide);
    v /= kSide * kSide;
  }
  v += a.first_tile;
  const int mat = v / a.tiles;
  int tm, tn;
  if constexpr (kIntoX) walk<8>(v % a.tiles, a.tiles_m, a.tiles_n, &tm, &tn);
  else walk_triangle(v % a.tiles, &tm, &tn);
  if constexpr (kT < 256) {
    tm = kSide * tm + part / kSide;
    tn = kSide * tn + part % kSide;
  }
  const int m0 = tm * kT, n0 = tn * kT;
  if (m0 >= a.mp || n0 >= (kIntoX ? a.np : a.mp) || (!kIntoX && tm > tn)) return;
  const int K = kWhat == kGram ? a.np : a.mp;
  const _Float16* x = a.x[a.step & 1] + int64_t(mat) * a.mp * a.np;
  _Float16* A = a.A + int64_t(mat) * a.mp * a.mp;
  _Float16* P = a.P + int64_t(mat) * a.mp * a.mp;
  const _Float16* left = kWhat == kGram ? x : kWhat == kPoly ? A : P;
  const _Float16* right = kWhat == kPoly ? A : x;
  const int ld = kWhat == kGram ? a.np : a.mp;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(left + int64_t(m0) * ld, int64_t(ld) * 2, a.mp - m0, wave, lane);
  if constexpr (kIntoX) on.at(right + n0, int64_t(a.np) * 2, a.np - n0, wave, lane);
  else on.at(right + int64_t(n0) * ld, int64_t(ld) * 2, a.mp - n0, wave, lane);
  // P needs this tile of A: in the smaller tiles it is on its way while the product runs (a
  // 256 tile has no registers for it)
  auto stored = [&](int m, int n) {
    return *reinterpret_cast<const f16x4*>(A + int64_t(min(m0 + m, a.mp - 1)) * a.mp +
                                           min(n0 + n, a.mp - 4));
  };
  constexpr bool kEarly = kWhat == kPoly && kT < 256;
  f16x4 old[kEarly ? T::kGroups : 1];
  if constexpr (kEarly)
    T::groups(wave, lane, [&](int e, int m, int n) { old[e] = stored(m, n); });
  const OrthogonalStart start = a.start[mat];
  const float f = a.step == 0 ? start.factor : kUnheld;   // X = f * 2^-e * what is held
  const int extra = start.extra - a.step * a.growth, e = max(extra, 0);
  // What the epilogue needs of a lane's rows is on its way while the product runs (rows past the
  // last ones read that: nothing of theirs is stored).
  float* const gap = a.gap + int64_t(mat) * a.mp;
  float* const row = a.row + int64_t(mat) * a.mp;
  constexpr bool kOfRows = kWhat == kPoly || (kIntoX && !kFlip);
  float of[kOfRows ? T::kRows / 32 : 1];
  if constexpr (kOfRows) {
#pragma unroll
    for (int i = 0; i < T::kRows / 32; ++i)
      of[i] = (kWhat == kPoly ? gap : row)[min(m0 + T::first_row(wave) + 32 * i + (lane & 31),
                                               a.mp - 1)];
  }
  T::product(acc, om, on, K, wave, lane);
  // s times P's factors for four accumulators at (row, col) of the tile
  auto factors = [&](float s, int r, int c) {
    if constexpr (kFlip) {
      return s * *reinterpret_cast<const f32x4*>(row + min(m0 + c, a.mp - 4));
    } else {
      const float v = s * of[kOfRows ? uint32_t(r - T::first_row(wave)) / 32 : 0];
      return f32x4{v, v, v, v};
    }
  };
  if constexpr (!kIntoX) {
    _Float16* to = kWhat == kGram ? A : P;
    const float s = ldexpf(f * f * a.held_a, -2 * e);
    const float p = a.poly_a, q = a.poly_aa, one = a.poly_one;
    T::change(acc, wave, lane, [&](int group, int m, int n, f32x4 c) {
      // which of the four is on the diagonal, which the lane's blocks of 32 on their own meet
      constexpr int kAcross = T::kCols / 32;
      const uint32_t on = uint32_t(m0 + m - n0 - n);
      const bool meets = group / 4 / kAcross == group / 4 % kAcross && on < 4;
      f32x4 r;
      float h = 0.0f;
      if constexpr (kWhat == kGram) {
        r = c * s;
      } else {
        f16x4 v;
        if constexpr (kEarly) v = old[group];
        else v = stored(m, n);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          r[k] = p * float(v[k]) + q * c[k];
          h = on == uint32_t(k) ? float(v[k]) : h;
        }
      }
      if (meets && m0 + m < a.mp) {
        float d = on == 0 ? r[0] : on == 1 ? r[1] : on == 2 ? r[2] : r[3];
        if constexpr (kWhat == kGram) {
          gap[m0 + m] = d - float(_Float16(d));
        } else {
          d += one + of[kWhat == kPoly ? group / 4 / kAcross : 0] * (p + 2.0f * q * h);
#pragma unroll
          for (int k = 0; k < 4; ++k) r[k] = on == uint32_t(k) ? d : r[k];
          const float held = float(_Float16(d));
          row[m0 + m] = fabsf(held) < 0x1p-14f ? 1.0f : d / held;
        }
      }
      return r;
    });
    auto round = [](int, int, float a0, float a1, float a2, float a3) {
      return half4(a0, a1, a2, a3);
    };
    T::out16(acc, wave, lane, round, [&](int m, int n, const u32x4& h) {
      if (m0 + m < a.mp && n0 + n < a.mp)
        *reinterpret_cast<u32x4*>(to + int64_t(m0 + m) * a.mp + n0 + n) = h;
    });
    if (tm == tn) return;
    T::out16_mirrored(acc, wave, lane, round, [&](int n, int m, const u32x4& h) {
      if (m0 + m < a.mp && n0 + n < a.mp)
        *reinterpret_cast<u32x4*>(to + int64_t(n0 + n) * a.mp + m0 + m) = h;
    });
  } else if constexpr (kWhat == kApply) {
    _Float16* to = a.x[(a.step & 1) ^ 1] + int64_t(mat) * a.mp * a.np;
    const float s = ldexpf(f * a.apply, max(extra - a.growth, 0) - e);
    T::out16(
        acc, wave, lane,
        [&](int r, int c, float a0, float a1, float a2, float a3) {
          const f32x4 v = factors(s, r, c);
          return half4(v[0] * a0, v[1] * a1, v[2] * a2, v[3] * a3);
        },
        [&](int m, int n, const u32x4& h) {
          if (m0 + m < a.mp && n0 + n < a.np)
            *reinterpret_cast<u32x4*>(to + int64_t(m0 + m) * a.np + n0 + n) = h;
        });
  } else {
    // rows of the update: m, or n with kFlip
    const int rows = kFlip ? a.n : a.m, cols = kFlip ? a.m : a.n;
    const int row0 = kFlip ? n0 : m0, col0 = kFlip ? m0 : n0;
    __bf16* out = a.out + int64_t(mat) * a.m * a.n;
    const bool whole = cols % 8 == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
    const float s = ldexpf(f * a.last, -e);
    T::out16(
        acc, wave, lane,
        [&](int r, int c, float a0, float a1, float a2, float a3) {
          const f32x4 v = factors(s, r, c);
          return u32x2{pack(v[0] * a0, v[1] * a1), pack(v[2] * a2, v[3] * a3)};
        },
        [&](int row, int col, const u32x4& h) {
          const int r = row0 + row, c = col0 + col;
          if (r >= rows || c >= cols) return;
          __bf16* to = out + int64_t(r) * cols + c;
          if (whole) {
            *reinterpret_cast<u32x4*>(to) = h;
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (c + k < cols)
                to[k] = __builtin_bit_cast(__bf16, uint16_t(h[k >> 1] >> (16 * (k & 1))));
          }
        });
  }
}

// Tiles [first, first + n) of 256 x 256 in the order of the walk, as such or cut into smaller ones.
template <int kWhat, bool kFlip, int kT>
void launch_tiles(Orthogonal a, int64_t first, int64_t n, hipStream_t s) {
  if (n == 0) return;
  a.first_tile = int32_t(first);
  a.num_tiles = int32_t(n * (256 / kT) * (256 / kT));
  hipLaunchKernelGGL((k8_product<kWhat, kFlip, kT>), dim3(unsigned(a.num_tiles)),
                     dim3(mm::kThreads), 0, s, a);
}

template <int kWhat, bool kFlip>
void launch_product(Orthogonal a, hipStream_t s) {
  constexpr bool kSquare = kWhat == kGram || kWhat == kPoly;
  a.tiles_m = (a.mp + 255) / 256;
  a.tiles_n = kSquare ? a.tiles_m : (a.np + 255) / 256;
  a.tiles = kSquare ? a.tiles_m * (a.tiles_m + 1) / 2 : a.tiles_m * a.tiles_n;
  const BatchLaunch b = batch_launch(kWhat == kGram   ? BatchProduct::kOfRows
                                     : kWhat == kPoly ? BatchProduct::kOfSquares
                                                      : BatchProduct::kOntoRows,
                                     a.count, a.mp, a.np);
  launch_tiles<kWhat, kFlip, 256>(a, 0, b.large, s);
  if (b.edge == 64) launch_tiles<kWhat, kFlip, 64>(a, b.large, b.all - b.large, s);
  else launch_tiles<kWhat, kFlip, 128>(a, b.large, b.all - b.large, s);
}

int pad(int x) { return (x + 63) / 64 * 64; }
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int64_t orthogonal_workgroups(const Orthogonal& a) {
  const int64_t mp = pad(std::min(a.rows, a.cols)), np = pad(std::max(a.rows, a.cols));
  return a.count * ((mp + 255) / 256) * ((np + 255) / 256) * 16;  // in tiles of 64
}

namespace {

// Workgroups that sum one matrix's squares: enough for the chip over all matrices, at
// least 8,192 values each.
int norm_parts(int64_t size, int count) {
  const int64_t most = std::max<int64_t>(1, 1024 / count);
  return int(std::min(most, (size + 8191) / 8192));
}

}  // namespace

int64_t orthogonal_workspace(int32_t rows, int32_t cols, int32_t count) {
  const int64_t mp = pad(std::min(rows, cols)), np = pad(std::max(rows, cols));
  return up256(int64_t(count) * norm_parts(int64_t(rows) * cols, count) * 8) +
         up256(int64_t(count) * int64_t(sizeof(OrthogonalStart))) + 2 * up256(count * mp * 4) +
         int64_t(count) * (2 * mp * np + 2 * mp * mp) * 2;
}

hipError_t launch_orthogonal(Orthogonal a, const gnmr_newton_schulz& z, void* workspace,
                             hipStream_t s) {
  a.flip = a.rows > a.cols;
  a.m = a.flip ? a.cols : a.rows;
  a.n = a.flip ? a.rows : a.cols;
  a.mp = pad(a.m);
  a.np = pad(a.n);
  const HeldExponents held = held_exponents(z.a, z.b, z.c, z.steps);
  a.held_a = ldexpf(1.0f, held.a);
  const float held_p = ldexpf(1.0f, held.p);
  a.growth = held.growth;
  // (all but the coefficients are powers of two)
  a.poly_a = z.b * (held_p / a.held_a);
  a.poly_aa = z.c * (held_p / a.held_a / a.held_a);
  a.poly_one = z.a * held_p;
  a.apply = kHeld / held_p;
  a.last = z.scale / held_p;
  char* w = static_cast<char*>(workspace);
  a.sums = reinterpret_cast<double*>(w);
  a.parts = norm_parts(int64_t(a.rows) * a.cols, a.count);
  w += up256(int64_t(a.count) * a.parts * 8);
  a.start = reinterpret_cast<OrthogonalStart*>(w);
  w += up256(int64_t(a.count) * int64_t(sizeof(OrthogonalStart)));
  a.gap = reinterpret_cast<float*>(w);
  w += up256(int64_t(a.count) * a.mp * 4);
  a.row = reinterpret_cast<float*>(w);
  w += up256(int64_t(a.count) * a.mp * 4);
  const int64_t xs = int64_t(a.count) * a.mp * a.np, as = int64_t(a.count) * a.mp * a.mp;
  a.x[0] = reinterpret_cast<_Float16*>(w);
  a.x[1] = a.x[0] + xs;
  a.A = a.x[1] + xs;
  a.P = a.A + as;
  const dim3 parts(unsigned(a.parts), unsigned(a.count));
  const dim3 tiles(unsigned(a.np / 64), unsigned(a.mp / 64), unsigned(a.count));
  if (a.f32) hipLaunchKernelGGL(k8_norm<true>, parts, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k8_norm<false>, parts, dim3(256), 0, s, a);
  if (a.f32 && a.flip) hipLaunchKernelGGL((k8_load<true, true>), tiles, dim3(256), 0, s, a);
  else if (a.f32) hipLaunchKernelGGL((k8_load<true, false>), tiles, dim3(256), 0, s, a);
  else if (a.flip) hipLaunchKernelGGL((k8_load<false, true>), tiles, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k8_load<false, false>), tiles, dim3(256), 0, s, a);
  for (a.step = 0; a.step < z.steps; ++a.step) {
    launch_product<kGram, false>(a, s);
    launch_product<kPoly, false>(a, s);
    if (a.step + 1 < z.steps) launch_product<kApply, false>(a, s);
    else if (a.flip) launch_product<kLast, true>(a, s);
    else launch_product<kLast, false>(a, s);
  }
  return hipGetLastError();
}

}  // namespace gnmr
