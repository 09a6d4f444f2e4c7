// K9: a gated feed-forward block by expert, around the products that K6 has.  Rows (tokens) lie
// sorted by expert, expert e's in [offsets[e], offsets[e+1]); W_e has 2 H rows, the gate's first:
//
//   linear      p[t] = W_e x[t],  h[t][j] = act(p[t][j]) p[t][H + j]
//   dgrad       d[t][j] = sum_o dy[t][o] V_e[o][j],
//               dp[t][j] = d act'(p[t][j]) p[t][H + j],  dp[t][H + j] = d act(p[t][j])
//   activation  h from a p that is there
//
//   silu: act(g) = g s, act'(g) = s (1 + g (1 - s)), s = 1 / (1 + e^-g)
//   gelu: act(g) = g F, act'(g) = F + g e^(-g g / 2) / sqrt(2 pi), F = erfc(-g / sqrt 2) / 2
//
// bf16 operands, fp32 sums and formulas, one rounding of each result: neither p (where it is not
// kept) nor d goes to memory.
//
// Bounds and times: a token's experts' weights for few rows (48 rows in 35 of 64 experts, 2048 to 2 x 1408:
// 404 MB in 78 us, 5.2 TB/s); the chip's power in 256 tiles for many (8,192 rows, 4096 to 2 x 11008: 1,112
// us, 1,330 TFLOP/s; with p 1,160 to 1,240 one after the other); weights from memory and the ends of ragged
// groups between them (24,576 rows in 64 experts, 2048 to 2 x 1408 with p: 341 to 360 us on several cards, 790
// to 830 TFLOP/s; its gradient 218 to 228 us).  h from 8,192 x 2 x 11008 products that are there takes
// 113 us, 4.8 TB/s.
//
// 256 tiles with p spill 17 registers (silu) or 18 at the end of their products, outside of any loop, those
// of h alone one.
#include <type_traits>

#include "gnmr_internal.h"
#include "groups.h"
#include "lane_ops.h"
#include "mm_stream.h"
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
__device__ __forceinline__ u32x2 pack(const f32x4& v) {
  return u32x2{pack(v[0], v[1]), pack(v[2], v[3])};
}
__device__ __forceinline__ f32x4 four(const u32x2& v) {
  return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u),
               __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u)};
}

// act(g) and its derivative.  Exponential and reciprocal are the hardware's, good to a few 2^-23
// of 1 / (1 + e^-g): a bf16 result does not see them.  They are 0 where they would lie below 2^-126
// (g below -87, or -13 for gelu).
struct Act {
  float value, slope;
};
template <int kAct>
__device__ __forceinline__ Act act(float g) {
  if constexpr (kAct == GNMR_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g));
    return Act{g * s, s * fmaf(g, 1.0f - s, 1.0f)};
  } else {
    // F(-u) for u >= 0 is e^(-u u / 2) times a function that falls as 1 / u: there t Q(t) with t =
    // 1 / (1 + 0.33 u) and Q of degree 7, fitted over u up to 83 for the least relative error
    // (1.0e-6; beyond, the exponential is 0).
    const float e = __builtin_amdgcn_exp2f(-0.72134752f * g * g);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.33f, fabsf(g), 1.0f));
    float q = 0.033059838f;
    q = fmaf(q, t, -0.10479434f);
    q = fmaf(q, t, 0.066074904f);
    q = fmaf(q, t, 0.034522207f);
    q = fmaf(q, t, 0.090520581f);
    q = fmaf(q, t, 0.11733179f);
    q = fmaf(q, t, 0.1316339f);
    q = fmaf(q, t, 0.1316516f);
    const float low = e * t * q, f = g < 0.0f ? low : 1.0f - low;
    return Act{g * f, fmaf(0.39894228f * g, e, f)};
  }
}

// Tiles of kT rows and kT columns, kT / 2 of gate and as many of the up projection.  kOnce: the
// weights are read past the caches.
template <int kT, bool kOnce>
struct GatedTile {
  static constexpr int kHidden = kT / 2;
  using D = mm::Depth<false, false, kT>;
  using T = mm::Tile<Bf16, false, false, kT, kT, 2, D::kStep, D::kStages, false,
                     mm::PairedOperand<Bf16, kT, D::kStep, kOnce>>;
};

template <int kAct, bool kKeep, int kT, Share kShare, bool kOnce>
__global__ __launch_bounds__(mm::kThreads, (mm::Depth<false, false, kT>::kPerCu)) void k9_linear(
    const GatedLinear a) {
  using G = GatedTile<kT, kOnce>;
  using T = typename G::T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_row_tile<kT, kShare>(a.g, a.tiles_n, blockIdx.x, lane, &t)) return;
  const int h0 = t.tn * G::kHidden;
  if (kShare == kRest && h0 >= a.H) return;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(a.x + int64_t(t.row) * a.x_stride, a.x_stride * 2, t.rows, wave, lane);
  const int64_t half = int64_t(a.H) * a.K;
  const uint16_t* w = a.w + (t.group < a.g.num ? t.group * 2 * half : 0);
  on.at(w + int64_t(h0) * a.K, half * 2, int64_t(a.K) * 2, a.H - h0, wave, lane);
  T::product(acc, om, on, t.group < a.g.num ? a.K : 0, wave, lane);
  if constexpr (kKeep) {
    T::out16(
        acc, wave, lane,
        [](int, int, float a0, float a1, float a2, float a3) {
          return u32x2{pack(a0, a1), pack(a2, a3)};
        },
        [&](int m, int n, const u32x4& v) {
          const int j = h0 + (n >> 5) * 16 + (n & 15);
          if (m < t.rows && j < a.H)
            put(reinterpret_cast<u32x4*>(a.pre + int64_t(t.row + m) * a.pre_stride +
                                         (n & 16 ? a.H : 0) + j), v, a.past);
        });
  }
  T::out16_joined(
      acc, wave, lane,
      [](const f32x4& g, const f32x4& u) {
        f32x4 h;
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = act<kAct>(g[k]).value * u[k];
        return pack(h);
      },
      [&](int m, int n, const u32x4& v) {
        if (m < t.rows && h0 + n < a.H)
          put(reinterpret_cast<u32x4*>(a.h + int64_t(t.row + m) * a.h_stride + h0 + n), v, a.past);
      });
}

// 16-byte chunk c of row r of a part of rows of kRowBytes staged in LDS: rows start in other banks.
template <int kRowBytes>
__device__ __forceinline__ char* chunk(char* at, int r, int c) {
  return at + r * kRowBytes + 16 * (c ^ (r & (kRowBytes / 16 - 1)));
}

// The same with the tiles of a compute unit one after the other (mm_stream.h); K a multiple of 64.
template <int kAct, bool kKeep, bool kPast>
__global__ __launch_bounds__(mm::kThreads, 1) void k9_linear_stream(const GatedLinear a) {
  using T = mm::Tile<Bf16, false, false, kStreamM, kStreamN, 2, 128, 3, false,
                     mm::PairedOperand<Bf16, kStreamN, 128>>;
  constexpr int kHidden = kStreamN / 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t half = int64_t(a.H) * a.K;
  auto place = [&](const RowTile& t, typename T::OpM* om, typename T::OpN* on) {
    const int h0 = t.tn * kHidden;
    const bool owned = t.group < a.g.num;
    om->at(a.x + int64_t(t.row) * a.x_stride, a.x_stride * 2, t.rows, wave, lane);
    on->at(a.w + (owned ? t.group * 2 * half : 0) + int64_t(h0) * a.K, half * 2, int64_t(a.K) * 2,
           a.H - h0, wave, lane);
    return owned;
  };
  const int m0 = T::first_row(wave), n0 = T::first_col(wave);
  auto out = [&](const typename T::Acc(&acc)[T::kBM][T::kBN], const RowTile& t, char* lds) {
    const int h0 = t.tn * kHidden;
    auto four = [&](int i, int j, int g) {
      const typename T::Acc& v = acc[i][j];
      return f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
    };
#pragma unroll
    for (int i = 0; i < T::kBM; ++i) {
      const int row = lane & 31;
      if constexpr (kKeep) {
#pragma unroll
        for (int j = 0; j < T::kBN; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<u32x2*>(chunk<256>(lds, row, 4 * j + g) + 8 * (lane >> 5)) =
                pack(four(i, j, g));
        mm::lanes_meet();
        char* const to = reinterpret_cast<char*>(a.pre + int64_t(t.row) * a.pre_stride + h0);
#pragma unroll
        for (int r = 0; r < 32; r += 4) {
          const int m = m0 + 32 * i + r + lane / 16, n = n0 + 8 * (lane & 15);
          const int col = (n >> 5) * 16 + (n & 15);
          mm::store_if<kPast>(to, m < t.rows && h0 + col < a.H,
                              2 * (uint32_t(m) * uint32_t(a.pre_stride) + (n & 16 ? a.H : 0) + col),
                              *reinterpret_cast<const u32x4*>(chunk<256>(lds, r + lane / 16, lane & 15)));
        }
        mm::lanes_meet();
      }
#pragma unroll
      for (int j = 0; j < T::kBN; ++j)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const f32x4 gate = four(i, j, g), up = four(i, j, g + 2);
          f32x4 h;
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = act<kAct>(gate[k]).value * up[k];
          *reinterpret_cast<u32x2*>(chunk<128>(lds, row, 2 * j + g) + 8 * (lane >> 5)) = pack(h);
        }
      mm::lanes_meet();
      char* const to = reinterpret_cast<char*>(a.h + int64_t(t.row) * a.h_stride + h0);
#pragma unroll
      for (int r = 0; r < 32; r += 8) {
        const int m = m0 + 32 * i + r + lane / 8, col = n0 / 2 + 8 * (lane & 7);
        mm::store_if<kPast>(to, m < t.rows && h0 + col < a.H,
                            2 * (uint32_t(m) * uint32_t(a.h_stride) + col),
                            *reinterpret_cast<const u32x4*>(chunk<128>(lds, r + lane / 8, lane & 7)));
      }
      mm::lanes_meet();
    }
  };
  mm::stream<T, T::kBM * (kKeep ? 12 : 4)>(a.g, a.tiles_n, a.K, wave, lane, place, [](const RowTile&) {}, out);
}

template <int kAct, bool kPast>
__global__ __launch_bounds__(mm::kThreads, 1) void k9_dgrad_stream(const GatedDgrad a) {
  using T = mm::Tile<Bf16, false, true, kStreamM, kStreamN, 2, 128, 3>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto place = [&](const RowTile& t, typename T::OpM* om, typename T::OpN* on) {
    const int n0 = t.tn * kStreamN;
    const bool owned = t.group < a.g.num;
    om->at(a.dy + int64_t(t.row) * a.dy_stride, a.dy_stride * 2, t.rows, wave, lane);
    on->at(a.w + (owned ? int64_t(t.group) * a.H * a.K : 0) + n0, int64_t(a.H) * 2, a.H - n0, wave,
           lane);
    return owned;
  };
  // The wavefront's part of d goes out in parts of 32 x 64; a lane has eight columns of four rows of
  // a part, whose p is on its way while the part before goes out.
  constexpr int kParts = 2 * T::kBM, kPieces = 4;
  u32x4 gate[2][kPieces], up[2][kPieces];
  auto row = [&](int part, int q) {
    return T::first_row(wave) + 32 * (part >> 1) + 8 * q + lane / 8;
  };
  auto col = [&](int part) { return T::first_col(wave) + 64 * (part & 1) + 8 * (lane & 7); };
  auto fetch = [&](const RowTile& t, int part) {
    // (rows and columns past the last ones read those)
    const int n = min(t.tn * kStreamN + col(part), a.H - 8);
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      const uint16_t* p =
          a.pre + int64_t(t.row + min(row(part, q), t.rows - 1)) * a.pre_stride + n;
      gate[part & 1][q] = *reinterpret_cast<const u32x4*>(p);
      up[part & 1][q] = *reinterpret_cast<const u32x4*>(p + a.H);
    }
  };
  auto out = [&](const typename T::Acc(&acc)[T::kBM][T::kBN], const RowTile& t, char* lds) {
    // rows of nobody get 0, whatever their p holds
    const uint32_t kept = t.group < a.g.num ? 0xFFFFFFFFu : 0u;
    const int n0 = t.tn * kStreamN;
    char* const to = reinterpret_cast<char*>(a.dpre + int64_t(t.row) * a.dpre_stride + n0);
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      if (part + 1 < kParts) fetch(t, part + 1);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const typename T::Acc& v = acc[part >> 1][2 * (part & 1) + j];
          *reinterpret_cast<f32x4*>(chunk<256>(lds, lane & 31, 8 * j + 2 * g + (lane >> 5))) =
              f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
        }
      mm::lanes_meet();
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {
        const u32x4 pg = gate[part & 1][q], pu = up[part & 1][q];
        u32x4 dg, du;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const f32x4 d = *reinterpret_cast<const f32x4*>(
              chunk<256>(lds, 8 * q + lane / 8, 2 * (lane & 7) + k));
          const f32x4 g = four(u32x2{pg[2 * k], pg[2 * k + 1]}), u = four(u32x2{pu[2 * k], pu[2 * k + 1]});
          f32x4 vg, vu;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const Act f = act<kAct>(g[e]);
            vg[e] = d[e] * f.slope * u[e];
            vu[e] = d[e] * f.value;
          }
          const u32x2 of_gate = pack(vg) & kept, of_up = pack(vu) & kept;
          dg[2 * k] = of_gate.x;
          dg[2 * k + 1] = of_gate.y;
          du[2 * k] = of_up.x;
          du[2 * k + 1] = of_up.y;
        }
        const int m = row(part, q), n = col(part);
        const bool there = m < t.rows && n0 + n < a.H;
        const uint32_t offset = 2 * (uint32_t(m) * uint32_t(a.dpre_stride) + n);
        mm::store_if<kPast>(to, there, offset, dg);
        mm::store_if<kPast>(to, there, offset + 2 * uint32_t(a.H), du);
      }
      mm::lanes_meet();
    }
  };
  mm::stream<T, 2 * kParts * kPieces>(a.g, a.tiles_n, a.K, wave, lane, place,
                                      [&](const RowTile& t) { fetch(t, 0); }, out);
}

template <int kAct, int kT, Share kShare>
__global__ __launch_bounds__(mm::kThreads, (mm::Depth<false, true, kT>::kPerCu)) void k9_dgrad(
    const GatedDgrad a) {
  using D = mm::Depth<false, true, kT>;
  using T = mm::Tile<Bf16, false, true, kT, kT, 2, D::kStep, D::kStages>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_row_tile<kT, kShare>(a.g, a.tiles_n, blockIdx.x, lane, &t)) return;
  const int n0 = t.tn * kT;
  if (kShare == kRest && n0 >= a.H) return;
  const bool owned = t.group < a.g.num;
  typename T::Acc acc[T::kBM][T::kBN];
  typename T::OpM om;
  typename T::OpN on;
  om.at(a.dy + int64_t(t.row) * a.dy_stride, a.dy_stride * 2, t.rows, wave, lane);
  const uint16_t* w = a.w + (owned ? int64_t(t.group) * a.H * a.K : 0);
  on.at(w + n0, int64_t(a.H) * 2, a.H - n0, wave, lane);
  T::product(acc, om, on, owned ? a.K : 0, wave, lane);
  struct Pair {
    u32x2 gate, up;
  };
  // (rows and columns past the last ones read those)
  const int col = n0 + T::col(wave, lane), edge = min(col, a.H - 4);
  T::out32(
      acc, wave, lane,
      [&](int q) {
        const uint16_t* p =
            a.pre + int64_t(t.row + min(T::row(q, wave, lane), t.rows - 1)) * a.pre_stride + edge;
        return Pair{*reinterpret_cast<const u32x2*>(p), *reinterpret_cast<const u32x2*>(p + a.H)};
      },
      [&](int q, const f32x4& d, const Pair& was) {
        const int row = T::row(q, wave, lane);
        if (row >= t.rows || col >= a.H) return;
        const f32x4 g = four(was.gate), u = four(was.up);
        f32x4 dg, du;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const Act f = act<kAct>(g[k]);
          // rows of nobody get 0, whatever their p holds
          dg[k] = owned ? d[k] * f.slope * u[k] : 0.0f;
          du[k] = owned ? d[k] * f.value : 0.0f;
        }
        uint16_t* p = a.dpre + int64_t(t.row + row) * a.dpre_stride + col;
        put(reinterpret_cast<u32x2*>(p), pack(dg), a.past);
        put(reinterpret_cast<u32x2*>(p + a.H), pack(du), a.past);
      });
}

// 64 rows x 512 columns to a workgroup, eight values to a lane.
constexpr int kActRows = 64, kActCols = 512;
template <int kAct>
__global__ __launch_bounds__(256) void k9_activation(const GatedActivation a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_row_tile<kActRows, kAll>(a.g, a.tiles_n, blockIdx.x, lane, &t)) return;
  const int col = t.tn * kActCols + 8 * lane;
  if (col >= a.H) return;
  const bool owned = t.group < a.g.num;
  const int rows = min(t.rows, kActRows);
#pragma unroll 4
  for (int r = wave; r < rows; r += 4) {
    const uint16_t* p = a.pre + int64_t(t.row + r) * a.pre_stride + col;
    const u32x4 g = *reinterpret_cast<const u32x4*>(p);
    const u32x4 u = *reinterpret_cast<const u32x4*>(p + a.H);
    u32x4 h;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f32x4 gate = four(u32x2{g[2 * k], g[2 * k + 1]}), up = four(u32x2{u[2 * k], u[2 * k + 1]});
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = owned ? act<kAct>(gate[i]).value * up[i] : 0.0f;
      const u32x2 two = pack(v);
      h[2 * k] = two.x;
      h[2 * k + 1] = two.y;
    }
    *reinterpret_cast<u32x4*>(a.h + int64_t(t.row + r) * a.h_stride + col) = h;
  }
}

template <int kAct, bool kKeep>
void launch_linear_of(GatedLinear a, hipStream_t s) {
  a.past = past_caches(a.g.rows, int64_t(a.H) * (kKeep ? 3 : 1));
  if (gated_linear_streams(a.g, a.H, a.K, kKeep)) {
    a.tiles_n = (2 * a.H + kStreamN - 1) / kStreamN;
    const dim3 grid(mm::kStreamWorkgroups), block(mm::kThreads);
    if (a.past) hipLaunchKernelGGL((k9_linear_stream<kAct, kKeep, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k9_linear_stream<kAct, kKeep, false>), grid, block, 0, s, a);
    return;
  }
  auto launch = [&](auto edge, auto share, int64_t wgs) {
    constexpr int kT = decltype(edge)::value;
    auto of = [&](auto once) {
      hipLaunchKernelGGL((k9_linear<kAct, kKeep, kT, decltype(share)::value,
                                    kT == 64 && decltype(once)::value>),
                         dim3(unsigned(wgs)), dim3(mm::kThreads), 0, s, a);
    };
    if (kT == 64 && gated_weights_once(a.g)) of(std::true_type{});
    else of(std::false_type{});
  };
  launch_row_tiles(a.g, 2 * a.H, a.K, 2, &a.tiles_n, launch);
}

template <int kAct>
void launch_dgrad_of(GatedDgrad a, hipStream_t s) {
  a.past = past_caches(a.g.rows, 2 * int64_t(a.H));
  if (gated_dgrad_streams(a.g, a.H, a.K)) {
    a.tiles_n = (a.H + kStreamN - 1) / kStreamN;
    const dim3 grid(mm::kStreamWorkgroups), block(mm::kThreads);
    if (a.past) hipLaunchKernelGGL((k9_dgrad_stream<kAct, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k9_dgrad_stream<kAct, false>), grid, block, 0, s, a);
    return;
  }
  auto launch = [&](auto edge, auto share, int64_t wgs) {
    hipLaunchKernelGGL((k9_dgrad<kAct, decltype(edge)::value, decltype(share)::value>),
                       dim3(unsigned(wgs)), dim3(mm::kThreads), 0, s, a);
  };
  launch_row_tiles(a.g, a.H, a.K, 2, &a.tiles_n, launch, kGatedDgradBeside);
}

}  // namespace

int64_t gated_workgroups(const GroupArgs& g, int32_t hidden) {
  return most_row_tiles(g, 64) * ((2 * int64_t(hidden) + 63) / 64);
}

hipError_t launch_gated_linear(const GatedLinear& a, int32_t activation, hipStream_t s) {
  const bool keep = a.pre != nullptr;
  if (activation == GNMR_ACT_SILU)
    keep ? launch_linear_of<GNMR_ACT_SILU, true>(a, s) : launch_linear_of<GNMR_ACT_SILU, false>(a, s);
  else
    keep ? launch_linear_of<GNMR_ACT_GELU, true>(a, s) : launch_linear_of<GNMR_ACT_GELU, false>(a, s);
  return hipGetLastError();
}

hipError_t launch_gated_dgrad(const GatedDgrad& a, int32_t activation, hipStream_t s) {
  if (activation == GNMR_ACT_SILU) launch_dgrad_of<GNMR_ACT_SILU>(a, s);
  else launch_dgrad_of<GNMR_ACT_GELU>(a, s);
  return hipGetLastError();
}

hipError_t launch_gated_activation(GatedActivation a, int32_t activation, hipStream_t s) {
  a.tiles_n = (a.H + kActCols - 1) / kActCols;
  const dim3 grid(unsigned(most_row_tiles(a.g, kActRows) * a.tiles_n));
  if (activation == GNMR_ACT_SILU)
    hipLaunchKernelGGL(k9_activation<GNMR_ACT_SILU>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k9_activation<GNMR_ACT_GELU>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace gnmr
