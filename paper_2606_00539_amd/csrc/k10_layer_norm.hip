// K10: layer norm of rows and its gradients, in fp32:
//
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), y = (x - m) r w + b
//   g = dy w, z = (x - m) r:  dx = r (g - mean(g) - z mean(g z)),
//   dw = sum over rows of dy z,  db = sum over rows of dy
//
// A row is held in registers by 8 to 64 lanes, or by a workgroup's wavefronts: it is read once.  Its
// mean is first taken in fp32 and then corrected by the mean of what is left, since where the mean is
// much larger than the deviations its rounding alone would show in x - m; the gradients' kernel does
// the same with the mean that it is given.  Both kernels take rows by turns, weights in registers and
// the next row on its way; the gradients' keeps its columns' sums over its rows in registers too.
//
// Bound by the rows' bytes.  42M values, TB/s of forward and gradients: fp32 6.0 to 6.5 and 5.3 to 6.0 at widths
// from 768 to 11,008 (odd ones 4.8 and 5.5), bf16 3.7 to 4.6 and 3.4 to 4.9 (odd ones 3.4 and 2.4), where the
// conversions, the gradients' sums and the comparisons of incomplete rows take as long as the bytes.
//
// Of the gradients' shapes two spill: two whole runs of bf16 six registers, outside of any loop, and fp32 rows
// of more than 8,192 columns in part three, of which a row reads two back.
#include <algorithm>

#include "gnmr_internal.h"
#include "lane_ops.h"
#include "values.h"

namespace gnmr {
namespace {

// How a row is held: by kLanes lanes of a wavefront (8 to 64, several rows to a wavefront or
// workgroup), or, kWide, by all lanes of `waves` wavefronts, as many as it needs; kEight runs of eight
// bf16 values (twice as many of four fp32 ones) to a lane.  kFill: what cols fills of them, kAll (kExact),
// kWhole runs, or one of them in part.
// kPast: the result is written past the caches.
enum Fill { kPart, kWhole, kAll };
template <bool kIsF32, int kLaneCount, bool kIsWide, int kEight, int kFilled, bool kIsPast = false>
struct Shape {
  static constexpr bool kF32 = kIsF32, kWide = kIsWide, kExact = kFilled == kAll, kPast = kIsPast;
  static constexpr int kFill = kFilled;
  static constexpr int kLanes = kLaneCount, N = kF32 ? 4 : 8, kRuns = kF32 ? 2 * kEight : kEight;
  static constexpr int kBytes = kF32 ? 4 : 2;
  static constexpr int kMost = kEight == 4 ? 8 : 16;   // wavefronts to a workgroup
  // whether the registers hold the gradients' next row beside the present one
  static constexpr bool kAhead = !(kWide && kEight == 4);
};
constexpr int kThreads = 256;     // of a workgroup of narrow rows
constexpr int kMaxWaves = 16;

// Where a lane is: row `slot` of those that the workgroup takes at a time, run `at` + i * lanes of it.
template <class S>
struct Place {
  int slot, at, lanes;
  int cols;
  int ragged;   // the run that one lane has in part, or -1

  __device__ __forceinline__ Place(int waves, int cols_) : cols(cols_) {
    lanes = S::kWide ? 64 * waves : S::kLanes;
    slot = threadIdx.x / lanes;
    at = threadIdx.x % lanes;
    ragged = cols % S::N != 0 ? cols / S::N / lanes : -1;
  }
  __device__ __forceinline__ int col(int i) const { return S::N * (at + i * lanes); }
  // values of run i that exist
  __device__ __forceinline__ int count(int i) const { return S::kExact ? S::N : cols - col(i); }
  __device__ __forceinline__ bool is(int i, int k) const {
    return S::kExact || col(i) + (S::kFill == kWhole ? 0 : k) < cols;
  }

  // Run i as it lies in memory, in one access whatever of it exists (a branch around loads of single
  // values would wait for them there): a run past the row's end is the row's last N values.
  template <bool kPast>
  __device__ __forceinline__ Raw<S::kF32, S::N> load(const char* row, int i) const {
    if constexpr (S::kExact) return load_raw<S::kF32, S::N, kPast>(row, col(i));
    if (S::kFill == kPart && cols < S::N) return load_raw_some<S::kF32, S::N>(row, col(i), count(i));
    return load_raw<S::kF32, S::N, kPast>(row, min(col(i), cols - S::N));
  }
  // its values; those that do not exist are others
  __device__ __forceinline__ Run<S::N> values(const Raw<S::kF32, S::N>& raw, int i) const {
    Run<S::N> e = raw.values();
    if (S::kFill == kPart && i == ragged && cols >= S::N) {
      const int n = count(i), by = n > 0 && n < S::N ? S::N - n : 0;    // that it was read too early
#pragma unroll
      for (int step = S::N / 2; step > 0; step /= 2)
#pragma unroll
        for (int k = 0; k + step < S::N; ++k)
          if (by & step) e.v[k] = e.v[k + step];
    }
    return e;
  }
  template <bool kPast>
  __device__ __forceinline__ void store(char* row, int i, const Run<S::N>& e) const {
    if (S::kExact || count(i) >= S::N) store_run<S::kF32, S::N, kPast>(row, col(i), e);
    else if (S::kFill == kPart && count(i) > 0) store_some<S::kF32, S::N>(row, col(i), count(i), e);
  }
  // run i of the weights or the biases, of either type, or ones or zeros
  __device__ __forceinline__ Run<S::N> weights(const void* w, bool f32, int i, float none) const {
    Run<S::N> e;
#pragma unroll
    for (int k = 0; k < S::N; ++k) {
      e.v[k] = none;
      if (w != nullptr && is(i, k))
        e.v[k] = f32 ? static_cast<const float*>(w)[col(i) + k]
                     : __uint_as_float(uint32_t(static_cast<const uint16_t*>(w)[col(i) + k]) << 16);
    }
    return e;
  }
};

// Sums of M values over a row's lanes, in each of them.  red: of the row, [M][kMaxWaves], where
// wavefronts leave theirs; between two uses of one lies a barrier of another's.
template <class S, int M>
__device__ __forceinline__ void row_sums(float (&v)[M], int waves, float* red) {
#pragma unroll
  for (int n = 0; n < M; ++n) {
    float s = v[n];
    if constexpr (S::kLanes >= 64) s = add_other<32>(s);
    if constexpr (S::kLanes >= 32) s = add_other<16>(s);
    if constexpr (S::kLanes >= 16) {
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
  if constexpr (S::kWide) {
    const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % waves;
#pragma unroll
    for (int n = 0; n < M; ++n)
      if (lane == 0) red[n * kMaxWaves + wave] = v[n];
    __syncthreads();
    // a lane to a wavefront's sum, in every row of 16 lanes
    const int of = lane & (kMaxWaves - 1);
#pragma unroll
    for (int n = 0; n < M; ++n) {
      float s = of < waves ? red[n * kMaxWaves + of] : 0.0f;
      s = add_other<8>(s);
      s = add_other<4>(s);
      s = add_other<2>(s);
      v[n] = add_other<1>(s);
    }
  }
}

template <class S>
__global__ __launch_bounds__(S::kWide ? 1024 : kThreads) void k10_forward(const LayerNorm a) {
  __shared__ float red[S::kWide ? 2 : 1][S::kWide ? 2 * kMaxWaves : 1];
  const Place<S> p(a.waves, a.cols);
  constexpr int slots = S::kWide ? 1 : kThreads / S::kLanes;
  Run<S::N> w[S::kRuns], b[S::kRuns];
#pragma unroll
  for (int i = 0; i < S::kRuns; ++i) {
    w[i] = p.weights(a.weight, a.weight_f32, i, 1.0f);
    b[i] = p.weights(a.bias, a.weight_f32, i, 0.0f);
  }
  const float n = float(a.cols);
  const int64_t turn = int64_t(gridDim.x) * slots;
  int64_t row = int64_t(blockIdx.x) * slots + p.slot, first = row - p.slot;
  Raw<S::kF32, S::N> next[S::kRuns];
  auto request = [&](int64_t r) {
    // (past the last row: that one again)
    const char* x = static_cast<const char*>(a.x) + min(r, a.rows - 1) * a.x_stride * S::kBytes;
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) next[i] = p.template load<false>(x, i);
  };
  request(row);
  for (; first < a.rows; first += turn, row += turn) {
    Run<S::N> v[S::kRuns];
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) {
      v[i] = p.values(next[i], i);
#pragma unroll
      for (int k = 0; k < S::N; ++k) s[0] += p.is(i, k) ? v[i].v[k] : 0.0f;
    }
    if (first + turn < a.rows) request(row + turn);
    row_sums<S, 1>(s, a.waves, red[0]);
    const float mean = s[0] / n;
    float d[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i)
#pragma unroll
      for (int k = 0; k < S::N; ++k) {
        v[i].v[k] = p.is(i, k) ? v[i].v[k] - mean : 0.0f;
        d[0] += v[i].v[k];
        d[1] = fmaf(v[i].v[k], v[i].v[k], d[1]);
      }
    row_sums<S, 2>(d, a.waves, red[S::kWide ? 1 : 0]);
    const float left = d[0] / n, var = d[1] / n - left * left;
    const float rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + a.eps);
    if (row >= a.rows) continue;
    if (p.at == 0) {
      if (a.mean != nullptr) a.mean[row] = mean + left;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
    char* y = static_cast<char*>(a.y) + row * a.y_stride * S::kBytes;
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) {
#pragma unroll
      for (int k = 0; k < S::N; ++k)
        v[i].v[k] = fmaf((v[i].v[k] - left) * rstd, w[i].v[k], b[i].v[k]);
      p.template store<S::kPast>(y, i, v[i]);
    }
  }
}

// What each workgroup's columns sum to goes to `parts`, [workgroup][dw, db][cols].
template <class S>
__global__ __launch_bounds__(S::kWide ? 64 * S::kMost : kThreads) void k10_backward(const LayerNormBackward a) {
  constexpr int kNarrow = kThreads / S::kLanes;
  __shared__ float red[2][S::kWide ? kMaxWaves * 3 * kMaxWaves : 1];
  __shared__ float sums[S::kWide ? 64 * kMaxWaves * S::N : kThreads * S::N];
  const Place<S> p(a.waves, a.cols);
  const int slots = S::kWide ? int(blockDim.x) / p.lanes : kNarrow;
  const float n = float(a.cols);
  Run<S::N> w[S::kRuns], dw[S::kRuns], db[S::kRuns];
#pragma unroll
  for (int i = 0; i < S::kRuns; ++i) {
    w[i] = p.weights(a.weight, a.weight_f32, i, 1.0f);
#pragma unroll
    for (int k = 0; k < S::N; ++k) dw[i].v[k] = db[i].v[k] = 0.0f;
  }
  const int64_t turn = int64_t(gridDim.x) * slots;
  int64_t row = int64_t(blockIdx.x) * slots + p.slot, first = row - p.slot;
  Raw<S::kF32, S::N> next_x[S::kRuns], next_g[S::kRuns];
  float next_mean, next_rstd;
  auto request = [&](int64_t r) {
    // (past the last row: that one again)
    const int64_t at = min(r, a.rows - 1);
    const char* x = static_cast<const char*>(a.x) + at * a.x_stride * S::kBytes;
    const char* dy = static_cast<const char*>(a.dy) + at * a.dy_stride * S::kBytes;
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) {
      next_x[i] = p.template load<true>(x, i);
      next_g[i] = p.template load<true>(dy, i);
    }
    next_mean = a.mean[at];
    next_rstd = a.rstd[at];
  };
  if (S::kAhead) request(row);
  int use = 0;
  for (; first < a.rows; first += turn, row += turn) {
    if (!S::kAhead) request(row);
    Run<S::N> v[S::kRuns], g[S::kRuns];
    const float mean = next_mean, rstd = next_rstd;
    float s[3] = {0.0f, 0.0f, 0.0f};    // of x - mean, g, g (x - mean)
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) {
      v[i] = p.values(next_x[i], i);
      g[i] = p.values(next_g[i], i);
#pragma unroll
      for (int k = 0; k < S::N; ++k) {
        const float d = p.is(i, k) ? v[i].v[k] - mean : 0.0f;
        g[i].v[k] = p.is(i, k) ? g[i].v[k] : 0.0f;
        const float q = g[i].v[k] * w[i].v[k];
        v[i].v[k] = d;
        s[0] += d;
        s[1] += q;
        s[2] = fmaf(q, d, s[2]);
      }
    }
    if (S::kAhead && first + turn < a.rows) request(row + turn);
    row_sums<S, 3>(s, a.waves, red[use] + (S::kWide ? p.slot * 3 * kMaxWaves : 0));
    use ^= 1;
    if (row >= a.rows) continue;
    const float left = s[0] / n, g1 = s[1] / n, gz = rstd * (s[2] / n - left * g1);
    char* dx = static_cast<char*>(a.dx) + row * a.dx_stride * S::kBytes;
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) {
      Run<S::N> out;
#pragma unroll
      for (int k = 0; k < S::N; ++k) {
        const float z = (v[i].v[k] - left) * rstd, q = g[i].v[k];
        out.v[k] = rstd * (fmaf(q, w[i].v[k], -g1) - z * gz);
        dw[i].v[k] = fmaf(q, z, dw[i].v[k]);
        db[i].v[k] += q;
      }
      if (a.dx != nullptr) p.template store<false>(dx, i, out);
    }
  }
  if (a.parts == nullptr) return;
  // the rows that the workgroup has had at a time, one after the other
  float* to = a.parts + int64_t(blockIdx.x) * 2 * a.cols;
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) {
      Run<S::N> e = which == 0 ? dw[i] : db[i];
      if (slots > 1) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < S::N; ++k) sums[(p.slot * S::N + k) * p.lanes + p.at] = e.v[k];
        __syncthreads();
        if (p.slot == 0) {
#pragma unroll
          for (int k = 0; k < S::N; ++k) e.v[k] = 0.0f;
#pragma unroll 4
          for (int q = 0; q < slots; ++q)
#pragma unroll
            for (int k = 0; k < S::N; ++k) e.v[k] += sums[(q * S::N + k) * p.lanes + p.at];
        }
      }
      if (p.slot == 0) {
#pragma unroll
        for (int k = 0; k < S::N; ++k)
          if (p.is(i, k)) to[which * a.cols + p.col(i) + k] = e.v[k];
      }
    }
}

// dw and db from the workgroups' sums: 64 columns to a workgroup, whose wavefronts take a
// share of the sums each, in order.
constexpr int kReduceWaves = 16;
__global__ __launch_bounds__(64 * kReduceWaves) void k10_reduce(const LayerNormBackward a) {
  __shared__ float red[kReduceWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (a.cols + 63) / 64, which = blockIdx.x / blocks;
  void* out = which == 0 ? a.dweight : a.dbias;
  if (out == nullptr) return;
  const int col = (blockIdx.x % blocks) * 64 + lane;
  const int share = (a.num_parts + kReduceWaves - 1) / kReduceWaves, lo = wave * share,
            hi = min(lo + share, a.num_parts);
  float s = 0.0f;
  if (col < a.cols) {
    const float* p = a.parts + which * a.cols + col;
#pragma unroll 8
    for (int k = lo; k < hi; ++k) s += p[int64_t(k) * 2 * a.cols];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || col >= a.cols) return;
  s = 0.0f;
#pragma unroll
  for (int k = 0; k < kReduceWaves; ++k) s += red[k][lane];
  if (a.weight_f32) store_one<true>(out, col, s);
  else store_one<false>(out, col, s);
}

// launch(lanes, wide, eight, fill): the shape of rows of that many columns.  8192 x 5120 bf16, two
// runs to a lane of five wavefronts: 34 us; one run to ten: 65.  The gradients of 8191 x 4096, one
// run to eight wavefronts: 45 us; two to four: 47.5.  20480 x 2048 bf16, two runs to two wavefronts and,
// gradients, one to four: 37 and 53 us; four runs to one wavefront 63 and 63.
//
// The gradients of bf16 rows that fill two runs of their wavefronts have them where more wavefronts then
// find a place among the workgroup's 16: 8192 x 5120, five to a row and three rows, 56 us; ten and one
// 67.  (Of fp32 they would need more registers than there are: 141 and 84.)
template <bool kBackward, int kFill, class Launch>
void by_width(int cols, bool f32, Launch&& launch) {
  using std::integral_constant;
  using std::bool_constant;
  constexpr int kWave = 512;    // columns that a wavefront holds with one run of eight to a lane
  auto of = [&](auto lanes, auto wide, auto eight) {
    launch(lanes, wide, eight, integral_constant<int, kFill>{});
  };
  const bool_constant<false> narrow;
  const bool_constant<true> wide;
  const integral_constant<int, 1> one;
  const integral_constant<int, 2> two;
  const integral_constant<int, 4> four;
  if (cols <= 64) return of(integral_constant<int, 8>{}, narrow, one);
  if (cols <= 128) return of(integral_constant<int, 16>{}, narrow, one);
  if (cols <= 256) return of(integral_constant<int, 32>{}, narrow, one);
  const integral_constant<int, 64> all;
  if (cols <= kWave) return of(all, narrow, one);
  if (cols <= 2 * kWave) return of(all, narrow, two);
  if constexpr (!kBackward) {
    of(all, wide, two);
  } else {
    auto used = [](int waves) { return waves * (16 / waves); };
    if constexpr (kFill == kAll)
      if (!f32 && cols <= 16 * kWave && cols % (2 * kWave) == 0 &&
          used(cols / (2 * kWave)) > used(cols / kWave))
        return of(all, wide, two);
    if (cols <= 16 * kWave) return of(all, wide, one);
    of(all, wide, four);
  }
}

// Who holds a row: wavefronts to one (1: or a part of it), rows that a workgroup takes at a time, and
// whether a row fills all of their registers.
struct Held {
  int waves, rows;
  bool exact;
};
template <bool kBackward>
Held held(int cols, bool f32) {
  Held r{};
  by_width<kBackward, kAll>(cols, f32, [&](auto lanes, auto wide, auto eight, auto) {
    constexpr int kPer = 8 * decltype(lanes)::value * decltype(eight)::value;
    if (decltype(wide)::value) {
      r.waves = (cols + kPer - 1) / kPer;
      // the gradients' workgroups are as large as may be: fewer sums to add in the end
      r.rows = kBackward ? std::max(1, (decltype(eight)::value == 4 ? 8 : 16) / r.waves) : 1;
    } else {
      r.waves = 1;
      r.rows = kThreads / decltype(lanes)::value;
    }
    r.exact = cols == kPer * r.waves;
  });
  return r;
}

// by_width with what the columns fill of its shape.  Rows of whole runs need one comparison to a run: the
// gradients of 54613 x 768 bf16 73.6 us as rows of runs in part, 57.6 so.
template <bool kBackward, class Launch>
void by_fill(const Held& h, int cols, bool f32, Launch&& launch) {
  if (h.exact) by_width<kBackward, kAll>(cols, f32, launch);
  else if (cols % (f32 ? 4 : 8) == 0) by_width<kBackward, kWhole>(cols, f32, launch);
  else by_width<kBackward, kPart>(cols, f32, launch);
}

}  // namespace

// Workgroups whose sums over their rows are added in the end: one to a CU, or as many as have 64 rows each,
// four to a CU at most and with no more than 8 MB of sums.  us with one and with four to a CU: 4096 x
// 1024 fp32 15.8 and 20.3, 16384 x 1024 bf16 25.7 and 29.1; 65536 x 512 fp32 73.1 and 70.7, 100000 x 128
// fp32 33.2 and 32.1.
int layer_norm_parts(int64_t rows, int cols, bool f32) {
  const Held h = held<true>(cols, f32);
  const int64_t most = h.waves > 1 ? 256 : std::min<int64_t>(rows / 64, std::min(1024, (1 << 20) / cols));
  return int(std::min<int64_t>((rows + h.rows - 1) / h.rows, std::max<int64_t>(256, most)));
}

hipError_t launch_layer_norm(LayerNorm a, bool f32, hipStream_t s) {
  const Held h = held<false>(a.cols, f32);
  a.waves = h.waves;
  const int64_t turns = (a.rows + h.rows - 1) / h.rows;
  // 8192 x 5120 bf16, us, through and past the caches: 39.9 and 34.2 (where they could hold them, what
  // reads the rows next gains more)
  const bool past = a.rows * a.cols * (f32 ? 4 : 2) > int64_t(32) << 20;
  auto launch = [&](auto lanes, auto wide, auto eight, auto fill) {
    constexpr bool kWide = decltype(wide)::value;
    constexpr int kFill = decltype(fill)::value;
    const dim3 block(kWide ? 64 * h.waves : kThreads);
    // 16 wavefronts to a CU, eight workgroups of several rows (8192 x 5120: with 24 wavefronts 50 us
    // instead of 40)
    const dim3 grid{unsigned(std::min<int64_t>(turns, 256 * (kWide ? std::max(1, 16 / h.waves) : 8)))};
    auto of = [&](auto type, auto beyond) {
      hipLaunchKernelGGL((k10_forward<Shape<decltype(type)::value, decltype(lanes)::value, kWide,
                                            decltype(eight)::value, kFill,
                                            decltype(beyond)::value>>),
                         grid, block, 0, s, a);
    };
    auto with = [&](auto type) {
      if (past) of(type, std::true_type{});
      else of(type, std::false_type{});
    };
    if (f32) with(std::true_type{});
    else with(std::false_type{});
  };
  by_fill<false>(h, a.cols, f32, launch);
  return hipGetLastError();
}

hipError_t launch_layer_norm_backward(LayerNormBackward a, bool f32, hipStream_t s) {
  const Held h = held<true>(a.cols, f32);
  a.waves = h.waves;
  a.num_parts = layer_norm_parts(a.rows, a.cols, f32);
  auto launch = [&](auto lanes, auto wide, auto eight, auto fill) {
    constexpr bool kWide = decltype(wide)::value;
    const dim3 block(kWide ? 64 * h.waves * h.rows : kThreads), grid{unsigned(a.num_parts)};
    auto of = [&](auto type) {
      hipLaunchKernelGGL((k10_backward<Shape<decltype(type)::value, decltype(lanes)::value, kWide,
                                             decltype(eight)::value, decltype(fill)::value>>),
                         grid, block, 0, s, a);
    };
    if constexpr (!kWide || decltype(eight)::value != 2)
      if (f32) return of(std::true_type{});
    of(std::false_type{});
  };
  if (a.rows > 0) {
    by_fill<true>(h, a.cols, f32, launch);
  }
  if (a.dweight != nullptr || a.dbias != nullptr)
    hipLaunchKernelGGL(k10_reduce, dim3(unsigned(2 * ((a.cols + 63) / 64))),
                       dim3(64 * kReduceWaves), 0, s, a);
  return hipGetLastError();
}

}  // namespace gnmr
