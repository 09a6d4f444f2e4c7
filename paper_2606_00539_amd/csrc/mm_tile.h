// One output tile of a matrix product on the CDNA4 matrix cores, shared by K6
// (grouped products), K7 (INT8) and K8 (orthogonalisation):
//
//   acc(m, n) = sum_k M(m, k) * N(n, k)        m < kTM, n < kTN
//
// Each operand lies in memory either with k contiguous ("rows", one row per m or
// n) or with k as the slow index ("cols", one row per k).  16-bit floats or
// 8-bit integers; sums in fp32 or int32.
//
// Operands go from memory to LDS without passing registers
// (global_load_lds, 16 bytes a lane): a wavefront's instruction fills 1 KiB of
// LDS in lane order, so the bank swizzle is applied to the address that a lane
// reads from.  A K step is 128 bytes of a "rows" operand (64 16-bit values, 128
// 8-bit ones).  kStages steps are in LDS at a time; a step's barrier stands before
// its last slot, and behind it the step kStages ahead is requested into the
// buffer that the workgroup has just finished reading.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace gnmr {
namespace mm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  typedef bf16x8 Frag;
  typedef f32x16 Acc;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ Acc mfma(Frag a, Frag b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
struct F16 {
  typedef f16x8 Frag;
  typedef f32x16 Acc;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ Acc mfma(Frag a, Frag b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
struct Int8 {
  typedef i32x4 Frag;
  typedef i32x16 Acc;
  static constexpr int kBytes = 1;
  static __device__ __forceinline__ Acc mfma(Frag a, Frag b, Acc c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
  }
};

constexpr int kThreads = 256, kWaves = 4;
constexpr int kStepBytes = 128;  // of a "rows" operand
constexpr int kSlots = 4;        // matrix-core instructions deep

// s_waitcnt vmcnt(n), nothing else waited for
template <int n>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14));
}

// The workgroup's barrier, with this wavefront's LDS reads done; loads to LDS stay in flight.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One operand of a tile: kT rows (m or n) of which `rows` exist.
template <class E, bool kCols, int kT>
struct Operand {
  static_assert(!kCols || E::kBytes == 2, "k as the slow index: 16-bit types only");
  static_assert(!kCols || kT >= 128, "the swizzle of a cols operand takes eight units a row");
  static constexpr int kStepK = kStepBytes / E::kBytes;    // k per step
  static constexpr int kBytes = kT * kStepBytes;           // of a stage in LDS
  static constexpr int kLoads = kBytes / 1024 / kWaves;    // instructions per wavefront and step
  static constexpr int kRowBytes = kCols ? kT * 2 : kStepBytes;

  const char* base;   // element (row 0, k 0) of the tile
  int64_t step;       // bytes between K steps
  uint32_t ld;        // bytes between memory rows
  uint32_t off[kLoads];

  // 32-byte units of a cols row: the four k rows and two units that 32 lanes of a
  // transposing read touch lie in different banks.
  static __device__ __forceinline__ int swizzle(int k) {
    return (2 * (k & 3)) ^ ((k >> 1) & 1);
  }

  __device__ __forceinline__ void at(const void* p, int64_t ld_bytes, int rows, int wave, int lane) {
    base = static_cast<const char*>(p);
    ld = uint32_t(ld_bytes);
    step = kCols ? int64_t(kStepK) * ld_bytes : kStepBytes;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) off[q] = offset(q, rows, wave, lane);
  }

  // Byte offset from the step's base of what lane `lane` brings with instruction q.
  // Rows past the last read the last one: nothing of theirs is used.
  __device__ __forceinline__ uint32_t offset(int q, int rows, int wave, int lane) const {
    const int first = wave * kLoads + q;  // 1 KiB piece
    if constexpr (kCols) {
      constexpr int kChunks = kT / 8, kPer = 64 / kChunks;
      const int k = first * kPer + lane / kChunks, slot = lane % kChunks;
      const int col = 8 * (2 * ((slot >> 1) ^ swizzle(k)) + (slot & 1));
      return uint32_t(k) * ld + 2u * uint32_t(col < rows - 8 ? col : rows - 8);
    } else {
      const int row = first * 8 + (lane >> 3);
      return uint32_t(row < rows ? row : rows - 1) * ld + 16u * ((lane & 7) ^ (lane >> 3));
    }
  }

  // Requests step s into `lds`.
  __device__ __forceinline__ void request(char* lds, int64_t s, int wave) const {
    const char* p = base + s * step;
#pragma unroll
    for (int q = 0; q < kLoads; ++q)
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(p + off[q]),
          (__attribute__((address_space(3))) void*)(lds + (wave * kLoads + q) * 1024), 16, 0, 0);
  }

  // Step s, of which only `left` values of k exist, the others zero.
  __device__ __forceinline__ void fill(char* lds, int64_t s, int left, int wave, int lane) const {
    const char* p = base + s * step;
    u32x4 v[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      v[q] = u32x4{0, 0, 0, 0};
      if constexpr (kCols) {
        const int k = (wave * kLoads + q) * (64 / (kT / 8)) + lane / (kT / 8);
        if (k < left) v[q] = *reinterpret_cast<const u32x4*>(p + off[q]);
      } else {
        // rows are multiples of 8 values long: of 8-bit ones, a chunk may be half there
        constexpr int kPer = 16 / E::kBytes;
        const int k = kPer * ((lane & 7) ^ (lane >> 3));
        if (k + kPer <= left) {
          v[q] = *reinterpret_cast<const u32x4*>(p + off[q]);
        } else if (k < left) {
          const u32x2 h = *reinterpret_cast<const u32x2*>(p + off[q]);
          v[q] = u32x4{h.x, h.y, 0, 0};
        }
      }
    }
#pragma unroll
    for (int q = 0; q < kLoads; ++q)
      *reinterpret_cast<u32x4*>(lds + (wave * kLoads + q) * 1024 + lane * 16) = v[q];
  }
};

// Fragments of kB 32-row blocks from row `first` of an operand's stage.
template <class E, bool kCols, int kT, int kB>
struct Reader {
  typedef typename E::Frag Frag;
  uint32_t addr[kCols ? kB : kSlots];

  __device__ __forceinline__ void at(int first, int lane) {
    if constexpr (kCols) {
      const int j = (lane & 15) >> 2, k = 8 * (lane >> 5) + j;
      const int s = Operand<E, true, kT>::swizzle(j);
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const int unit = ((first + 32 * b) >> 4) + ((lane >> 4) & 1);
        addr[b] = k * kT * 2 + 32 * (unit ^ s) + 8 * (lane & 3);
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < kSlots; ++kk)
        addr[kk] = (first + (lane & 31)) * kStepBytes + 16 * ((2 * kk + (lane >> 5)) ^ (lane & 7));
    }
  }

  __device__ __forceinline__ Frag get(const char* lds, int kk, int b) const {
    if constexpr (kCols) {
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      const char* p = lds + addr[b] + kk * 16 * kT * 2;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * kT * 2));
      return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *reinterpret_cast<const Frag*>(lds + addr[kk] + b * 32 * kStepBytes);
    }
  }
};

// kTM x kTN tiles by kWM x (4 / kWM) wavefronts.
template <class E, bool kColsM, bool kColsN, int kTM, int kTN, int kWM, int kStages>
struct Tile {
  static constexpr int kWN = kWaves / kWM;
  static constexpr int kWaveM = kTM / kWM, kWaveN = kTN / kWN;  // a wavefront's part
  static constexpr int kBM = kWaveM / 32, kBN = kWaveN / 32;
  typedef Operand<E, kColsM, kTM> OpM;
  typedef Operand<E, kColsN, kTN> OpN;
  static constexpr int kStepK = OpM::kStepK;
  static constexpr int kStage = OpM::kBytes + OpN::kBytes;
  typedef typename E::Acc Acc;
  static_assert(kStages >= 2 && kStages <= 4, "stages");

  // K values, of which K % kStepK ones are taken first: their step has to be filled
  // through registers, and there that costs least.
  // kSwap: registers hold four rows of a column instead of four columns of a row.
  template <bool kSwap = false>
  static __device__ __forceinline__ void product(Acc (&acc)[kBM][kBN], const OpM& om, const OpN& on,
                                                 int64_t K, int wave, int lane) {
    // (distinct variables: the compiler then knows which loads a read has to wait for)
    __shared__ __attribute__((aligned(16))) char s0[kStage];
    __shared__ __attribute__((aligned(16))) char s1[kStage];
    __shared__ __attribute__((aligned(16))) char s2[kStages > 2 ? kStage : 16];
    __shared__ __attribute__((aligned(16))) char s3[kStages > 3 ? kStage : 16];
    auto stage = [&](auto i) -> char* {
      constexpr int k = decltype(i)::value % kStages;
      if constexpr (k == 0) return s0;
      else if constexpr (k == 1) return s1;
      else if constexpr (k == 2) return s2;
      else return s3;
    };
#pragma unroll
    for (int i = 0; i < kBM; ++i)
#pragma unroll
      for (int j = 0; j < kBN; ++j) acc[i][j] = Acc{};
    const int64_t full = K / kStepK;
    const int left = int(K - full * kStepK);
    const int64_t nk = full + (left > 0 ? 1 : 0);
    if (nk == 0) return;
    constexpr int kLoads = OpM::kLoads + OpN::kLoads;

    Reader<E, kColsM, kTM, kBM> rm;
    Reader<E, kColsN, kTN, kBN> rn;
    rm.at((wave / kWN) * kWaveM, lane);
    rn.at((wave % kWN) * kWaveN, lane);
    typename E::Frag fm[2][kBM], fn[2][kBN];
    auto read = [&](int set, const char* st, int kk) {
#pragma unroll
      for (int b = 0; b < kBM; ++b) fm[set][b] = rm.get(st, kk, b);
#pragma unroll
      for (int b = 0; b < kBN; ++b) fn[set][b] = rn.get(st + OpM::kBytes, kk, b);
    };
    auto mfma = [&](int set) {
#pragma unroll
      for (int i = 0; i < kBM; ++i)
#pragma unroll
        for (int j = 0; j < kBN; ++j) 
          acc[i][j] = kSwap ? E::mfma(fm[set][i], fn[set][j], acc[i][j])
                            : E::mfma(fn[set][j], fm[set][i], acc[i][j]);
    };
    // Memory order of the steps: the partial one first, then 0, 1, ...
    const int64_t shift = left > 0 ? -1 : 0;
    auto request = [&](char* st, int64_t s) {
      om.request(st, s + shift, wave);
      on.request(st + OpM::kBytes, s + shift, wave);
    };
    using std::integral_constant;
    if (left == 0) request(s0, 0);
    if (nk > 1) request(s1, 1);
    if constexpr (kStages > 2)
      if (nk > 2) request(s2, 2);
    if constexpr (kStages > 3)
      if (nk > 3) request(s3, 3);
    if (left > 0) {
      om.fill(s0, full, left, wave, lane);
      on.fill(s0 + OpM::kBytes, full, left, wave, lane);
    }
    wait_loads<0>();
    meet();
    read(0, s0, 0);

    auto one = [&](int64_t s, auto u) {
      char* const cur = stage(u);
      char* const nxt = stage(integral_constant<int, decltype(u)::value + 1>{});
      read(1, cur, 1);
      mfma(0);
      read(0, cur, 2);
      mfma(1);
      read(1, cur, 3);
      mfma(0);
      __builtin_amdgcn_sched_barrier(0);
      // step s+1 has landed (the steps behind it may still be under way)
      if (kStages > 2 && s + kStages - 1 < nk) wait_loads<(kStages - 2) * kLoads>();
      else wait_loads<0>();
      meet();
      __builtin_amdgcn_sched_barrier(0);
      if (s + kStages < nk) request(cur, s + kStages);
      if (s + 1 < nk) read(0, nxt, 0);
      mfma(1);
    };
    for (int64_t s = 0; s < nk; s += kStages) {
      one(s, integral_constant<int, 0>{});
      if (s + 1 >= nk) break;
      one(s + 1, integral_constant<int, 1>{});
      if constexpr (kStages > 2) {
        if (s + 2 >= nk) break;
        one(s + 2, integral_constant<int, 2>{});
      }
      if constexpr (kStages > 3) {
        if (s + 3 >= nk) break;
        one(s + 3, integral_constant<int, 3>{});
      }
    }
  }

  // fn(i, j, g, m, n): accumulator registers 4g .. 4g+3 of block (i, j) are row m,
  // columns n .. n+3 of the tile (kSwap: column n, rows m .. m+3).
  template <bool kSwap = false, class Fn>
  static __device__ __forceinline__ void each(int wave, int lane, Fn&& fn) {
    const int a = lane & 31, b = 4 * (lane >> 5);
    const int m0 = (wave / kWN) * kWaveM + (kSwap ? b : a);
    const int n0 = (wave % kWN) * kWaveN + (kSwap ? a : b);
#pragma unroll
    for (int i = 0; i < kBM; ++i)
#pragma unroll
      for (int j = 0; j < kBN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          fn(i, j, g, m0 + 32 * i + (kSwap ? 8 * g : 0), n0 + 32 * j + (kSwap ? 0 : 8 * g));
  }
};

}  // namespace mm
}  // namespace gnmr
