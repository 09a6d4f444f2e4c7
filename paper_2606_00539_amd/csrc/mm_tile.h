// One output tile of a matrix product on the CDNA4 matrix cores, shared by K6
// (grouped products), K7 (INT8) and K8 (orthogonalisation):
//
//   acc(m, n) = sum_k M(m, k) * N(n, k)        m < kTM, n < kTN
//
// Each operand lies in memory either with k contiguous ("rows", one row per m or
// n) or with k as the slow index ("cols", one row per k).  16-bit floats or
// 8-bit integers; sums in fp32 or int32.
//
// Operands go from memory to LDS without passing registers (buffer loads to LDS,
// 16 bytes a lane): a wavefront's instruction fills 1 KiB of LDS in lane order, so
// the bank swizzle is applied to the address that a lane reads from.  A K step is 64 or 128
// bytes of a "rows" operand (32 or 64 16-bit values).  kStages steps are in LDS at a time.
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
typedef float f32x4 __attribute__((ext_vector_type(4)));
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
constexpr int kBufferWord3 = 0x00020000;  // raw buffers of the gfx9 family

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

// Between what lanes of a wavefront write to LDS and what others of it read there: the hardware
// keeps a wavefront's LDS operations in order, and this keeps the compiler to it.
__device__ __forceinline__ void lanes_meet() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// One operand of a tile: kT rows (m or n) of which `rows` exist.  kStep: bytes of a K
// step in a "rows" operand.
template <class E, bool kCols, int kT, int kStep>
struct Operand {
  static_assert(!kCols || E::kBytes == 2, "k as the slow index: 16-bit types only");
  static_assert(!kCols || kT >= 64, "the swizzle of a cols operand takes four units a row");
  static constexpr int kStepK = kStep / E::kBytes;       // k per step
  static constexpr int kBytes = kT * kStep;              // of a stage in LDS
  static constexpr int kLoads = kBytes / 1024 / kWaves;  // instructions per wavefront and step
  static_assert(kLoads * 1024 * kWaves == kBytes, "whole instructions for each wavefront");
  static constexpr int kChunks = kCols ? kT / 8 : kStep / 16;  // of 16 bytes in a row in LDS
  static constexpr int kPer = 64 / kChunks;                    // such rows per instruction

  const char* base;   // element (row 0, k 0) of the tile
  int64_t step;       // bytes between K steps
  uint32_t ld;        // bytes between memory rows
  uint32_t off[kLoads];

  // 16-byte chunk c of row r of a rows stage lies in place c ^ spread(r): the 16 rows that a
  // read takes a chunk of at a time fill all banks.
  static __device__ __forceinline__ int spread(int row) {
    return (row / (16 / kChunks)) & (kChunks - 1);
  }

  // 32-byte unit u of row k of a cols stage lies in place u ^ swizzle(k): the four k rows and
  // two units that 32 lanes of a transposing read touch fill all banks.
  static __device__ __forceinline__ int swizzle(int k) {
    return kT >= 128 ? (2 * (k & 3)) ^ ((k >> 1) & 1) : k & 2;
  }

  __device__ __forceinline__ void at(const void* p, int64_t ld_bytes, int rows, int wave, int lane) {
    base = static_cast<const char*>(p);
    ld = uint32_t(ld_bytes);
    step = kCols ? int64_t(kStepK) * ld_bytes : kStep;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) off[q] = offset(q, rows, wave, lane);
  }

  // Byte offset from the step's base of what lane `lane` brings with instruction q.
  // Rows past the last read the last one: nothing of theirs is used.
  __device__ __forceinline__ uint32_t offset(int q, int rows, int wave, int lane) const {
    const int row = (wave * kLoads + q) * kPer + lane / kChunks, slot = lane % kChunks;
    if constexpr (kCols) {
      const int col = 8 * (2 * ((slot >> 1) ^ swizzle(row)) + (slot & 1));
      return uint32_t(row) * ld + 2u * uint32_t(col < rows - 8 ? col : rows - 8);
    } else {
      return uint32_t(row < rows ? row : rows - 1) * ld + 16u * (slot ^ spread(row));
    }
  }

  // Requests parts [lo, hi) of step s into `lds`; with `there` false nothing is read (an
  // empty buffer resource), so that the steps behind the last need no branch.
  __device__ __forceinline__ void request(char* lds, int64_t s, bool there, int wave, int lo,
                                          int hi) const {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(base + s * step), 0, there ? 0x7FFFFFFF : 0, kBufferWord3);
#pragma unroll
    for (int q = lo; q < hi; ++q)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          r, (__attribute__((address_space(3))) void*)(lds + (wave * kLoads + q) * 1024), 16,
          off[q], 0, 0, 0);
  }

  // Step s, of which only `left` values of k exist, the others zero.
  __device__ __forceinline__ void fill(char* lds, int64_t s, int left, int wave, int lane) const {
    const char* p = base + s * step;
    u32x4 v[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
      v[q] = u32x4{0, 0, 0, 0};
      const int row = (wave * kLoads + q) * kPer + lane / kChunks;
      if constexpr (kCols) {
        if (row < left) v[q] = *reinterpret_cast<const u32x4*>(p + off[q]);
      } else {
        // rows are multiples of 8 values long: of 8-bit ones, a chunk may be half there
        constexpr int kValues = 16 / E::kBytes;
        const int k = kValues * ((lane % kChunks) ^ spread(row));
        if (k + kValues <= left) {
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
template <class E, bool kCols, int kT, int kStep, int kB>
struct Reader {
  typedef typename E::Frag Frag;
  typedef Operand<E, kCols, kT, kStep> Op;
  static constexpr int kSlots = kStep / 32;
  uint32_t addr[kCols ? kB : kSlots];

  __device__ __forceinline__ void at(int first, int lane) {
    if constexpr (kCols) {
      const int j = (lane & 15) >> 2, k = 8 * (lane >> 5) + j;
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const int unit = ((first + 32 * b) >> 4) + ((lane >> 4) & 1);
        addr[b] = k * kT * 2 + 32 * (unit ^ Op::swizzle(j)) + 8 * (lane & 3);
      }
    } else {
      const int row = first + (lane & 31);
#pragma unroll
      for (int kk = 0; kk < kSlots; ++kk)
        addr[kk] = row * kStep + 16 * ((2 * kk + (lane >> 5)) ^ Op::spread(row));
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
      return *reinterpret_cast<const Frag*>(lds + addr[kk] + b * 32 * kStep);
    }
  }
};

// Stages and the bytes of their steps.  Of a "rows" operand a step takes whole 128-byte
// lines; where both are "cols" finer steps keep more of them under way in the same LDS:
// 8192 x 13824 x 5120, us: rows and rows 863 in two steps of 128 bytes, 965 in four of 64;
// rows and cols 935 and 983; cols and cols 974 and 922.
template <bool kColsM, bool kColsN, int kT>
struct Depth {
  static constexpr int kStep = kColsM && kColsN ? 64 : 128;
  static constexpr int kStages = (kColsM && kColsN) || kT == 64 ? 4 : 2;
  static constexpr int kPerCu = kT == 256 ? 1 : 2;
};

// kTM x kTN tiles by kWM x (4 / kWM) wavefronts.  kSwap: accumulator registers hold
// four rows of a column instead of four columns of a row.
template <class E, bool kColsM, bool kColsN, int kTM, int kTN, int kWM, int kStep, int kStages,
          bool kSwap = false>
struct Tile {
  static constexpr int kWN = kWaves / kWM;
  static constexpr int kWaveM = kTM / kWM, kWaveN = kTN / kWN;  // a wavefront's part
  static constexpr int kBM = kWaveM / 32, kBN = kWaveN / 32;
  typedef Operand<E, kColsM, kTM, kStep> OpM;
  typedef Operand<E, kColsN, kTN, kStep> OpN;
  static constexpr int kStepK = OpM::kStepK;
  static constexpr int kStage = OpM::kBytes + OpN::kBytes;
  typedef typename E::Acc Acc;
  static constexpr int kSlots = kStep / 32;  // matrix-core instructions deep
  static constexpr int kLoads = OpM::kLoads + OpN::kLoads;
  // Requests made in a step's last slot and up to the end of the next one's first.
  static constexpr int kFirst = kSlots == 2 ? kLoads : kLoads * 6 / 16;
  static constexpr int kSecond = kSlots == 2 ? kLoads : kLoads * 12 / 16;
  static_assert(kStages >= 2 && kStages <= 5, "stages");

  // Stage k's memory.  (Distinct variables: the compiler then knows which requests a
  // read has to wait for.)
  template <int k>
  static __device__ __forceinline__ char* stage() {
    __shared__ __attribute__((aligned(16))) char lds[kStage];
    return lds;
  }

  // K values, of which K % kStepK ones are taken first: their step has to be filled
  // through registers, and there that costs least.
  static __device__ __forceinline__ void product(Acc (&acc)[kBM][kBN], const OpM& om, const OpN& on,
                                                 int64_t K, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kBM; ++i)
#pragma unroll
      for (int j = 0; j < kBN; ++j) acc[i][j] = Acc{};
    const int64_t full = K / kStepK;
    const int left = int(K - full * kStepK);
    const int64_t nk = full + (left > 0 ? 1 : 0);
    if (nk == 0) return;

    Reader<E, kColsM, kTM, kStep, kBM> rm;
    Reader<E, kColsN, kTN, kStep, kBN> rn;
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
    // Parts [lo, hi) of the kLoads requests of step s, the M operand's first.
    auto request = [&](char* st, int64_t s, int lo = 0, int hi = kLoads) {
      constexpr int kM = OpM::kLoads;
      if (lo < kM) om.request(st, s + shift, s < nk, wave, lo, hi < kM ? hi : kM);
      if (hi > kM)
        on.request(st + OpM::kBytes, s + shift, s < nk, wave, lo > kM ? lo - kM : 0, hi - kM);
    };
    using std::integral_constant;
    if (left == 0) {
      request(stage<0>(), 0);
    } else {
      om.fill(stage<0>(), full, left, wave, lane);
      on.fill(stage<0>() + OpM::kBytes, full, left, wave, lane);
    }
    // (of the last stage's step only what the step before would have requested)
    auto ahead = [&](auto u) {
      constexpr int k = decltype(u)::value;
      if constexpr (k < kStages) request(stage<k>(), k, 0, k + 1 < kStages ? kLoads : kFirst);
    };
    ahead(integral_constant<int, 1>{});
    ahead(integral_constant<int, 2>{});
    ahead(integral_constant<int, 3>{});
    ahead(integral_constant<int, 4>{});
    wait_loads<(kStages - 2) * kLoads + kFirst>();
    meet();
    read(0, stage<0>(), 0);

    // Instruction order inside a slot (scheduling hints only): the next slot's
    // fragments first, then, in a step's last slot, the requests, spread over the
    // matrix-core instructions.
    constexpr int kMfma = kBM * kBN;
    constexpr int kReads = kBM * (kColsM ? 2 : 1) + kBN * (kColsN ? 2 : 1);
    constexpr int kEach = (kReads + (kMfma + 1) / 2 - 1) / ((kMfma + 1) / 2);
    auto order = [](auto loads) {
      constexpr int kL = decltype(loads)::value, kPer = (kL + kMfma - 1) / kMfma;
#pragma unroll
      for (int i = 0; i < kMfma; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                          // MFMA
        if (i * kEach < kReads) __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);  // LDS read
        if (i * kPer < kL) __builtin_amdgcn_sched_group_barrier(0x020, kPer, 0);     // load
      }
    };
    // The slots of a step: fragments are read a slot ahead, into two sets of registers.
    // Behind the last slot but one nothing of the step's stage is left to read: the workgroup
    // meets there, and the step kStages ahead is requested into that stage.
    auto one = [&](int64_t s, auto u) {
      char* const cur = stage<decltype(u)::value>();
      char* const nxt = stage<(decltype(u)::value + 1) % kStages>();
      char* const old = stage<(decltype(u)::value + kStages - 1) % kStages>();
#pragma unroll
      for (int kk = 0; kk + 1 < kSlots; ++kk) {
        read((kk + 1) & 1, cur, kk + 1);
        if (kk == 0 && kFirst < kLoads) request(old, s + kStages - 1, kFirst, kSecond);
        if (kk == 1 && kSecond < kLoads) request(old, s + kStages - 1, kSecond, kLoads);
        mfma(kk & 1);
        if (kk == 0) order(integral_constant<int, kSecond - kFirst>{});
        else if (kk == 1) order(integral_constant<int, kLoads - kSecond>{});
        else order(integral_constant<int, 0>{});
      }
      __builtin_amdgcn_sched_barrier(0);
      // step s+1 has landed (the steps behind it may still be under way)
      wait_loads<(kStages - 2) * kLoads>();
      meet();
      __builtin_amdgcn_sched_barrier(0);
      request(cur, s + kStages, 0, kFirst);
      read(0, nxt, 0);
      mfma(1);
      order(integral_constant<int, kFirst>{});
    };
    // A round over the stages that has fewer steps left is finished with steps of zeros (what
    // lies past an empty resource arrives as zero): with a way out between its steps the
    // compiler moves accumulators through memory.
#pragma unroll 1
    for (int64_t s = 0; s < nk; s += kStages) {
      one(s, integral_constant<int, 0>{});
      one(s + 1, integral_constant<int, 1>{});
      if constexpr (kStages > 2) {
        one(s + 2, integral_constant<int, 2>{});
      }
      if constexpr (kStages > 3) {
        one(s + 3, integral_constant<int, 3>{});
      }
      if constexpr (kStages > 4) {
        one(s + 4, integral_constant<int, 4>{});
      }
    }
    wait_loads<0>();  // requests behind the last step still write to LDS
  }

  // The wavefront's part of the tile, as it leaves: rows are m (kSwap: n), and the four
  // registers of a group are consecutive columns.
  static constexpr int kRows = kSwap ? kWaveN : kWaveM, kCols = kSwap ? kWaveM : kWaveN;
  // LDS a wavefront has for itself: half of stage 0 or 1, or a stage
  static constexpr int kRegion = kStages < 4 ? kStage / 2 : kStage;

  static __device__ __forceinline__ int first_row(int wave) {
    return kSwap ? (wave % kWN) * kWaveN : (wave / kWN) * kWaveM;
  }
  static __device__ __forceinline__ int first_col(int wave) {
    return kSwap ? (wave / kWN) * kWaveM : (wave % kWN) * kWaveN;
  }
  static __device__ __forceinline__ char* region(int wave) {
    if constexpr (kStages < 4) {
      return (wave & 2 ? stage<1>() : stage<0>()) + (wave & 1) * kRegion;
    } else {
      char* const lo = wave & 1 ? stage<1>() : stage<0>();
      char* const hi = wave & 1 ? stage<3>() : stage<2>();
      return wave & 2 ? hi : lo;
    }
  }

  // 16-byte chunk c of row r of a staged part: rows start in different banks.
  template <int kRowBytes>
  static __device__ __forceinline__ char* chunk(char* at, int r, int c) {
    return at + r * kRowBytes + 16 * (c ^ (r & (kRowBytes / 16 - 1)));
  }

  // 32-row blocks that a region holds at a time: all, a half, a quarter
  static constexpr int pass(int row_bytes) {
    int n = kRows / 32;
    while (n > 1 && n * 32 * row_bytes > kRegion) n /= 2;
    return n;
  }

  // Sends the tile out in whole rows, through LDS: a wavefront's own registers are 32
  // rows of 16 bytes each.  round(j, g, i, row, col, a) makes 16-bit values of the four
  // accumulators a[0..3] at row, col .. col+3 of the tile (two packed words); put(row,
  // col, v) gets eight values of a row at a time (u32x4).
  template <class Round, class Put>
  static __device__ __forceinline__ void out16(const Acc (&acc)[kBM][kBN], int wave, int lane,
                                               Round&& round, Put&& put) {
    constexpr int kRowBytes = kCols * 2, kChunks = kRowBytes / 16, kAtOnce = 64 / kChunks;
    constexpr int kPass = pass(kRowBytes);
    static_assert(kRows / 32 % kPass == 0 && kPass * 32 * kRowBytes <= kRegion, "whole passes");
    char* const at = region(wave);
    const int r0 = first_row(wave), c0 = first_col(wave);
    meet();
#pragma unroll
    for (int p = 0; p < kRows / 32; p += kPass) {
#pragma unroll
      for (int j = 0; j < kCols / 32; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int i = 0; i < kPass; ++i) {
            const int row = 32 * i + (lane & 31), col = 32 * j + 8 * g + 4 * (lane >> 5);
            const Acc& a = kSwap ? acc[j][p + i] : acc[p + i][j];
            const u32x2 v = round(r0 + 32 * p + row, c0 + col, a[4 * g], a[4 * g + 1],
                                  a[4 * g + 2], a[4 * g + 3]);
            *reinterpret_cast<u32x2*>(chunk<kRowBytes>(at, row, col / 8) + 8 * (lane >> 5)) = v;
          }
      lanes_meet();
#pragma unroll 4
      for (int r = 0; r < 32 * kPass; r += kAtOnce) {
        const int row = r + lane / kChunks, c = lane % kChunks;
        put(r0 + 32 * p + row, c0 + 8 * c,
            *reinterpret_cast<const u32x4*>(chunk<kRowBytes>(at, row, c)));
      }
      lanes_meet();
    }
  }

  // The tile mirrored: put(col, row, v) gets eight values of a column at a time.  round makes
  // 16-bit values as above.
  template <class Round, class Put>
  static __device__ __forceinline__ void out16_mirrored(const Acc (&acc)[kBM][kBN], int wave,
                                                        int lane, Round&& round, Put&& put) {
    constexpr int kRowBytes = kRows * 2, kChunks = kRowBytes / 16, kAtOnce = 64 / kChunks;
    static_assert(kCols * kRowBytes <= kRegion, "a part fits its region");
    char* const at = region(wave);
    const int r0 = first_row(wave), c0 = first_col(wave);
    meet();
#pragma unroll
    for (int i = 0; i < kRows / 32; ++i)
#pragma unroll
      for (int j = 0; j < kCols / 32; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int row = 32 * i + (lane & 31), col = 32 * j + 8 * g + 4 * (lane >> 5);
          const Acc& a = kSwap ? acc[j][i] : acc[i][j];
          const u32x2 v = round(r0 + row, c0 + col, a[4 * g], a[4 * g + 1], a[4 * g + 2],
                                a[4 * g + 3]);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *reinterpret_cast<uint16_t*>(chunk<kRowBytes>(at, col + k, row / 8) + 2 * (row & 7)) =
                uint16_t(v[k >> 1] >> (16 * (k & 1)));
        }
    lanes_meet();
#pragma unroll 4
    for (int c = 0; c < kCols; c += kAtOnce) {
      const int col = c + lane / kChunks, r = lane % kChunks;
      put(c0 + col, r0 + 8 * r, *reinterpret_cast<const u32x4*>(chunk<kRowBytes>(at, col, r)));
    }
  }

  // A lane's groups of four accumulators: fn(e, row, col) for group e at row, col .. col+3.
  static constexpr int kGroups = kRows * kCols / 256;
  template <class Fn>
  static __device__ __forceinline__ void groups(int wave, int lane, Fn&& fn) {
    const int r0 = first_row(wave) + (lane & 31), c0 = first_col(wave) + 4 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < kRows / 32; ++i)
#pragma unroll
      for (int j = 0; j < kCols / 32; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          fn((i * (kCols / 32) + j) * 4 + g, r0 + 32 * i, c0 + 32 * j + 8 * g);
  }

  // fn(e, row, col, v) gives group e's four accumulators new values.
  template <class Fn>
  static __device__ __forceinline__ void change(Acc (&acc)[kBM][kBN], int wave, int lane, Fn&& fn) {
    groups(wave, lane, [&](int e, int row, int col) {
      const int i = e / 4 / (kCols / 32), j = e / 4 % (kCols / 32), g = e % 4;
      Acc& a = kSwap ? acc[j][i] : acc[i][j];
      const f32x4 v = fn(e, row, col, f32x4{a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]});
#pragma unroll
      for (int k = 0; k < 4; ++k) a[4 * g + k] = v[k];
    });
  }

  // Where out32 puts a lane's pieces: piece e of kPieces is four of row row(e), from column
  // col(e) of the tile.
  static constexpr int kChunks32 = kCols / 4, kAtOnce32 = 64 / kChunks32;
  static constexpr int kPieces = kRows / kAtOnce32;
  static __device__ __forceinline__ int row(int e, int wave, int lane) {
    return first_row(wave) + e * kAtOnce32 + lane / kChunks32;
  }
  static __device__ __forceinline__ int col(int wave, int lane) {
    return first_col(wave) + 4 * (lane % kChunks32);
  }

  // The same with the accumulators as they are: put(e, v, w) gets piece e and what fetch(e) made.
  // All of a pass's fetches (loads from memory) are on their way before its first put.
  template <class Fetch, class Put>
  static __device__ __forceinline__ void out32(const Acc (&acc)[kBM][kBN], int wave, int lane,
                                               Fetch&& fetch, Put&& put) {
    constexpr int kRowBytes = kCols * 4;
    constexpr int kPass = pass(kRowBytes), kAtOnce = 32 * kPass / kAtOnce32;
    static_assert(kRows / 32 % kPass == 0 && kPass * 32 * kRowBytes <= kRegion, "whole passes");
    char* const at = region(wave);
    meet();
#pragma unroll
    for (int p = 0; p < kRows / 32 / kPass; ++p) {
      decltype(fetch(0)) had[kAtOnce];
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) had[e] = fetch(p * kAtOnce + e);
#pragma unroll
      for (int i = 0; i < kPass; ++i)
#pragma unroll
        for (int j = 0; j < kCols / 32; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int row = 32 * i + (lane & 31), col = 32 * j + 8 * g + 4 * (lane >> 5);
            const Acc& a = kSwap ? acc[j][p * kPass + i] : acc[p * kPass + i][j];
            *reinterpret_cast<f32x4*>(chunk<kRowBytes>(at, row, col / 4)) =
                f32x4{a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]};
          }
      lanes_meet();
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e)
        put(p * kAtOnce + e,
            *reinterpret_cast<const f32x4*>(
                chunk<kRowBytes>(at, e * kAtOnce32 + lane / kChunks32, lane % kChunks32)),
            had[e]);
      lanes_meet();
    }
  }
};

}  // namespace mm
}  // namespace gnmr
