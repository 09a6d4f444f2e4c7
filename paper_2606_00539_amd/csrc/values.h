// Runs of values of bf16 or fp32 from and to memory at any element alignment, as fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gnmr {

// Vectors that need the alignment of their elements only.
typedef uint32_t AnyU32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float AnyF32x4 __attribute__((ext_vector_type(4), aligned(4)));

struct Eight {
  float v[8];
};

__device__ __forceinline__ float bf16_value(uint16_t bits) {
  return __uint_as_float(uint32_t(bits) << 16);
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 Two __attribute__((ext_vector_type(2)));
  typedef float F32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(F32x2{lo, hi}, Two));
}

// The eight values from element i on.
template <bool kF32>
__device__ __forceinline__ Eight load_eight(const void* p, int64_t i) {
  Eight e;
  if constexpr (kF32) {
    const AnyF32x4* q = reinterpret_cast<const AnyF32x4*>(static_cast<const float*>(p) + i);
    const AnyF32x4 a = q[0], b = q[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      e.v[k] = a[k];
      e.v[4 + k] = b[k];
    }
  } else {
    const AnyU32x4 a = *reinterpret_cast<const AnyU32x4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      e.v[2 * k] = __uint_as_float(a[k] << 16);
      e.v[2 * k + 1] = __uint_as_float(a[k] & 0xFFFF0000u);
    }
  }
  return e;
}

template <bool kF32>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
  if constexpr (kF32) return static_cast<const float*>(p)[i];
  else return bf16_value(static_cast<const uint16_t*>(p)[i]);
}

// `count` values from element i on, zeros behind them.
template <bool kF32>
__device__ __forceinline__ Eight load_some(const void* p, int64_t i, int count) {
  if (count >= 8) return load_eight<kF32>(p, i);
  Eight e;
#pragma unroll
  for (int k = 0; k < 8; ++k) e.v[k] = k < count ? load_one<kF32>(p, i + k) : 0.0f;
  return e;
}

template <bool kF32>
__device__ __forceinline__ void store_eight(void* p, int64_t i, const Eight& e) {
  if constexpr (kF32) {
    AnyF32x4* q = reinterpret_cast<AnyF32x4*>(static_cast<float*>(p) + i);
    q[0] = AnyF32x4{e.v[0], e.v[1], e.v[2], e.v[3]};
    q[1] = AnyF32x4{e.v[4], e.v[5], e.v[6], e.v[7]};
  } else {
    *reinterpret_cast<AnyU32x4*>(static_cast<uint16_t*>(p) + i) =
        AnyU32x4{bf16_pair(e.v[0], e.v[1]), bf16_pair(e.v[2], e.v[3]),
                 bf16_pair(e.v[4], e.v[5]), bf16_pair(e.v[6], e.v[7])};
  }
}

template <bool kF32>
__device__ __forceinline__ void store_one(void* p, int64_t i, float v) {
  if constexpr (kF32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = uint16_t(bf16_pair(v, v));
}

template <bool kF32>
__device__ __forceinline__ void store_some(void* p, int64_t i, int count, const Eight& e) {
  if (count >= 8) return store_eight<kF32>(p, i, e);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < count) store_one<kF32>(p, i + k, e.v[k]);
}

}  // namespace gnmr
