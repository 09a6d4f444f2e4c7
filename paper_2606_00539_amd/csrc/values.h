// Runs of values of bf16 or fp32 from and to memory at any element alignment, as fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gnmr {

template <int N>
struct Run {
  float v[N];
};

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 Two __attribute__((ext_vector_type(2)));
  typedef float F32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(F32x2{lo, hi}, Two));
}

// N values (4, or 8 of bf16) as they lie in memory: one access of up to 16 bytes.
template <bool kF32, int N>
struct Raw {
  static_assert(N == 4 || (N == 8 && !kF32), "16 bytes at most");
  static constexpr int kWords = kF32 ? N : N / 2, kBytes = kF32 ? 4 : 2;
  typedef uint32_t Words __attribute__((ext_vector_type(kWords), aligned(kBytes)));
  uint32_t w[kWords];

  __device__ __forceinline__ Run<N> values() const {
    Run<N> e;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      if constexpr (kF32) {
        e.v[k] = __uint_as_float(w[k]);
      } else {
        e.v[2 * k] = __uint_as_float(w[k] << 16);
        e.v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      }
    }
    return e;
  }
};

// The values from element i on, through the caches or past them.
template <bool kF32, int N, bool kPast = false>
__device__ __forceinline__ Raw<kF32, N> load_raw(const void* p, int64_t i) {
  typedef Raw<kF32, N> R;
  typedef typename R::Words Words;
  const Words* q = reinterpret_cast<const Words*>(static_cast<const char*>(p) + i * R::kBytes);
  Words v;
  if constexpr (kPast) v = __builtin_nontemporal_load(q);
  else v = *q;
  R r;
#pragma unroll
  for (int k = 0; k < R::kWords; ++k) r.w[k] = v[k];
  return r;
}

// `count` of them, zeros behind.
template <bool kF32, int N>
__device__ __forceinline__ Raw<kF32, N> load_raw_some(const void* p, int64_t i, int count) {
  if (count >= N) return load_raw<kF32, N>(p, i);
  Raw<kF32, N> r;
#pragma unroll
  for (int k = 0; k < Raw<kF32, N>::kWords; ++k) {
    r.w[k] = 0;
    if constexpr (kF32) {
      if (k < count) r.w[k] = static_cast<const uint32_t*>(p)[i + k];
    } else {
      const uint16_t* q = static_cast<const uint16_t*>(p) + i + 2 * k;
      if (2 * k < count) r.w[k] = q[0];
      if (2 * k + 1 < count) r.w[k] |= uint32_t(q[1]) << 16;
    }
  }
  return r;
}

template <bool kF32, int N, bool kPast = false>
__device__ __forceinline__ Run<N> load_run(const void* p, int64_t i) {
  return load_raw<kF32, N, kPast>(p, i).values();
}
template <bool kF32, int N>
__device__ __forceinline__ Run<N> load_some(const void* p, int64_t i, int count) {
  return load_raw_some<kF32, N>(p, i, count).values();
}

template <bool kF32, int N, bool kPast = false>
__device__ __forceinline__ void store_run(void* p, int64_t i, const Run<N>& e) {
  typedef Raw<kF32, N> R;
  typedef typename R::Words Words;
  Words v;
#pragma unroll
  for (int k = 0; k < R::kWords; ++k) {
    if constexpr (kF32) v[k] = __float_as_uint(e.v[k]);
    else v[k] = bf16_pair(e.v[2 * k], e.v[2 * k + 1]);
  }
  Words* q = reinterpret_cast<Words*>(static_cast<char*>(p) + i * R::kBytes);
  if constexpr (kPast) __builtin_nontemporal_store(v, q);
  else *q = v;
}

template <bool kF32>
__device__ __forceinline__ void store_one(void* p, int64_t i, float v) {
  if constexpr (kF32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = uint16_t(bf16_pair(v, v));
}

template <bool kF32, int N>
__device__ __forceinline__ void store_some(void* p, int64_t i, int count, const Run<N>& e) {
  if (count >= N) return store_run<kF32, N>(p, i, e);
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (k < count) store_one<kF32>(p, i + k, e.v[k]);
}

}  // namespace gnmr
