// What the C entry points share: the error of the last call, HIP status checks
// and overlaps of byte ranges.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "gnmr.h"

namespace gnmr {

// Keeps `msg` for gnmr_last_error (per thread) and returns `st`.
gnmr_status fail(gnmr_status st, const std::string& msg);

#define GNMR_HIP(expr)                                                                 \
  do {                                                                                 \
    hipError_t e_ = (expr);                                                            \
    if (e_ != hipSuccess)                                                              \
      return gnmr::fail(GNMR_E_HIP, std::string(#expr) + ": " + hipGetErrorString(e_)); \
  } while (0)

// A byte range [lo, hi) of device memory that buffer `id` covers.
struct Span {
  uintptr_t lo, hi;
  int64_t id;
};

inline Span span_of(const void* p, int64_t bytes, int64_t id) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return Span{lo, lo + uintptr_t(bytes), id};
}

inline bool intersect(const Span& a, const Span& b) {
  return a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi;
}

}  // namespace gnmr
