// What the C entry points of the operators on rows check (K6 to K11).
#pragma once

#include <stdint.h>

#include <string>

#include "gnmr_internal.h"
#include "host_call.h"

namespace gnmr {

constexpr int64_t kMaxWorkgroups = int64_t(UINT32_MAX) / 256;  // a grid holds < 2^32 lanes
constexpr int32_t kMaxFeatures = 1 << 22;   // tiles address a row block with 32-bit offsets
constexpr int32_t kMaxQuantized = 1 << 17;  // 2^17 products of codes stay below 2^31
constexpr int64_t kMaxRows = INT32_MAX - 256;

// Runs a call's body; no exception (of an allocation for a message) leaves it.
template <class Fn>
gnmr_status call(Fn&& body) noexcept {
  try {
    return body();
  } catch (...) {
    return GNMR_E_NOMEM;
  }
}

inline bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline gnmr_status check_groups(const gnmr_groups* g, GroupArgs* out) {
  if (g == nullptr) return fail(GNMR_E_INVALID, "groups is NULL");
  if (g->rows < 0 || g->rows > kMaxRows)
    return fail(GNMR_E_INVALID, "rows must be in [0, 2^31 - 257]");
  if (g->num_groups < 1 || g->num_groups > 65536)
    return fail(GNMR_E_INVALID, "num_groups must be in [1, 65536]");
  if (g->offsets == nullptr && g->num_groups != 1)
    return fail(GNMR_E_INVALID, "offsets may be NULL only with one group");
  if (!aligned(g->offsets, 4)) return fail(GNMR_E_INVALID, "offsets must be 4-byte aligned");
  if (g->mask_value != 0 && g->mask_value != 1)
    return fail(GNMR_E_INVALID, "mask_value must be 0 or 1");
  *out = GroupArgs{g->offsets, g->d_mask, g->num_groups, g->mask_value, int32_t(g->rows)};
  return GNMR_OK;
}

inline gnmr_status check_features(int32_t out, int32_t in, int32_t most_in) {
  if (out <= 0 || in <= 0 || out % 8 != 0 || in % 8 != 0)
    return fail(GNMR_E_INVALID, "out_features and in_features must be positive multiples of 8");
  if (out >= kMaxFeatures || in >= most_in)
    return fail(GNMR_E_INVALID, "out_features must be < 2^22 and in_features < " +
                                    std::to_string(most_in));
  return GNMR_OK;
}

// A matrix of `rows` rows of `cols` elements, `stride` apart.
inline gnmr_status check_matrix(const char* name, const void* p, int64_t rows, int64_t cols,
                         int64_t stride, int64_t align) {
  const std::string n = name;
  if (stride < cols || stride % 8 != 0 || stride >= kMaxFeatures)
    return fail(GNMR_E_INVALID, n + "_stride must be at least the features, a multiple of 8 and "
                                    "< 2^22");
  if (rows > 0 && p == nullptr) return fail(GNMR_E_INVALID, n + " must be a device pointer");
  if (!aligned(p, uintptr_t(align)))
    return fail(GNMR_E_INVALID, n + " must be " + std::to_string(align) + "-byte aligned");
  return GNMR_OK;
}

inline Span matrix_span(const void* p, int64_t rows, int64_t cols, int64_t stride, int64_t size) {
  return span_of(p, rows == 0 ? 0 : ((rows - 1) * stride + cols) * size, 0);
}

}  // namespace gnmr
