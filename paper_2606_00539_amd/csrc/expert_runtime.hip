// The C entry points of the expert step's operators (K6, K7, K8): argument checks
// and launches.
#include <math.h>

#include <string>

#include "row_checks.h"

namespace {

using namespace gnmr;

gnmr_status grouped_rows(const gnmr_groups* groups, const void* in, int64_t in_stride,
                         const void* w, void* out, int64_t out_stride, int32_t out_features,
                         int32_t in_features, bool dgrad, void* stream) {
  gnmr::GroupedRows a{};
  gnmr_status r = check_groups(groups, &a.g);
  if (r == GNMR_OK) r = check_features(out_features, in_features, kMaxFeatures);
  if (r != GNMR_OK) return r;
  a.N = dgrad ? in_features : out_features;
  a.K = dgrad ? out_features : in_features;
  r = check_matrix(dgrad ? "dy" : "x", in, groups->rows, a.K, in_stride, 16);
  if (r == GNMR_OK) r = check_matrix(dgrad ? "dx" : "y", out, groups->rows, a.N, out_stride, 16);
  if (r != GNMR_OK) return r;
  if (w == nullptr || !aligned(w, 16))
    return fail(GNMR_E_INVALID, "w must be a 16-byte aligned device pointer");
  const Span so = matrix_span(out, groups->rows, a.N, out_stride, 2);
  if (intersect(so, matrix_span(in, groups->rows, a.K, in_stride, 2)) ||
      intersect(so, span_of(w, int64_t(a.g.num) * a.N * a.K * 2, 0)))
    return fail(GNMR_E_INVALID, "the output overlaps an input");
  if (groups->rows == 0) return GNMR_OK;
  if (gnmr::grouped_rows_workgroups(a) > kMaxWorkgroups)
    return fail(GNMR_E_INVALID, "too many output tiles for one launch");
  a.in = static_cast<const uint16_t*>(in);
  a.w = static_cast<const uint16_t*>(w);
  a.out = static_cast<uint16_t*>(out);
  a.in_stride = in_stride;
  a.out_stride = out_stride;
  GNMR_HIP(gnmr::launch_grouped_rows(a, dgrad, static_cast<hipStream_t>(stream)));
  return GNMR_OK;
}

}  // namespace

extern "C" {

gnmr_status gnmr_grouped_linear(const gnmr_groups* groups, const void* x, int64_t x_stride,
                                const void* w, void* y, int64_t y_stride, int32_t out_features,
                                int32_t in_features, void* stream) {
  return call([&] {
    return grouped_rows(groups, x, x_stride, w, y, y_stride, out_features, in_features, false,
                        stream);
  });
}

gnmr_status gnmr_grouped_dgrad(const gnmr_groups* groups, const void* dy, int64_t dy_stride,
                               const void* w, void* dx, int64_t dx_stride, int32_t out_features,
                               int32_t in_features, void* stream) {
  return call([&] {
    return grouped_rows(groups, dy, dy_stride, w, dx, dx_stride, out_features, in_features, true,
                        stream);
  });
}

int64_t gnmr_grouped_wgrad_num_partials(int32_t out_features, int32_t in_features) {
  if (out_features <= 0 || in_features <= 0) return 0;
  const int64_t b = gnmr::kGroupedBlock;
  return (out_features + b - 1) / b * ((in_features + b - 1) / b);
}

gnmr_status gnmr_grouped_wgrad(const gnmr_groups* groups, const void* dy, int64_t dy_stride,
                               const void* x, int64_t x_stride, void* dw, int32_t dw_dtype,
                               int32_t accumulate, float* partials, int32_t out_features,
                               int32_t in_features, void* stream) {
  return call([&]() -> gnmr_status {
    gnmr::GroupedWgrad a{};
    gnmr_status r = check_groups(groups, &a.g);
    if (r == GNMR_OK) r = check_features(out_features, in_features, kMaxFeatures);
    if (r == GNMR_OK) r = check_matrix("dy", dy, groups->rows, out_features, dy_stride, 16);
    if (r == GNMR_OK) r = check_matrix("x", x, groups->rows, in_features, x_stride, 16);
    if (r != GNMR_OK) return r;
    if (dw_dtype != GNMR_F32 && dw_dtype != GNMR_BF16)
      return fail(GNMR_E_INVALID, "dw_dtype must be GNMR_F32 or GNMR_BF16");
    if (accumulate != 0 && accumulate != 1)
      return fail(GNMR_E_INVALID, "accumulate must be 0 or 1");
    if (dw == nullptr || !aligned(dw, 16))
      return fail(GNMR_E_INVALID, "dw must be a 16-byte aligned device pointer");
    if (partials == nullptr || !aligned(partials, 4))
      return fail(GNMR_E_INVALID, "partials must be a device pointer");
    const int64_t size = dw_dtype == GNMR_F32 ? 4 : 2;
    const int64_t blocks = gnmr_grouped_wgrad_num_partials(out_features, in_features);
    const Span sw = span_of(dw, int64_t(a.g.num) * out_features * in_features * size, 0);
    const Span sp = span_of(partials, int64_t(a.g.num) * blocks * 4, 0);
    const Span sy = matrix_span(dy, groups->rows, out_features, dy_stride, 2);
    const Span sx = matrix_span(x, groups->rows, in_features, x_stride, 2);
    if (intersect(sw, sp) || intersect(sw, sy) || intersect(sw, sx) || intersect(sp, sy) ||
        intersect(sp, sx))
      return fail(GNMR_E_INVALID, "dw or partials overlaps another buffer");
    if (a.g.num * (blocks + gnmr::kNumXcd) > kMaxWorkgroups)
      return fail(GNMR_E_INVALID, "too many output tiles for one launch");
    a.dy = static_cast<const uint16_t*>(dy);
    a.x = static_cast<const uint16_t*>(x);
    a.dw = dw;
    a.partials = partials;
    a.dy_stride = dy_stride;
    a.x_stride = x_stride;
    a.M = out_features;
    a.N = in_features;
    GNMR_HIP(gnmr::launch_grouped_wgrad(a, dw_dtype == GNMR_F32, accumulate != 0,
                                        static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

gnmr_status gnmr_quantize_rows(const void* x, int32_t x_dtype, int64_t x_stride, void* codes,
                               float* scale, int64_t rows, int32_t cols, void* stream) {
  return call([&]() -> gnmr_status {
    if (rows < 0 || rows > kMaxWorkgroups)
      return fail(GNMR_E_INVALID, "rows must be in [0, " + std::to_string(kMaxWorkgroups) + "]");
    if (cols <= 0 || cols % 8 != 0 || cols >= kMaxQuantized)
      return fail(GNMR_E_INVALID, "cols must be a positive multiple of 8 below 2^17");
    if (x_dtype != GNMR_F32 && x_dtype != GNMR_BF16)
      return fail(GNMR_E_INVALID, "x_dtype must be GNMR_F32 or GNMR_BF16");
    const gnmr_status r = check_matrix("x", x, rows, cols, x_stride, 16);
    if (r != GNMR_OK) return r;
    if (rows > 0 && (codes == nullptr || scale == nullptr))
      return fail(GNMR_E_INVALID, "codes and scale must be device pointers");
    if (!aligned(codes, 8) || !aligned(scale, 4))
      return fail(GNMR_E_INVALID, "codes must be 8-byte aligned, scale 4-byte");
    const Span sx = matrix_span(x, rows, cols, x_stride, x_dtype == GNMR_F32 ? 4 : 2);
    const Span sc = span_of(codes, rows * cols, 0), ss = span_of(scale, rows * 4, 0);
    if (intersect(sx, sc) || intersect(sx, ss) || intersect(sc, ss))
      return fail(GNMR_E_INVALID, "codes or scale overlaps another buffer");
    gnmr::QuantizeRows a{x, static_cast<int8_t*>(codes), scale, x_stride, cols, int32_t(rows),
                         cols};
    GNMR_HIP(gnmr::launch_quantize_rows(a, x_dtype == GNMR_F32, static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

int64_t gnmr_quantized_linear_workspace(int64_t rows, int32_t in_features) {
  if (rows <= 0 || in_features <= 0) return 0;
  return gnmr::quantized_codes_stride(in_features) * rows + 4 * rows;
}

gnmr_status gnmr_quantized_linear(const gnmr_groups* groups, const void* x, int64_t x_stride,
                                  const float* x_scale, const void* codes, const float* w_scale,
                                  void* y, int64_t y_stride, int32_t out_features,
                                  int32_t in_features, void* workspace, int64_t workspace_bytes,
                                  void* stream) {
  return call([&]() -> gnmr_status {
    gnmr::QuantizedLinear a{};
    gnmr_status r = check_groups(groups, &a.g);
    if (r == GNMR_OK) r = check_features(out_features, in_features, kMaxQuantized);
    if (r != GNMR_OK) return r;
    const int64_t rows = groups->rows;
    r = check_matrix("x", x, rows, in_features, x_stride, x_scale == nullptr ? 16 : 8);
    if (r == GNMR_OK) r = check_matrix("y", y, rows, out_features, y_stride, 16);
    if (r != GNMR_OK) return r;
    if (codes == nullptr || !aligned(codes, 8))
      return fail(GNMR_E_INVALID, "codes must be an 8-byte aligned device pointer");
    if (w_scale == nullptr || !aligned(w_scale, 4) || !aligned(x_scale, 4))
      return fail(GNMR_E_INVALID, "w_scale and x_scale must be device pointers");
    const int64_t need = x_scale == nullptr ? gnmr_quantized_linear_workspace(rows, in_features) : 0;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned(workspace, 16)))
      return fail(GNMR_E_INVALID, "workspace must be a 16-byte aligned device pointer to " +
                                      std::to_string(need) + " bytes");
    const int64_t weights = int64_t(a.g.num) * out_features;
    const Span sy = matrix_span(y, rows, out_features, y_stride, 2);
    const Span sx = matrix_span(x, rows, in_features, x_stride, x_scale == nullptr ? 2 : 1);
    const Span sc = span_of(codes, weights * in_features, 0), sw = span_of(w_scale, weights * 4, 0);
    const Span sk = span_of(workspace, need, 0);
    const Span ss = span_of(x_scale, x_scale == nullptr ? 0 : rows * 4, 0);
    for (const Span& in : {sx, sc, sw, sk, ss})
      if (intersect(sy, in)) return fail(GNMR_E_INVALID, "y overlaps an input or the workspace");
    for (const Span& in : {sx, sc, sw})
      if (intersect(sk, in)) return fail(GNMR_E_INVALID, "the workspace overlaps an input");
    if (rows == 0) return GNMR_OK;
    if (gnmr::quantized_linear_workgroups(a.g, out_features) > kMaxWorkgroups ||
        (x_scale == nullptr && rows > kMaxWorkgroups))
      return fail(GNMR_E_INVALID, "too many output tiles for one launch");
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_scale == nullptr && gnmr::quantized_token(a.g, in_features)) {
      const gnmr::QuantizedToken one{static_cast<const uint16_t*>(x),
                                     static_cast<const int8_t*>(codes),
                                     w_scale,
                                     static_cast<uint16_t*>(y),
                                     a.g.mask,
                                     a.g.mask_value,
                                     out_features,
                                     in_features};
      GNMR_HIP(gnmr::launch_quantized_token(one, st));
      return GNMR_OK;
    }
    a.w = static_cast<const int8_t*>(codes);
    a.w_scale = w_scale;
    a.y = static_cast<uint16_t*>(y);
    a.y_stride = y_stride;
    a.N = out_features;
    a.K = in_features;
    if (x_scale == nullptr) {
      a.q_stride = gnmr::quantized_codes_stride(in_features);
      int8_t* q = static_cast<int8_t*>(workspace);
      float* s = reinterpret_cast<float*>(q + a.q_stride * rows);
      a.q = q;
      a.q_scale = s;
      const gnmr::QuantizeRows z{x, q, s, x_stride, a.q_stride, int32_t(rows), in_features};
      GNMR_HIP(gnmr::launch_quantize_rows(z, false, st));
    } else {
      a.q = static_cast<const int8_t*>(x);
      a.q_stride = x_stride;
      a.q_scale = x_scale;
    }
    GNMR_HIP(gnmr::launch_quantized_linear(a, st));
    return GNMR_OK;
  });
}

int64_t gnmr_orthogonalize_workspace(int32_t rows, int32_t cols, int32_t count) {
  if (rows <= 0 || cols <= 0 || count <= 0) return 0;
  return gnmr::orthogonal_workspace(rows, cols, count);
}

gnmr_status gnmr_orthogonalize(const void* in, int32_t in_dtype, void* out, int32_t rows,
                               int32_t cols, int32_t count, const gnmr_newton_schulz* settings,
                               void* workspace, int64_t workspace_bytes, void* stream) {
  return call([&]() -> gnmr_status {
    if (rows < 1 || cols < 1 || rows > 65536 || cols > 65536)
      return fail(GNMR_E_INVALID, "rows and cols must be in [1, 65536]");
    if (count < 0 || count > 65535) return fail(GNMR_E_INVALID, "count must be in [0, 65535]");
    if (in_dtype != GNMR_F32 && in_dtype != GNMR_BF16)
      return fail(GNMR_E_INVALID, "in_dtype must be GNMR_F32 or GNMR_BF16");
    if (settings == nullptr) return fail(GNMR_E_INVALID, "settings is NULL");
    const gnmr_newton_schulz& z = *settings;
    if (z.steps < 1 || z.steps > 100) return fail(GNMR_E_INVALID, "steps must be in [1, 100]");
    if (!isfinite(z.a) || !isfinite(z.b) || !isfinite(z.c) || !isfinite(z.scale) ||
        !isfinite(z.eps) || z.eps < 0.0f)
      return fail(GNMR_E_INVALID, "a, b, c, scale and eps must be finite, eps >= 0");
    if (count == 0) return GNMR_OK;
    const int64_t size = in_dtype == GNMR_F32 ? 4 : 2, n = int64_t(count) * rows * cols;
    if (in == nullptr || out == nullptr || !aligned(in, uintptr_t(size)) || !aligned(out, 2))
      return fail(GNMR_E_INVALID, "in and out must be device pointers aligned to their elements");
    const int64_t need = gnmr_orthogonalize_workspace(rows, cols, count);
    if (workspace == nullptr || workspace_bytes < need || !aligned(workspace, 256))
      return fail(GNMR_E_INVALID, "workspace must be a 256-byte aligned device pointer to " +
                                      std::to_string(need) + " bytes");
    const Span si = span_of(in, n * size, 0), so = span_of(out, n * 2, 0),
               sw = span_of(workspace, need, 0);
    if (intersect(si, so) || intersect(si, sw) || intersect(so, sw))
      return fail(GNMR_E_INVALID, "out or the workspace overlaps another buffer");
    gnmr::Orthogonal a{};
    a.in = in;
    a.out = static_cast<__bf16*>(out);
    a.rows = rows;
    a.cols = cols;
    a.count = count;
    a.eps = z.eps;
    a.f32 = in_dtype == GNMR_F32;
    if (gnmr::orthogonal_workgroups(a) > kMaxWorkgroups)
      return fail(GNMR_E_INVALID, "too many output tiles for one launch");
    GNMR_HIP(gnmr::launch_orthogonal(a, z, workspace, static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

}  // extern "C"
