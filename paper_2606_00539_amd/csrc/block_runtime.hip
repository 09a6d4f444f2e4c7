// The C entry points of a gated block's operators (K9, K10, K11): argument checks and launches.
#include <math.h>

#include <algorithm>
#include <string>
#include <vector>

#include "row_checks.h"

namespace {

using namespace gnmr;

gnmr_status check_activation(int32_t activation) {
  if (activation != GNMR_ACT_SILU && activation != GNMR_ACT_GELU)
    return fail(GNMR_E_INVALID, "activation must be GNMR_ACT_SILU or GNMR_ACT_GELU");
  return GNMR_OK;
}

// hidden features, of which two a row make the gated matrices, and the others
gnmr_status check_gated(int32_t hidden, int32_t other) {
  if (hidden <= 0 || other <= 0 || hidden % 8 != 0 || other % 8 != 0)
    return fail(GNMR_E_INVALID, "hidden and the other features must be positive multiples of 8");
  if (hidden >= kMaxFeatures / 2 || other >= kMaxFeatures)
    return fail(GNMR_E_INVALID, "hidden must be < 2^21 and the other features < 2^22");
  return GNMR_OK;
}

constexpr int64_t kMaxRowStride = int64_t(1) << 28;

int64_t size_of(int32_t dtype) { return dtype == GNMR_F32 ? 4 : 2; }
bool is_dtype(int32_t dtype) { return dtype == GNMR_F32 || dtype == GNMR_BF16; }

// A matrix of layer norm's: rows at any stride, elements at their own alignment.
gnmr_status check_rows(const char* name, const void* p, int64_t rows, int64_t cols, int64_t stride,
                       int64_t size) {
  const std::string n = name;
  if (stride < cols || stride > kMaxRowStride)
    return fail(GNMR_E_INVALID, n + "_stride must be in [cols, 2^28]");
  if (rows > 0 && p == nullptr) return fail(GNMR_E_INVALID, n + " must be a device pointer");
  if (!aligned(p, uintptr_t(size)))
    return fail(GNMR_E_INVALID, n + " must be aligned to its elements");
  return GNMR_OK;
}

gnmr_status check_norm(int64_t rows, int32_t cols, int32_t x_dtype, int32_t weight_dtype) {
  if (rows < 0 || rows > kMaxWorkgroups)
    return fail(GNMR_E_INVALID, "rows must be in [0, " + std::to_string(kMaxWorkgroups) + "]");
  if (cols < 1 || cols > kLayerNormCols)
    return fail(GNMR_E_INVALID, "cols must be in [1, " + std::to_string(kLayerNormCols) + "]");
  if (!is_dtype(x_dtype) || !is_dtype(weight_dtype))
    return fail(GNMR_E_INVALID, "x_dtype and weight_dtype must be GNMR_F32 or GNMR_BF16");
  return GNMR_OK;
}

// Whether one of the outputs meets another or an input.
bool any_overlap(const std::vector<Span>& outputs, const std::vector<Span>& inputs) {
  for (size_t i = 0; i < outputs.size(); ++i) {
    for (size_t k = i + 1; k < outputs.size(); ++k)
      if (intersect(outputs[i], outputs[k])) return true;
    for (const Span& in : inputs)
      if (intersect(outputs[i], in)) return true;
  }
  return false;
}

Span vector_span(const void* p, int64_t bytes) { return span_of(p, p == nullptr ? 0 : bytes, 0); }

// Launches of kClipTensors tensors each of those that `wanted` says.
template <class Wanted>
std::vector<ClipTensors> clip_launches(const gnmr_gradient* t, int64_t num, Wanted&& wanted) {
  std::vector<ClipTensors> all;
  for (int64_t k = 0; k < num;) {
    ClipTensors l{};
    int64_t values = 0;
    for (; k < num && l.num < kClipTensors; ++k) {
      if (t[k].numel == 0 || !wanted(t[k])) continue;
      l.t[l.num++] = ClipTensor{t[k].in, t[k].out, t[k].numel, 0, uint8_t(t[k].in_dtype == GNMR_F32),
                                uint8_t(t[k].out_dtype == GNMR_F32)};
      values += t[k].numel;
    }
    if (l.num == 0) break;
    // chunks few enough to count, and small enough for all workgroups to have as many
    l.chunk = kClipLeast;
    while (l.chunk < kClipMost && values / l.chunk > 16 * kClipWorkgroups) l.chunk *= 2;
    for (int32_t i = 0; i < l.num; ++i) {
      l.t[i].first = l.chunks;
      l.chunks += int32_t((l.t[i].numel + l.chunk - 1) / l.chunk);
    }
    all.push_back(l);
  }
  return all;
}

}  // namespace

extern "C" {

gnmr_status gnmr_gated_linear(const gnmr_groups* groups, const void* x, int64_t x_stride,
                              const void* w, void* pre, int64_t pre_stride, void* h,
                              int64_t h_stride, int32_t hidden, int32_t in_features,
                              int32_t activation, void* stream) {
  return call([&]() -> gnmr_status {
    GatedLinear a{};
    gnmr_status r = check_groups(groups, &a.g);
    if (r == GNMR_OK) r = check_gated(hidden, in_features);
    if (r == GNMR_OK) r = check_activation(activation);
    if (r != GNMR_OK) return r;
    const int64_t rows = groups->rows;
    r = check_matrix("x", x, rows, in_features, x_stride, 16);
    if (r == GNMR_OK) r = check_matrix("h", h, rows, hidden, h_stride, 16);
    if (r == GNMR_OK && pre != nullptr)
      r = check_matrix("pre", pre, rows, 2 * int64_t(hidden), pre_stride, 16);
    if (r != GNMR_OK) return r;
    if (w == nullptr || !aligned(w, 16))
      return fail(GNMR_E_INVALID, "w must be a 16-byte aligned device pointer");
    const Span sp = pre == nullptr ? Span{} : matrix_span(pre, rows, 2 * int64_t(hidden),
                                                          pre_stride, 2);
    if (any_overlap({matrix_span(h, rows, hidden, h_stride, 2), sp},
                    {matrix_span(x, rows, in_features, x_stride, 2),
                     span_of(w, int64_t(a.g.num) * hidden * 4 * in_features, 0)}))
      return fail(GNMR_E_INVALID, "an output overlaps another buffer");
    if (rows == 0) return GNMR_OK;
    if (gated_workgroups(a.g, hidden) > kMaxWorkgroups)
      return fail(GNMR_E_INVALID, "too many output tiles for one launch");
    a.x = static_cast<const uint16_t*>(x);
    a.w = static_cast<const uint16_t*>(w);
    a.pre = static_cast<uint16_t*>(pre);
    a.h = static_cast<uint16_t*>(h);
    a.x_stride = x_stride;
    a.pre_stride = pre_stride;
    a.h_stride = h_stride;
    a.H = hidden;
    a.K = in_features;
    GNMR_HIP(launch_gated_linear(a, activation, static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

gnmr_status gnmr_gated_activation(const gnmr_groups* groups, const void* pre, int64_t pre_stride,
                                  void* h, int64_t h_stride, int32_t hidden, int32_t activation,
                                  void* stream) {
  return call([&]() -> gnmr_status {
    GatedActivation a{};
    gnmr_status r = check_groups(groups, &a.g);
    if (r == GNMR_OK) r = check_gated(hidden, 8);
    if (r == GNMR_OK) r = check_activation(activation);
    if (r != GNMR_OK) return r;
    const int64_t rows = groups->rows;
    r = check_matrix("pre", pre, rows, 2 * int64_t(hidden), pre_stride, 16);
    if (r == GNMR_OK) r = check_matrix("h", h, rows, hidden, h_stride, 16);
    if (r != GNMR_OK) return r;
    if (intersect(matrix_span(h, rows, hidden, h_stride, 2),
                  matrix_span(pre, rows, 2 * int64_t(hidden), pre_stride, 2)))
      return fail(GNMR_E_INVALID, "h overlaps pre");
    if (rows == 0) return GNMR_OK;
    if (gated_workgroups(a.g, hidden) > kMaxWorkgroups)
      return fail(GNMR_E_INVALID, "too many output tiles for one launch");
    a.pre = static_cast<const uint16_t*>(pre);
    a.h = static_cast<uint16_t*>(h);
    a.pre_stride = pre_stride;
    a.h_stride = h_stride;
    a.H = hidden;
    GNMR_HIP(launch_gated_activation(a, activation, static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

gnmr_status gnmr_gated_dgrad(const gnmr_groups* groups, const void* dy, int64_t dy_stride,
                             const void* w, const void* pre, int64_t pre_stride, void* dpre,
                             int64_t dpre_stride, int32_t out_features, int32_t hidden,
                             int32_t activation, void* stream) {
  return call([&]() -> gnmr_status {
    GatedDgrad a{};
    gnmr_status r = check_groups(groups, &a.g);
    if (r == GNMR_OK) r = check_gated(hidden, out_features);
    if (r == GNMR_OK) r = check_activation(activation);
    if (r != GNMR_OK) return r;
    const int64_t rows = groups->rows, both = 2 * int64_t(hidden);
    r = check_matrix("dy", dy, rows, out_features, dy_stride, 16);
    if (r == GNMR_OK) r = check_matrix("pre", pre, rows, both, pre_stride, 16);
    if (r == GNMR_OK) r = check_matrix("dpre", dpre, rows, both, dpre_stride, 16);
    if (r != GNMR_OK) return r;
    if (w == nullptr || !aligned(w, 16))
      return fail(GNMR_E_INVALID, "w must be a 16-byte aligned device pointer");
    if (any_overlap({matrix_span(dpre, rows, both, dpre_stride, 2)},
                    {matrix_span(dy, rows, out_features, dy_stride, 2),
                     matrix_span(pre, rows, both, pre_stride, 2),
                     span_of(w, int64_t(a.g.num) * hidden * 2 * out_features, 0)}))
      return fail(GNMR_E_INVALID, "dpre overlaps an input");
    if (rows == 0) return GNMR_OK;
    if (gated_workgroups(a.g, hidden) > kMaxWorkgroups)
      return fail(GNMR_E_INVALID, "too many output tiles for one launch");
    a.dy = static_cast<const uint16_t*>(dy);
    a.w = static_cast<const uint16_t*>(w);
    a.pre = static_cast<const uint16_t*>(pre);
    a.dpre = static_cast<uint16_t*>(dpre);
    a.dy_stride = dy_stride;
    a.pre_stride = pre_stride;
    a.dpre_stride = dpre_stride;
    a.H = hidden;
    a.K = out_features;
    GNMR_HIP(launch_gated_dgrad(a, activation, static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

gnmr_status gnmr_layer_norm(const void* x, int32_t x_dtype, int64_t x_stride, const void* weight,
                            const void* bias, int32_t weight_dtype, void* y, int64_t y_stride,
                            float* mean, float* rstd, int64_t rows, int32_t cols, float eps,
                            void* stream) {
  return call([&]() -> gnmr_status {
    gnmr_status r = check_norm(rows, cols, x_dtype, weight_dtype);
    if (r != GNMR_OK) return r;
    if (!isfinite(eps) || eps < 0.0f) return fail(GNMR_E_INVALID, "eps must be finite and >= 0");
    const int64_t size = size_of(x_dtype), ws = size_of(weight_dtype);
    r = check_rows("x", x, rows, cols, x_stride, size);
    if (r == GNMR_OK) r = check_rows("y", y, rows, cols, y_stride, size);
    if (r != GNMR_OK) return r;
    if (!aligned(weight, uintptr_t(ws)) || !aligned(bias, uintptr_t(ws)) || !aligned(mean, 4) ||
        !aligned(rstd, 4))
      return fail(GNMR_E_INVALID, "weight, bias, mean and rstd must be aligned to their elements");
    if (any_overlap({matrix_span(y, rows, cols, y_stride, size), vector_span(mean, 4 * rows),
                     vector_span(rstd, 4 * rows)},
                    {matrix_span(x, rows, cols, x_stride, size), vector_span(weight, cols * ws),
                     vector_span(bias, cols * ws)}))
      return fail(GNMR_E_INVALID, "an output overlaps another buffer");
    if (rows == 0) return GNMR_OK;
    const LayerNorm a{x,        weight,   bias, y,    mean, rstd, x_stride,
                      y_stride, rows,     cols, eps,  weight_dtype == GNMR_F32, 0};
    GNMR_HIP(launch_layer_norm(a, x_dtype == GNMR_F32, static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

int64_t gnmr_layer_norm_backward_workspace(int64_t rows, int32_t cols) {
  if (rows <= 0 || cols <= 0 || cols > kLayerNormCols) return 0;
  // (for either type)
  return int64_t(std::max(layer_norm_parts(rows, cols, true), layer_norm_parts(rows, cols, false))) *
         2 * cols * 4;
}

gnmr_status gnmr_layer_norm_backward(const void* dy, int64_t dy_stride, const void* x,
                                     int32_t x_dtype, int64_t x_stride, const float* mean,
                                     const float* rstd, const void* weight, int32_t weight_dtype,
                                     void* dx, int64_t dx_stride, void* dweight, void* dbias,
                                     int64_t rows, int32_t cols, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
  return call([&]() -> gnmr_status {
    gnmr_status r = check_norm(rows, cols, x_dtype, weight_dtype);
    if (r != GNMR_OK) return r;
    const int64_t size = size_of(x_dtype), ws = size_of(weight_dtype);
    r = check_rows("dy", dy, rows, cols, dy_stride, size);
    if (r == GNMR_OK) r = check_rows("x", x, rows, cols, x_stride, size);
    if (r == GNMR_OK && dx != nullptr) r = check_rows("dx", dx, rows, cols, dx_stride, size);
    if (r != GNMR_OK) return r;
    if (rows > 0 && (mean == nullptr || rstd == nullptr))
      return fail(GNMR_E_INVALID, "mean and rstd must be device pointers");
    if (!aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, uintptr_t(ws)) ||
        !aligned(dweight, uintptr_t(ws)) || !aligned(dbias, uintptr_t(ws)))
      return fail(GNMR_E_INVALID,
                  "mean, rstd, weight and its gradients must be aligned to their elements");
    const bool sums = dweight != nullptr || dbias != nullptr;
    const int64_t need = sums ? gnmr_layer_norm_backward_workspace(rows, cols) : 0;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned(workspace, 16)))
      return fail(GNMR_E_INVALID, "workspace must be a 16-byte aligned device pointer to " +
                                      std::to_string(need) + " bytes");
    const Span sx = dx == nullptr ? Span{} : matrix_span(dx, rows, cols, dx_stride, size);
    if (any_overlap({sx, vector_span(dweight, cols * ws), vector_span(dbias, cols * ws),
                     span_of(workspace, need, 0)},
                    {matrix_span(dy, rows, cols, dy_stride, size),
                     matrix_span(x, rows, cols, x_stride, size), vector_span(mean, 4 * rows),
                     vector_span(rstd, 4 * rows), vector_span(weight, cols * ws)}))
      return fail(GNMR_E_INVALID, "an output or the workspace overlaps another buffer");
    if (dx == nullptr && !sums) return GNMR_OK;
    const LayerNormBackward a{dy,        x,        mean,      rstd,
                              weight,    dx,       dweight,   dbias,
                              sums ? static_cast<float*>(workspace) : nullptr,
                              dy_stride, x_stride, dx_stride, rows,
                              cols,      weight_dtype == GNMR_F32, 0, 0};
    GNMR_HIP(launch_layer_norm_backward(a, x_dtype == GNMR_F32, static_cast<hipStream_t>(stream)));
    return GNMR_OK;
  });
}

int64_t gnmr_clip_gradients_workspace(int64_t num) {
  if (num <= 0) return 8;
  return 8 + 8 * int64_t(kClipWorkgroups) * ((num + kClipTensors - 1) / kClipTensors);
}

gnmr_status gnmr_clip_gradients(const gnmr_gradient* gradients, int64_t num, const double* norms,
                                int64_t num_norms, double max_norm, double eps, double* norm,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  return call([&]() -> gnmr_status {
    if (num < 0 || num > kClipNumber)
      return fail(GNMR_E_INVALID, "num must be in [0, " + std::to_string(kClipNumber) + "]");
    if (num > 0 && gradients == nullptr) return fail(GNMR_E_INVALID, "gradients is NULL");
    if (num_norms < 0 || num_norms > INT32_MAX || (num_norms > 0 && norms == nullptr))
      return fail(GNMR_E_INVALID, "norms must be a device pointer to num_norms >= 0 norms");
    if (!(max_norm >= 0.0) || !(eps >= 0.0) || isinf(eps))
      return fail(GNMR_E_INVALID, "max_norm must be >= 0, eps finite and >= 0");
    if (norm == nullptr || !aligned(norm, 8) || !aligned(norms, 8))
      return fail(GNMR_E_INVALID, "norm and norms must be 8-byte aligned device pointers");
    const int64_t need = gnmr_clip_gradients_workspace(num);
    if (workspace == nullptr || workspace_bytes < need || !aligned(workspace, 16))
      return fail(GNMR_E_INVALID, "workspace must be a 16-byte aligned device pointer to " +
                                      std::to_string(need) + " bytes");
    // (ids: the gradients' places, and behind them the others)
    std::vector<Span> out{span_of(norm, 8, num), span_of(workspace, need, num + 1)};
    std::vector<Span> in{span_of(norms, 8 * num_norms, num + 2)};
    int64_t values = 0, written = 0;
    for (int64_t k = 0; k < num; ++k) {
      const gnmr_gradient& g = gradients[k];
      auto bad = [&](const char* what) {
        return fail(GNMR_E_INVALID, "gradient " + std::to_string(k) + ": " + what);
      };
      if (g.numel < 0 || g.numel > kClipValues || (values += g.numel) > kClipValues)
        return bad("numel must be >= 0, 2^44 in all at most");
      if (!is_dtype(g.in_dtype) || !is_dtype(g.out_dtype))
        return bad("types must be GNMR_F32 or GNMR_BF16");
      if (g.known != 0 && g.known != 1) return bad("known must be 0 or 1");
      if (g.numel > 0 && (g.in == nullptr || g.out == nullptr))
        return bad("in and out must be device pointers");
      const int64_t si = size_of(g.in_dtype), so = size_of(g.out_dtype);
      if (!aligned(g.in, uintptr_t(si)) || !aligned(g.out, uintptr_t(so)))
        return bad("in and out must be aligned to their elements");
      in.push_back(span_of(g.in, g.numel * si, k));
      out.push_back(span_of(g.out, g.numel * so, k));
      written += g.numel * so;
      if (intersect(in.back(), out.back()) && (g.in != g.out || g.in_dtype != g.out_dtype))
        return bad("out overlaps in (in place needs the same address and type)");
    }
    const int64_t met = find_overlap(out, in);
    if (met != -1)
      return fail(GNMR_E_INVALID,
                  (met >= num ? std::string("norm or the workspace")
                              : "gradient " + std::to_string(met) + ": out") +
                      " overlaps another buffer");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    double* const parts = static_cast<double*>(workspace) + 1;
    ClipScale s{parts, norms, norm, max_norm, eps, num_norms, 0};
    const auto read = clip_launches(gradients, num,
                                    [](const gnmr_gradient& g) { return g.known == 0; });
    for (const ClipTensors& l : read) {
      const int wgs = std::min(l.chunks, kClipWorkgroups);
      GNMR_HIP(launch_clip_squares(l, wgs, parts + s.num_parts, st));
      s.num_parts += wgs;
    }
    if (s.num_parts + num_norms > kClipEach) {
      double* const total = static_cast<double*>(workspace);
      GNMR_HIP(launch_clip_total(s, total, st));
      s.parts = total;
      s.num_parts = 1;
      s.num_norms = 0;
    }
    auto scaled = clip_launches(gradients, num, [](const gnmr_gradient&) { return true; });
    if (scaled.empty()) scaled.push_back(ClipTensors{});
    for (const ClipTensors& l : scaled) GNMR_HIP(launch_clip_scale(l, s, written > kClipCached, st));
    return GNMR_OK;
  });
}

}  // extern "C"
