// kan_ops_api.cpp -- the C ABI of the operators around the layer (layer norm, log
// probabilities, gradient clipping) declared in include/kan.h: argument validation (host
// only, before any HIP call), launch planning and dispatch onto the caller's stream.
#include "kan.h"

#include <cmath>
#include <cstdint>

#include "kan_checks.h"
#include "kan_clip_lists.h"
#include "kan_ops.h"

namespace {

using kan::aligned;
using kan::Buf;
using kan::check_rows;
using kan::device_status;
using kan::dtype_size;
using kan::known;
using kan::logits_bytes;
using kan::overlap;
using kan::placed;

constexpr int32_t kMaxNormRow = 1 << 24;

kan_status check_norm(kan_dtype dtype, kan_dtype param_dtype, int64_t rows, int32_t n) {
    if (!known(dtype) || !known(param_dtype)) return KAN_ERR_UNSUPPORTED;
    if (dtype == KAN_F32 && param_dtype != KAN_F32) return KAN_ERR_UNSUPPORTED;
    return check_rows(rows, n, kMaxNormRow);
}

constexpr int32_t kMaxClasses = 1 << 30;

kan_status check_logits(kan_dtype dtype, int64_t rows, int32_t classes) {
    if (!known(dtype)) return KAN_ERR_UNSUPPORTED;
    return check_rows(rows, classes, kMaxClasses);
}

// Shared validation of the calls on many tensors.
kan_status check_clip(const kan::ClipList& l, const void* workspace, size_t workspace_bytes,
                      const float* norm) {
    if (l.count < 0 || l.count > kan::kClipMaxTensors) return KAN_ERR_INVALID_ARG;
    if (l.count > 0 && (l.in == nullptr || l.sizes == nullptr || l.dtypes == nullptr))
        return KAN_ERR_INVALID_ARG;
    const size_t need = kan::clip_workspace(l.count);
    if (norm == nullptr || !aligned(norm, 4) || workspace == nullptr || !aligned(workspace, 16) ||
        workspace_bytes < need)
        return KAN_ERR_INVALID_ARG;
    const Buf own[] = {{norm, 4, 4}, {workspace, need, 16}};
    if (overlap(own[0], own[1])) return KAN_ERR_INVALID_ARG;
    int64_t total = 0;
    for (int64_t t = 0; t < l.count; ++t) {
        if (l.dtypes[t] != KAN_F32 && l.dtypes[t] != KAN_BF16) return KAN_ERR_UNSUPPORTED;
        const int64_t n = l.sizes[t];
        if (n < 0 || n > kan::kClipMaxElements - total) return KAN_ERR_INVALID_ARG;
        total += n;
        if (n == 0) continue;
        const size_t es = l.bf16(t) ? 2 : 4;
        const Buf in = {l.in[t], (size_t)n * es, es};
        if (in.p == nullptr || !aligned(in.p, es) || overlap(in, own[0]) || overlap(in, own[1]))
            return KAN_ERR_INVALID_ARG;
        if (l.out == nullptr || l.out[t] == in.p) continue;
        const Buf out = {l.out[t], in.n, es};
        if (out.p == nullptr || !aligned(out.p, es) || overlap(out, own[0]) ||
            overlap(out, own[1]))
            return KAN_ERR_INVALID_ARG;
    }
    return KAN_OK;
}

size_t norm_part_bytes(const kan::NormPlan& p, int32_t n) {
    return (size_t)2 * p.parts * n * sizeof(float);
}

}  // namespace

extern "C" {

kan_status kan_layer_norm(kan_dtype dtype, kan_dtype param_dtype, int64_t rows, int32_t n,
                          const void* x, const void* residual, const void* weight,
                          const void* bias, float eps, void* h, void* y, float* mean, float* rstd,
                          void* stream) {
    const kan_status st = check_norm(dtype, param_dtype, rows, n);
    if (st != KAN_OK) return st;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return KAN_ERR_INVALID_ARG;
    if (rows == 0) return KAN_OK;
    if (x == nullptr || y == nullptr || (h != nullptr && residual == nullptr) ||
        (mean == nullptr) != (rstd == nullptr))
        return KAN_ERR_INVALID_ARG;
    const size_t es = dtype_size(dtype), ps = dtype_size(param_dtype);
    const size_t t = (size_t)rows * n * es, w = (size_t)n * ps, s = (size_t)rows * 4;
    if (!placed({{x, t, es}, {residual, t, es}, {weight, w, ps}, {bias, w, ps}},
                {{h, t, es}, {y, t, es}, {mean, s, 4}, {rstd, s, 4}}))
        return KAN_ERR_INVALID_ARG;
    const kan::NormArgs a = {x, residual, weight, bias, h, y, mean, rstd, rows, n, eps, 0, 0};
    return device_status(kan::launch_norm(dtype == KAN_BF16, param_dtype == KAN_BF16,
                                          kan::norm_plan(rows, n, (int)es, false), a,
                                          static_cast<hipStream_t>(stream)));
}

kan_status kan_layer_norm_backward_workspace_bytes(kan_dtype dtype, int64_t rows, int32_t n,
                                                   size_t* bytes) {
    if (bytes == nullptr) return KAN_ERR_INVALID_ARG;
    const kan_status st = check_norm(dtype, KAN_F32, rows, n);
    if (st != KAN_OK) return st;
    *bytes = norm_part_bytes(kan::norm_plan(rows, n, (int)dtype_size(dtype), true), n);
    return KAN_OK;
}

kan_status kan_layer_norm_backward(kan_dtype dtype, kan_dtype param_dtype, int64_t rows,
                                   int32_t n, const void* h, const float* mean, const float* rstd,
                                   const void* weight, const void* dy, const void* dh, void* dx,
                                   void* dweight, void* dbias, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    const kan_status st = check_norm(dtype, param_dtype, rows, n);
    if (st != KAN_OK) return st;
    const bool params = dweight != nullptr || dbias != nullptr;
    if (dx == nullptr && (!params || dh != nullptr)) return KAN_ERR_INVALID_ARG;
    const size_t es = dtype_size(dtype), ps = dtype_size(param_dtype);
    const size_t t = (size_t)rows * n * es, w = (size_t)n * ps, s = (size_t)rows * 4;
    const kan::NormPlan p = kan::norm_plan(rows, n, (int)es, true);
    const size_t need = params ? norm_part_bytes(p, n) : 0;
    if (rows > 0 && (h == nullptr || mean == nullptr || rstd == nullptr || dy == nullptr))
        return KAN_ERR_INVALID_ARG;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return KAN_ERR_INVALID_ARG;
    if (!placed({{h, t, es}, {mean, s, 4}, {rstd, s, 4}, {weight, w, ps}, {dy, t, es}, {dh, t, es}},
                {{dx, t, es}, {dweight, w, ps}, {dbias, w, ps},
                 {need > 0 ? workspace : nullptr, need, 16}}))
        return KAN_ERR_INVALID_ARG;
    if (rows == 0 && !params) return KAN_OK;
    const kan::NormGradArgs a = {h, weight, dy, dh, mean, rstd, dx,
                                 // (one part is written as the gradients themselves)
                                 p.parts > 1 ? static_cast<float*>(workspace) : nullptr,
                                 dweight, dbias, rows, n, 0, 0};
    return device_status(kan::launch_norm_grad(dtype == KAN_BF16, param_dtype == KAN_BF16, p, a,
                                               static_cast<hipStream_t>(stream)));
}

kan_status kan_token_logprobs_workspace_bytes(kan_dtype dtype, int64_t rows, int32_t classes,
                                              int32_t top_k, size_t* bytes) {
    if (bytes == nullptr) return KAN_ERR_INVALID_ARG;
    const kan_status st = check_logits(dtype, rows, classes);
    if (st != KAN_OK) return st;
    if (top_k < 0 || top_k > kan::kMaxTop || top_k > classes) return KAN_ERR_INVALID_ARG;
    *bytes = kan::logprob_plan(rows, classes, (int)dtype_size(dtype), top_k).bytes;
    return KAN_OK;
}

kan_status kan_token_logprobs(kan_dtype dtype, int64_t rows, int32_t classes, const void* logits,
                              int64_t row_stride, const int64_t* targets, int64_t ignore_index,
                              int32_t top_k, float* logp, float* stats, float* entropy,
                              float* top_logp, int64_t* top_index, void* workspace,
                              size_t workspace_bytes, void* stream) {
    const kan_status st = check_logits(dtype, rows, classes);
    if (st != KAN_OK) return st;
    if (top_k < 0 || top_k > kan::kMaxTop || top_k > classes) return KAN_ERR_INVALID_ARG;
    if (rows == 0) return KAN_OK;
    const size_t es = dtype_size(dtype), z = logits_bytes(rows, classes, row_stride, es);
    if (z == 0 || logits == nullptr || targets == nullptr || logp == nullptr || stats == nullptr)
        return KAN_ERR_INVALID_ARG;
    if ((top_logp != nullptr) != (top_k > 0) || (top_index != nullptr) != (top_k > 0))
        return KAN_ERR_INVALID_ARG;
    const kan::LogprobPlan p = kan::logprob_plan(rows, classes, (int)es, top_k);
    if (p.bytes > 0 && (workspace == nullptr || workspace_bytes < p.bytes))
        return KAN_ERR_INVALID_ARG;
    const size_t s = (size_t)rows * 4;
    if (!placed({{logits, z, es}, {targets, 2 * s, 8}},
                {{logp, s, 4}, {stats, 2 * s, 4}, {entropy, s, 4}, {top_logp, s * top_k, 4},
                 {top_index, 2 * s * top_k, 8}, {p.bytes > 0 ? workspace : nullptr, p.bytes, 16}}))
        return KAN_ERR_INVALID_ARG;
    kan::LogprobArgs a = {};
    a.z = logits;
    a.targets = targets;
    a.rows = rows;
    a.stride = row_stride;
    a.ignore = ignore_index;
    a.classes = classes;
    a.k = top_k;
    a.logp = logp;
    a.stats = stats;
    a.entropy = entropy;
    a.top_logp = top_logp;
    a.top_index = top_index;
    return device_status(kan::launch_logprob(dtype == KAN_BF16, p, a, workspace,
                                             static_cast<hipStream_t>(stream)));
}

kan_status kan_token_logprobs_backward(kan_dtype dtype, int64_t rows, int32_t classes,
                                       const void* logits, int64_t row_stride,
                                       const int64_t* targets, int64_t ignore_index,
                                       const float* stats, const float* dlogp,
                                       const float* entropy, const float* dentropy, void* dlogits,
                                       int64_t dlogits_stride, void* stream) {
    const kan_status st = check_logits(dtype, rows, classes);
    if (st != KAN_OK) return st;
    if (rows == 0) return KAN_OK;
    const size_t es = dtype_size(dtype), z = logits_bytes(rows, classes, row_stride, es);
    const size_t dz = logits_bytes(rows, classes, dlogits_stride, es), s = (size_t)rows * 4;
    if (z == 0 || dz == 0 || logits == nullptr || targets == nullptr || stats == nullptr ||
        dlogp == nullptr || dlogits == nullptr || (entropy == nullptr) != (dentropy == nullptr))
        return KAN_ERR_INVALID_ARG;
    // (in place: each gradient over its own logit)
    const bool in_place = dlogits == logits && dlogits_stride == row_stride;
    if (!placed({{in_place ? nullptr : logits, z, es}, {targets, 2 * s, 8}, {stats, 2 * s, 4},
                 {dlogp, s, 4}, {entropy, s, 4}, {dentropy, s, 4}},
                {{dlogits, dz, es}}))
        return KAN_ERR_INVALID_ARG;
    kan::LogprobGradArgs a = {};
    a.z = logits;
    a.targets = targets;
    a.stats = stats;
    a.dlogp = dlogp;
    a.entropy = entropy;
    a.dentropy = dentropy;
    a.dz = dlogits;
    a.rows = rows;
    a.stride = row_stride;
    a.dstride = dlogits_stride;
    a.ignore = ignore_index;
    a.classes = classes;
    return device_status(kan::launch_logprob_grad(dtype == KAN_BF16, a,
                                                  static_cast<hipStream_t>(stream)));
}

kan_status kan_grad_norm_workspace_bytes(int32_t count, size_t* bytes) {
    if (bytes == nullptr || count < 0 || count > kan::kClipMaxTensors) return KAN_ERR_INVALID_ARG;
    *bytes = kan::clip_workspace(count);
    return KAN_OK;
}

kan_status kan_grad_norm(int32_t count, const void* const* grads, const int64_t* sizes,
                         const int32_t* dtypes, void* workspace, size_t workspace_bytes,
                         float* norm, void* stream) {
    const kan::ClipList l = {count, grads, nullptr, sizes, dtypes};
    const kan_status st = check_clip(l, workspace, workspace_bytes, norm);
    if (st != KAN_OK) return st;
    return device_status(
        kan::launch_clip(l, {0.0f, 0.0f, norm}, workspace, static_cast<hipStream_t>(stream)));
}

kan_status kan_clip_grad_norm(int32_t count, const void* const* grads, const int64_t* sizes,
                              const int32_t* dtypes, float max_norm, float eps, void* const* out,
                              void* workspace, size_t workspace_bytes, float* norm,
                              void* stream) {
    if (!(max_norm >= 0.0f) || !(eps >= 0.0f) || !std::isfinite(eps)) return KAN_ERR_INVALID_ARG;
    if (count > 0 && out == nullptr) return KAN_ERR_INVALID_ARG;
    void* const none = nullptr;
    const kan::ClipList l = {count, grads, count > 0 ? out : &none, sizes, dtypes};
    const kan_status st = check_clip(l, workspace, workspace_bytes, norm);
    if (st != KAN_OK) return st;
    if (kan::clip_outputs_clash(l)) return KAN_ERR_INVALID_ARG;
    return device_status(kan::launch_clip(l, {max_norm, eps, norm}, workspace,
                                          static_cast<hipStream_t>(stream)));
}

}  // extern "C"
