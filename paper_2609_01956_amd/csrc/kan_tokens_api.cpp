// kan_tokens_api.cpp -- the C ABI of the token operators (embedding, log probabilities under a
// linear head) declared in include/kan.h: argument validation (host only, before any HIP call) and
// dispatch onto the caller's stream.
#include <cmath>
#include <cstdint>

#include "kan.h"
#include "kan_checks.h"
#include "kan_head.h"

namespace {

using kan::aligned;
using kan::device_status;
using kan::dtype_size;
using kan::known;
using kan::logits_bytes;
using kan::placed;

constexpr int64_t kMaxTokens = INT64_C(1) << 30;
constexpr int32_t kMaxClasses = 1 << 30, kMaxEmbedRow = 1 << 24;
constexpr int64_t kMaxHeadRows = 1 << 20;
constexpr int32_t kMaxHeadRow = 1 << 20;
constexpr int64_t kMost = INT64_C(1) << 48;

kan_status check_embedding(int64_t rows, int32_t classes, int32_t n) {
    if (rows < 0 || rows > kMaxTokens || classes < 1 || classes > kMaxClasses || n < 1 ||
        n > kMaxEmbedRow || rows > kMost / n || classes > kMost / n)
        return KAN_ERR_INVALID_ARG;
    return KAN_OK;
}

kan_status check_table(kan_dtype dtype, kan_dtype table_dtype, float scale) {
    if (!known(dtype) || !known(table_dtype)) return KAN_ERR_UNSUPPORTED;
    if (dtype == KAN_F32 && table_dtype != KAN_F32) return KAN_ERR_UNSUPPORTED;
    return std::isfinite(scale) ? KAN_OK : KAN_ERR_INVALID_ARG;
}

// Rows that the tiles' 16-byte loads and 32-bit offsets (256 rows) can take as they stand.
bool direct(const void* p, int64_t stride, int32_t n, int es) {
    return aligned(p, 16) && n % (16 / es) == 0 && stride % (16 / es) == 0 &&
           stride <= (INT64_C(1) << 22) / es;
}

kan_status head_shape(kan_dtype dtype, int64_t rows, int32_t classes, int32_t n, const void* x,
                      int64_t x_stride, const void* weight, int64_t weight_stride,
                      kan::HeadShape* s) {
    if (!known(dtype)) return KAN_ERR_UNSUPPORTED;
    if (rows < 0 || rows > kMaxHeadRows || classes < 1 || classes > kMaxClasses || n < 1 ||
        n > kMaxHeadRow || x_stride < n || weight_stride < n)
        return KAN_ERR_INVALID_ARG;
    if ((rows > 0 && rows > kMost / x_stride) || classes > kMost / weight_stride)
        return KAN_ERR_INVALID_ARG;
    const int es = (int)dtype_size(dtype);
    *s = {rows, classes, n, es, direct(x, x_stride, n, es), direct(weight, weight_stride, n, es),
          x_stride, weight_stride};
    return KAN_OK;
}

}  // namespace

extern "C" {

kan_status kan_embedding(kan_dtype dtype, kan_dtype table_dtype, int64_t rows, int32_t classes,
                         int32_t n, const int64_t* tokens, int64_t ignore_index, const void* table,
                         int64_t table_stride, float scale, void* y, void* stream) {
    kan_status st = check_table(dtype, table_dtype, scale);
    if (st != KAN_OK) return st;
    st = check_embedding(rows, classes, n);
    if (st != KAN_OK) return st;
    if (rows == 0) return KAN_OK;
    const size_t es = dtype_size(dtype), ts = dtype_size(table_dtype);
    const size_t t = logits_bytes(classes, n, table_stride, ts);
    if (t == 0 || tokens == nullptr || table == nullptr || y == nullptr) return KAN_ERR_INVALID_ARG;
    if (!placed({{tokens, (size_t)rows * 8, 8}, {table, t, ts}}, {{y, (size_t)rows * n * es, es}}))
        return KAN_ERR_INVALID_ARG;
    const kan::EmbedArgs a = {tokens, table, y, rows, table_stride, classes, n, ignore_index, scale};
    return device_status(kan::launch_embed(dtype == KAN_BF16, table_dtype == KAN_BF16, a,
                                           static_cast<hipStream_t>(stream)));
}

kan_status kan_embedding_backward_workspace_bytes(int64_t rows, int32_t classes, int32_t n,
                                                  size_t* bytes) {
    if (bytes == nullptr) return KAN_ERR_INVALID_ARG;
    const kan_status st = check_embedding(rows, classes, n);
    if (st != KAN_OK) return st;
    *bytes = kan::embed_grad_workspace(rows, classes, n);
    return KAN_OK;
}

kan_status kan_embedding_backward(kan_dtype dtype, kan_dtype table_dtype, int64_t rows,
                                  int32_t classes, int32_t n, const int64_t* tokens,
                                  int64_t ignore_index, const void* dy, int64_t dy_stride,
                                  float scale, const void* base, void* dtable, void* workspace,
                                  size_t workspace_bytes, void* stream) {
    kan_status st = check_table(dtype, table_dtype, scale);
    if (st != KAN_OK) return st;
    st = check_embedding(rows, classes, n);
    if (st != KAN_OK) return st;
    const size_t es = dtype_size(dtype), ts = dtype_size(table_dtype);
    const size_t g = rows > 0 ? logits_bytes(rows, n, dy_stride, es) : 0;
    const size_t t = (size_t)classes * n * ts, need = kan::embed_grad_workspace(rows, classes, n);
    if (dtable == nullptr || workspace == nullptr || workspace_bytes < need ||
        (rows > 0 && (g == 0 || tokens == nullptr || dy == nullptr)))
        return KAN_ERR_INVALID_ARG;
    if (!placed({{tokens, (size_t)rows * 8, 8}, {dy, g, es}, {base == dtable ? nullptr : base, t, ts}},
                {{dtable, t, ts}, {workspace, need, 16}}))
        return KAN_ERR_INVALID_ARG;
    const kan::EmbedGradArgs a = {tokens, dy, base, dtable, rows, dy_stride, classes, n, ignore_index,
                                  scale};
    return device_status(kan::launch_embed_grad(dtype == KAN_BF16, table_dtype == KAN_BF16, a,
                                                workspace, static_cast<hipStream_t>(stream)));
}

kan_status kan_linear_logprobs_workspace_bytes(kan_dtype dtype, int64_t rows, int32_t classes,
                                               int32_t n, const void* x, int64_t x_stride,
                                               const void* weight, int64_t weight_stride,
                                               size_t* bytes) {
    if (bytes == nullptr) return KAN_ERR_INVALID_ARG;
    kan::HeadShape s;
    const kan_status st =
        head_shape(dtype, rows, classes, n, x, x_stride, weight, weight_stride, &s);
    if (st != KAN_OK) return st;
    *bytes = kan::head_workspace(s);
    return KAN_OK;
}

kan_status kan_linear_logprobs(kan_dtype dtype, int64_t rows, int32_t classes, int32_t n,
                               const void* x, int64_t x_stride, const void* weight,
                               int64_t weight_stride, float scale, const int64_t* targets,
                               int64_t ignore_index, float* logp, float* stats, int64_t* best,
                               void* workspace, size_t workspace_bytes, void* stream) {
    kan::HeadShape s;
    const kan_status st =
        head_shape(dtype, rows, classes, n, x, x_stride, weight, weight_stride, &s);
    if (st != KAN_OK) return st;
    if (!std::isfinite(scale)) return KAN_ERR_INVALID_ARG;
    if (rows == 0) return KAN_OK;
    const size_t es = dtype_size(dtype), need = kan::head_workspace(s), r = (size_t)rows * 4;
    if (x == nullptr || weight == nullptr || targets == nullptr || logp == nullptr ||
        stats == nullptr || workspace == nullptr || workspace_bytes < need)
        return KAN_ERR_INVALID_ARG;
    if (!placed({{x, logits_bytes(rows, n, x_stride, es), es},
                 {weight, logits_bytes(classes, n, weight_stride, es), es},
                 {targets, 2 * r, 8}},
                {{logp, r, 4}, {stats, 2 * r, 4}, {best, 2 * r, 8}, {workspace, need, 16}}))
        return KAN_ERR_INVALID_ARG;
    const kan::HeadArgs a = {x, weight, targets, ignore_index, scale, logp, stats, best};
    return device_status(kan::launch_head(s, a, workspace, static_cast<hipStream_t>(stream)));
}

kan_status kan_linear_logprobs_backward_workspace_bytes(
    kan_dtype dtype, int64_t rows, int32_t classes, int32_t n, const void* x, int64_t x_stride,
    const void* weight, int64_t weight_stride, size_t* bytes) {
    if (bytes == nullptr) return KAN_ERR_INVALID_ARG;
    kan::HeadShape s;
    const kan_status st =
        head_shape(dtype, rows, classes, n, x, x_stride, weight, weight_stride, &s);
    if (st != KAN_OK) return st;
    *bytes = kan::head_grad_workspace(s, true, true);
    return KAN_OK;
}

kan_status kan_linear_logprobs_backward(kan_dtype dtype, int64_t rows, int32_t classes, int32_t n,
                                        const void* x, int64_t x_stride, const void* weight,
                                        int64_t weight_stride, float scale, const int64_t* targets,
                                        int64_t ignore_index, const float* stats,
                                        const float* dlogp, void* dx, void* dweight,
                                        void* workspace, size_t workspace_bytes, void* stream) {
    kan::HeadShape s;
    const kan_status st =
        head_shape(dtype, rows, classes, n, x, x_stride, weight, weight_stride, &s);
    if (st != KAN_OK) return st;
    if (!std::isfinite(scale) || (dx == nullptr && dweight == nullptr)) return KAN_ERR_INVALID_ARG;
    const size_t es = dtype_size(dtype), r = (size_t)rows * 4;
    const size_t need = kan::head_grad_workspace(s, dx != nullptr, dweight != nullptr);
    if (rows > 0 && (x == nullptr || weight == nullptr || targets == nullptr || stats == nullptr ||
                     dlogp == nullptr || workspace == nullptr || workspace_bytes < need))
        return KAN_ERR_INVALID_ARG;
    if (!placed({{x, rows > 0 ? logits_bytes(rows, n, x_stride, es) : 0, es},
                 {weight, logits_bytes(classes, n, weight_stride, es), es},
                 {targets, 2 * r, 8},
                 {stats, 2 * r, 4},
                 {dlogp, r, 4}},
                {{dx, (size_t)rows * n * es, es},
                 {dweight, (size_t)classes * n * es, es},
                 {rows > 0 ? workspace : nullptr, need, 16}}))
        return KAN_ERR_INVALID_ARG;
    const kan::HeadGradArgs a = {x, weight, targets, ignore_index, scale, stats, dlogp, dx, dweight};
    return device_status(kan::launch_head_grad(s, a, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
