// kan_checks.h -- argument checks shared by the C ABI of the operators around the layer (host only).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

#include "kan.h"

namespace kan {

inline size_t dtype_size(kan_dtype dt) { return dt == KAN_BF16 ? 2 : 4; }
inline bool known(kan_dtype dt) { return dt == KAN_F32 || dt == KAN_BF16; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline kan_status device_status(hipError_t e) { return e == hipSuccess ? KAN_OK : KAN_ERR_DEVICE; }

// `n` bytes at p (p NULL: not given), of elements of `a` bytes.
struct Buf {
    const void* p;
    size_t n;
    size_t a;
};

inline bool overlap(const Buf& x, const Buf& y) {
    if (x.p == nullptr || y.p == nullptr || x.n == 0 || y.n == 0) return false;
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
    return a < b + y.n && b < a + x.n;
}

// Every buffer aligned to its elements, no output over another output or an input.
inline bool placed(std::initializer_list<Buf> ins, std::initializer_list<Buf> outs) {
    for (const Buf& i : ins)
        if (!aligned(i.p, i.a)) return false;
    for (const Buf* o = outs.begin(); o != outs.end(); ++o) {
        if (!aligned(o->p, o->a)) return false;
        for (const Buf& i : ins)
            if (overlap(*o, i)) return false;
        for (const Buf* q = outs.begin(); q != o; ++q)
            if (overlap(*o, *q)) return false;
    }
    return true;
}

// Rows of n elements: sizes that the kernels' indexes hold.
inline kan_status check_rows(int64_t rows, int32_t n, int32_t most) {
    if (rows < 0 || n < 1 || n > most) return KAN_ERR_INVALID_ARG;
    if (rows > (INT64_C(1) << 48) / n) return KAN_ERR_INVALID_ARG;
    return KAN_OK;
}

// Bytes from the first to past the last logit of rows `stride` elements apart; 0 for
// strides that rows of `classes` elements do not fit or that pass the indexes.
inline size_t logits_bytes(int64_t rows, int32_t classes, int64_t stride, size_t es) {
    if (stride < classes || rows > (INT64_C(1) << 48) / stride) return 0;
    return ((size_t)(rows - 1) * stride + classes) * es;
}

}  // namespace kan
