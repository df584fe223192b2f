// kan_clip_lists.h -- host check of the tensor lists of the gradient clipping.
#pragma once

#include <algorithm>
#include <cstdint>

#include "kan_ops.h"

namespace kan {

// Does any output overlap another output, or an input that is not its own in place?  (Tensors of
// no elements are not looked at.)
//
// Outputs are taken in blocks, sorted by address: disjoint ones overlap another tensor only if
// the last of them that starts before its end does.  A block is 16 KB on the stack whatever the
// count, as nothing is allocated and a caller's thread may have little (all outputs and inputs,
// sorted at once, took 128 KB).  Lists in order of address cost two comparisons per block and
// tensor, others a search (16384 shuffled tensors: 1.9 ms; in blocks of 1024 9.6 ms).
template <int BLOCK = 8192>
bool clip_outputs_clash(const ClipList& l) {
    static_assert(kClipMaxTensors <= 1 << 16, "16-bit tensor numbers");
    uint16_t block[BLOCK];
    auto size = [&](int64_t t) { return (uintptr_t)l.sizes[t] * (l.bf16(t) ? 2 : 4); };
    auto start = [&](int64_t t) { return reinterpret_cast<uintptr_t>(l.out[t]); };
    auto end = [&](int64_t t) { return start(t) + size(t); };
    auto before = [&](uint16_t a, uint16_t b) { return start(a) < start(b); };
    for (int64_t from = 0, to = 0; from < l.count; from = to) {
        int n = 0;
        for (; to < l.count && n < BLOCK; ++to)
            if (l.sizes[to] > 0) block[n++] = (uint16_t)to;
        if (n == 0) break;
        if (!std::is_sorted(block, block + n, before)) std::sort(block, block + n, before);
        for (int k = 1; k < n; ++k)
            if (start(block[k]) < end(block[k - 1])) return true;
        const uintptr_t lo = start(block[0]), hi = end(block[n - 1]);
        auto hits = [&](const void* p, uintptr_t bytes) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = a + bytes;
            if (a >= hi || b <= lo) return false;
            const uint16_t* it =
                std::lower_bound(block, block + n, b,
                                 [&](uint16_t t, uintptr_t v) { return start(t) < v; });
            return it != block && end(it[-1]) > a;
        };
        for (int64_t t = 0; t < l.count; ++t) {
            if (l.sizes[t] == 0) continue;
            if (l.in[t] != l.out[t] && hits(l.in[t], size(t))) return true;
            if (t >= to && hits(l.out[t], size(t))) return true;
        }
    }
    return false;
}

}  // namespace kan
