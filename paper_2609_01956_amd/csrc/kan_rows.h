// kan_rows.h -- device helpers of the kernels that work on rows (layer norm, log
// probabilities): 16-byte loads and stores at any alignment, and sums and maxima over
// groups of lanes.
#pragma once

#include "kan_device.h"

namespace kan {

// 16 bytes at the alignment of an element (the memory pipeline takes any; rows of odd
// length start anywhere).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Bytes from which an output is stored past the caches: it would push out what the next
// kernel reads, and takes longer (clipping 64 x 2^20 fp32 into other tensors 165 us against 136;
// 25 MB and below no different, and likely to be read next).
constexpr int64_t kPastCaches = INT64_C(64) << 20;

// Elements of T in 16 bytes.
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

__device__ __forceinline__ void widen(u32x4 r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r[i] << 16);
        v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(u32x4 r, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ u32x4 narrow(const float (&v)[8]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2 p = __builtin_convertvector((floatx2){v[2 * i], v[2 * i + 1]}, bf16x2);
        r[i] = __builtin_bit_cast(uint32_t, p);
    }
    return r;
}
__device__ __forceinline__ u32x4 narrow(const float (&v)[4]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
    return r;
}

// The unit from column c >= 0 on (a 32-bit byte offset from the row: one register, where
// the row is the wave's).
template <typename T>
__device__ __forceinline__ u32x4_any* unit_at(T* row, int c) {
    return reinterpret_cast<u32x4_any*>(reinterpret_cast<char*>(row) + (uint32_t)c * (uint32_t)sizeof(T));
}
template <typename T>
__device__ __forceinline__ const u32x4_any* unit_at(const T* row, int c) {
    return unit_at(const_cast<T*>(row), c);
}

// A unit's elements moved down by `bits` (16 .. 112), with those of `fill` (a pattern that
// repeats every 32 bits) above them.
__device__ __forceinline__ u32x4 shift_down(u32x4 r, int bits, uint32_t fill) {
    const uint64_t f = (uint64_t)fill << 32 | fill;
    const uint64_t lo = (uint64_t)r[1] << 32 | r[0], hi = (uint64_t)r[3] << 32 | r[2];
    const int s = bits & 63;
    // (twice by half of 64 - s, so that a shift by 64 is none: s may be 0)
    const uint64_t up = (hi >> s) | (f << 1 << (63 - s));
    const uint64_t low = (lo >> s) | (hi << 1 << (63 - s));
    const uint64_t l = bits >= 64 ? up : low, h = bits >= 64 ? f : up;
    return u32x4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}

// Rows as 16-byte units in registers.  A lane's N units of a row of n elements start at
// columns col + u step; the first FULL are known to lie within the row.  They come in two
// calls, so that loads can be in flight while other work goes on:
//
// issue_units loads.  A unit that ends past the row's end is loaded where it ends with it,
// and one that starts past it is too: one 16-byte load each, under no condition.  Rows
// shorter than a unit (TINY: there may be such) are loaded by elements.
//
// settle_units, before the units are used, moves the former into place and puts `fill` (bits
// of T) past the row's end.  There n may be 0 for lanes without a row, whatever they loaded.
template <int FULL, bool TINY, typename T, int N>
__device__ __forceinline__ void issue_units(const T* row, int col, int step, int n, uint32_t fill,
                                            u32x4 (&raw)[N]) {
    constexpr int V = kVec<T>;
    if (TINY && n < V) {
        const uint32_t f = sizeof(T) == 2 ? fill << 16 | fill : fill;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            raw[u] = u32x4{f, f, f, f};
            const int c = col + u * step;
#pragma unroll
            for (int i = 0; i + 1 < V; ++i) {
                if (c + i >= n) continue;
                if constexpr (sizeof(T) == 2)
                    raw[u][i / 2] = i % 2 ? (raw[u][i / 2] & 0xffffu) | (uint32_t)row[c + i] << 16
                                          : (raw[u][i / 2] & 0xffff0000u) | row[c + i];
                else
                    raw[u][i] = __float_as_uint(row[c + i]);
            }
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int c = col + u * step;
        raw[u] = *unit_at(row, u < FULL ? c : min(c, n - V));
    }
}

template <int FULL, bool TINY, typename T, int N>
__device__ __forceinline__ void settle_units(int col, int step, int n, uint32_t fill,
                                             u32x4 (&raw)[N]) {
    constexpr int V = kVec<T>;
    const uint32_t f = sizeof(T) == 2 ? fill << 16 | fill : fill;
    if (n % V != 0 && !(TINY && n < V)) {
        const int bits = (V - n % V) * 8 * (int)sizeof(T);
#pragma unroll
        for (int u = FULL; u < N; ++u) {
            const u32x4 moved = shift_down(raw[u], bits, f);
            const bool ends = col + u * step + V > n;
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[u][i] = ends ? moved[i] : raw[u][i];
        }
    }
#pragma unroll
    for (int u = FULL; u < N; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[u][i] = col + u * step < n ? raw[u][i] : f;
}

// One unit as fp32, of a row of any length.
template <typename T, int V>
__device__ __forceinline__ void load_unit(const T* row, int col, int n, uint32_t fill,
                                          float (&v)[V]) {
    static_assert(V == kVec<T>, "one unit");
    u32x4 raw[1];
    issue_units<0, true>(row, col, 0, n, fill, raw);
    settle_units<0, true, T>(col, 0, n, fill, raw);
    widen(raw[0], v);
}

// Bits of -infinity.
template <typename T> constexpr uint32_t kNegInfBits = sizeof(T) == 2 ? 0xff80u : 0xff800000u;

// One unit of a row of n elements, those within the row: the last unit's n % V elements as
// 8, 4 and 2 bytes.  PAST: whole units go past the caches (outputs that do not fit there).
template <bool FULL, bool PAST = false, typename T, int V>
__device__ __forceinline__ void store_unit(T* row, int col, int n, const float (&v)[V]) {
    static_assert(V == kVec<T>, "one unit");
    typedef uint32_t u32_any __attribute__((aligned(2)));
    typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    const u32x4 r = narrow(v);
    if (FULL || col + V <= n) {
        if constexpr (PAST) __builtin_nontemporal_store(r, unit_at(row, col));
        else *unit_at(row, col) = r;
        return;
    }
    if (col >= n) return;
    const int left = n - col;
    constexpr int W = 4 / (int)sizeof(T);  // elements per word
    T* p = row + col;
    if (left & (2 * W)) *reinterpret_cast<u32x2_any*>(p) = (u32x2_any){r[0], r[1]};
    if (left & W)
        *reinterpret_cast<u32_any*>(p + (left & (2 * W))) = left & (2 * W) ? r[2] : r[0];
    if (W == 2 && (left & 1)) {
        const uint32_t w = left & 4 ? (left & 2 ? r[3] : r[2]) : left & 2 ? r[1] : r[0];
        p[left & 6] = (T)w;
    }
}

// V parameters (of the rows' own type or fp32) from column col on, `fill` past the end or
// where there are none (p == nullptr).
template <bool TINY, typename TP, int V>
__device__ __forceinline__ void load_params(const TP* p, int col, int n, float fill,
                                            float (&v)[V]) {
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = fill;
        return;
    }
    constexpr int U = kVec<TP>;
    u32x4 raw[V / U];
    const uint32_t f = sizeof(TP) == 2 ? __float_as_uint(fill) >> 16 : __float_as_uint(fill);
    issue_units<0, TINY>(p, col, U, n, f, raw);
    settle_units<0, TINY, TP>(col, U, n, f, raw);
#pragma unroll
    for (int k = 0; k < V / U; ++k) {
        float u[U];
        widen(raw[k], u);
#pragma unroll
        for (int i = 0; i < U; ++i) v[k * U + i] = u[i];
    }
}

// Every lane's value from another lane of its row of 16, by a DPP pattern.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float dppf(float v) {
    return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
// The previous lane's value (lane 0 keeps its own).
__device__ __forceinline__ uint32_t dpp_shr(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x138, 0xf, 0xf, false);
}
constexpr int kDppFlip4 = 0x1B;        // quad_perm [3, 2, 1, 0]
constexpr int kDppRor8 = 0x128;        // lane i of 16 <- (i + 8) % 16
constexpr int kDppXor1 = 0xB1;         // quad_perm [1, 0, 3, 2]
constexpr int kDppXor2 = 0x4E;         // quad_perm [2, 3, 0, 1]
constexpr int kDppHalfMirror = 0x141;  // lane i of 8 <-> 7 - i
constexpr int kDppMirror = 0x140;      // lane i of 16 <-> 15 - i

// op over the `lanes` (a power of two) neighbouring lanes of each group; every lane
// gets the same bits (each step adds the same two values in either order).  All lanes
// of the wave take part.
template <typename Op>
__device__ __forceinline__ float group_reduce(float v, int lanes, Op op) {
    if (lanes > 1) v = op(v, dppf<kDppXor1>(v));
    if (lanes > 2) v = op(v, dppf<kDppXor2>(v));
    // (the groups of 4, then of 8, hold one value each: a mirror swaps neighbours)
    if (lanes > 4) v = op(v, dppf<kDppHalfMirror>(v));
    if (lanes > 8) v = op(v, dppf<kDppMirror>(v));
    if (lanes > 16) v = op(v, __shfl_xor(v, 16));
    if (lanes > 32) v = op(v, __shfl_xor(v, 32));
    return v;
}
__device__ __forceinline__ float group_sum(float v, int lanes) {
    return group_reduce(v, lanes, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float group_max(float v, int lanes) {
    return group_reduce(v, lanes, [](float a, float b) { return __builtin_fmaxf(a, b); });
}

// The same over all 64 lanes, in fewer steps: the last two rows of 16 are reached by
// broadcasts, and the last lane's value is read (uniform over the wave).
template <typename Op>
__device__ __forceinline__ float wave_reduce(float v, float none, Op op) {
    v = op(v, dppf<kDppXor1>(v));
    v = op(v, dppf<kDppXor2>(v));
    v = op(v, dppf<kDppHalfMirror>(v));
    v = op(v, dppf<kDppMirror>(v));
    const int z = (int)__float_as_uint(none);
    // row 0 to row 1 and row 2 to row 3, then row 1 to rows 2 and 3
    v = op(v, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                  z, (int)__float_as_uint(v), 0x142, 0xa, 0xf, false)));
    v = op(v, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                  z, (int)__float_as_uint(v), 0x143, 0xc, 0xf, false)));
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}
__device__ __forceinline__ float wave_sum(float v) {
    return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_reduce(v, -__builtin_huge_valf(),
                       [](float a, float b) { return __builtin_fmaxf(a, b); });
}

}  // namespace kan
