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

// Elements col .. col + V - 1 of a row of n elements as fp32, V = one 16-byte unit; past
// the row's end `fill`.  FULL: the unit is known to lie within the row.
template <bool FULL, typename T, int V>
__device__ __forceinline__ void load_unit(const T* row, int col, int n, float fill, float (&v)[V]) {
    static_assert(V == kVec<T>, "one unit");
    if (FULL || col + V <= n) {
        widen(*reinterpret_cast<const u32x4_any*>(row + col), v);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = col + i < n ? Storage<T>::load(row + col + i) : fill;
}

template <bool FULL, typename T, int V>
__device__ __forceinline__ void store_unit(T* row, int col, int n, const float (&v)[V]) {
    static_assert(V == kVec<T>, "one unit");
    if (FULL || col + V <= n) {
        *reinterpret_cast<u32x4_any*>(row + col) = narrow(v);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (col + i < n) Storage<T>::store(row + col + i, v[i]);
}

// V parameters (of T's own type or fp32) from column col on, `fill` past the end or
// where there are none (p == nullptr).
template <typename TP, int V>
__device__ __forceinline__ void load_params(const TP* p, int col, int n, float fill,
                                            float (&v)[V]) {
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = fill;
        return;
    }
    constexpr int U = kVec<TP>;
#pragma unroll
    for (int k = 0; k < V / U; ++k) {
        float u[U];
        load_unit<false>(p, col + k * U, n, fill, u);
#pragma unroll
        for (int i = 0; i < U; ++i) v[k * U + i] = u[i];
    }
}

// One lane's value moved by a DPP pattern (lanes without a source keep `old`).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, 0xf, 0xf, false);
}
template <int CTRL>
__device__ __forceinline__ float dppf(float v) {
    const uint32_t u = __float_as_uint(v);
    return __uint_as_float(dpp<CTRL>(u, u));
}
constexpr int kDppXor1 = 0xB1;         // quad_perm [1, 0, 3, 2]
constexpr int kDppXor2 = 0x4E;         // quad_perm [2, 3, 0, 1]
constexpr int kDppHalfMirror = 0x141;  // lane i of 8 <-> 7 - i
constexpr int kDppMirror = 0x140;      // lane i of 16 <-> 15 - i
constexpr int kDppWaveShr1 = 0x138;    // lane i <- lane i - 1

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

}  // namespace kan
