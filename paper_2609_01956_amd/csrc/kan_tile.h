// kan_tile.h -- a workgroup's tile of out[q][p] = sum_k P[p][k] Q[q][k] on the matrix cores, both
// operands with k contiguous, in bf16 or fp32 with fp32 accumulation.
//
// A step takes 128 bytes of k (64 bf16, 32 fp32) of the tile's rows into LDS, straight from
// memory (16 bytes per lane, no registers between), two steps' buffers in turn: the next step's
// loads are in flight while this one's products run, one barrier per step, before its last quarter.  In LDS a row's eight
// 16-byte chunks stand at chunk ^ (row & 7), so that eight lanes that read one chunk of eight
// rows use all banks.  Rows past an operand's end are 0 (the buffer's bounds), and so are chunks
// past k's end; k must be a whole number of chunks, rows 16-byte aligned.
//
// Each wave holds RP x RQ tiles of 32 x 32: a lane's accumulators are 16 values of p (in fours of
// neighbours) for one q, so that sums over p stay in the lane.
#pragma once

#include "kan_device.h"

namespace kan {

#define KAN_LDS __attribute__((address_space(3)))

// One operand's rows of a tile, from the tile's first row on.
struct TileRows {
    __amdgpu_buffer_rsrc_t rsrc;
    uint32_t stride;  // bytes from row to row
};

// rows: from the tile's first on (at least 1); es bytes an element, k elements a row.
__device__ __forceinline__ TileRows tile_rows(const void* p, int64_t first, int64_t rows, int most,
                                              int64_t stride_bytes, int64_t k_bytes) {
    const int64_t left = rows - first < most ? rows - first : most;
    const char* at = static_cast<const char*>(p) + first * stride_bytes;
    TileRows t;
    t.rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0,
                                               (int)((left - 1) * stride_bytes + k_bytes),
                                               kBufferWord3);
    t.stride = (uint32_t)stride_bytes;
    return t;
}

template <typename T, int WP_, int WQ_, int RP_, int RQ_>
struct Tile {
    static constexpr int WP = WP_, WQ = WQ_, RP = RP_, RQ = RQ_;
    static constexpr int W = WP * WQ, THREADS = 64 * W;
    static constexpr int BP = 32 * RP * WP, BQ = 32 * RQ * WQ;
    static constexpr int STAGE = (BP + BQ) * 128;
    // (LDS of a workgroup: two steps, or rows of fp32 results)
    static constexpr int BYTES = 2 * STAGE > 32 * WQ * (BP * 4 + 16) ? 2 * STAGE : 32 * WQ * (BP * 4 + 16);
    static constexpr int IP = BP / 8 / W, IQ = BQ / 8 / W;  // loads per wave and step
    static_assert(BP % (8 * W) == 0 && BQ % (8 * W) == 0, "whole loads");

    floatx16 acc[RP][RQ];

    // (the order in which the compiler may move memory accesses: not past these)
    static __device__ __forceinline__ void arrive() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }

    static __device__ __forceinline__ void issue(const TileRows& p, const TileRows& q,
                                                 const uint32_t (&vp)[IP], const uint32_t (&vq)[IQ],
                                                 bool past, int at, char KAN_LDS* dst, int wave) {
#pragma unroll
        for (int i = 0; i < IP; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                p.rsrc, (void KAN_LDS*)(dst + (wave * IP + i) * 1024), 16,
                (int)(past ? 0x80000000u : vp[i]), at, 0, 0);
#pragma unroll
        for (int i = 0; i < IQ; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                q.rsrc, (void KAN_LDS*)(dst + BP * 128 + (wave * IQ + i) * 1024), 16,
                (int)(past ? 0x80000000u : vq[i]), at, 0, 0);
    }

    __device__ __forceinline__ void multiply(const u32x4& a, const u32x4& b, floatx16& c) {
        if constexpr (sizeof(T) == 2) {
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                        __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]),
                                                         __uint_as_float(b[i]), c, 0, 0, 0);
        }
    }

    // The fragments of the c-th quarter of a step.
    static __device__ __forceinline__ void fetch(const char KAN_LDS* src, int pp, int qq, int chunk,
                                                 u32x4 (&a)[RP], u32x4 (&b)[RQ]) {
#pragma unroll
        for (int i = 0; i < RP; ++i)
            a[i] = *(const u32x4 KAN_LDS*)(src + pp + i * 32 * 128 + chunk);
#pragma unroll
        for (int j = 0; j < RQ; ++j)
            b[j] = *(const u32x4 KAN_LDS*)(src + BP * 128 + qq + j * 32 * 128 + chunk);
    }
    __device__ __forceinline__ void products(const u32x4 (&a)[RP], const u32x4 (&b)[RQ]) {
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int j = 0; j < RQ; ++j) multiply(a[i], b[j], acc[i][j]);
    }

    struct Lane {
        uint32_t vp[IP], vq[IQ];  // its loads' places in the operands
        int pp, qq;               // its rows in LDS
        int chunk[4];             // its chunk of a row in each quarter of a step
        int wave, tail;           // tail: bytes of k before its loads' chunk
    };

    // One step from `cur`, whose first quarter's fragments are at hand; they end as those of the step
    // in `nxt`.  Before the last quarter's products all waves have read `cur` (and `nxt` has
    // arrived), so that the loads of the step after the next go there while these products, and
    // the next step's, run.
    __device__ __forceinline__ void step(char KAN_LDS* cur, const char KAN_LDS* nxt,
                                         const TileRows& p, const TileRows& q, const Lane& l,
                                         int at, int end, u32x4 (&a)[2][RP], u32x4 (&b)[2][RQ]) {
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            fetch(cur, l.pp, l.qq, l.chunk[c + 1], a[(c + 1) & 1], b[(c + 1) & 1]);
            products(a[c & 1], b[c & 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        arrive();
        __builtin_amdgcn_sched_barrier(0);
        if (at < end) issue(p, q, l.vp, l.vq, at + l.tail >= end, at, cur, l.wave);
        fetch(nxt, l.pp, l.qq, l.chunk[0], a[0], b[0]);
        products(a[1], b[1]);
        __builtin_amdgcn_sched_barrier(0);
    }

    // (The two buffers are told apart by the compiler: reads of one do not wait for loads to the
    // other.)
    __device__ __forceinline__ void steps(char KAN_LDS* __restrict b0, char KAN_LDS* __restrict b1,
                                          const TileRows& p, const TileRows& q, const Lane& l,
                                          int at, int end) {
        u32x4 a[2][RP], b[2][RQ];
        issue(p, q, l.vp, l.vq, at + l.tail >= end, at, b0, l.wave);
        int next = at + 128;
        if (next < end) issue(p, q, l.vp, l.vq, next + l.tail >= end, next, b1, l.wave);
        arrive();
        fetch(b0, l.pp, l.qq, l.chunk[0], a[0], b[0]);
        // (one way out of the loop: with two the accumulators are moved about in it)
        for (; at + 128 < end; at += 256) {
            step(b0, b1, p, q, l, at + 256, end, a, b);
            step(b1, b0, p, q, l, at + 384, end, a, b);
        }
        if (at < end) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c < 3) fetch(b0, l.pp, l.qq, l.chunk[c + 1], a[(c + 1) & 1], b[(c + 1) & 1]);
                products(a[c & 1], b[c & 1]);
            }
        }
        arrive();
    }

    // The sum over k of [k_from, k_from + k_bytes), multiples of 16.  lds: BYTES.
    __device__ __forceinline__ void run(char KAN_LDS* lds, const TileRows& p, const TileRows& q,
                                        int64_t k_from, int64_t k_bytes) {
        const int lane = threadIdx.x & 63;
        Lane l;
        l.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int j = 0; j < RQ; ++j) acc[i][j] = floatx16{};
        // a load's 64 lanes: eight rows of eight chunks, the chunk that stands there
        const int row = lane >> 3, chunk = (lane & 7) ^ row;
        l.tail = chunk * 16;
#pragma unroll
        for (int i = 0; i < IP; ++i) l.vp[i] = ((l.wave * IP + i) * 8 + row) * p.stride + chunk * 16;
#pragma unroll
        for (int i = 0; i < IQ; ++i) l.vq[i] = ((l.wave * IQ + i) * 8 + row) * q.stride + chunk * 16;
        l.pp = ((l.wave % WP) * 32 * RP + (lane & 31)) * 128;
        l.qq = ((l.wave / WP) * 32 * RQ + (lane & 31)) * 128;
#pragma unroll
        for (int c = 0; c < 4; ++c) l.chunk[c] = ((2 * c + (lane >> 5)) ^ (lane & 7)) * 16;
        steps(lds, lds + STAGE, p, q, l, (int)k_from, (int)(k_from + k_bytes));
    }

    // Values v(i, e, acc[i][j][e]) of this thread's q of j as T in LDS, rows (one per q of the
    // workgroup's waves, ROWS in all) of BP values, PITCH bytes apart.
    static constexpr int ROWS = 32 * WQ;
    template <typename U> static constexpr int PITCH = BP * (int)sizeof(U) + 16;
    template <typename U, typename F>
    __device__ __forceinline__ void put(char* lds, int thread, int j, F&& v) {
        typedef U four __attribute__((ext_vector_type(4)));
        const int wave = thread >> 6, lane = thread & 63;
        char* const row = lds + ((wave / WP) * 32 + (lane & 31)) * PITCH<U> +
                          ((wave % WP) * 32 * RP + 4 * (lane >> 5)) * (int)sizeof(U);
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<four*>(row + (i * 32 + g * 8) * (int)sizeof(U)) =
                    four{v(i, 4 * g, acc[i][j][4 * g]), v(i, 4 * g + 1, acc[i][j][4 * g + 1]),
                         v(i, 4 * g + 2, acc[i][j][4 * g + 2]), v(i, 4 * g + 3, acc[i][j][4 * g + 3])};
    }
    // The q, within the tile, of a row that `put` filled.
    static __device__ __forceinline__ int q_of_row(int row, int j) {
        return (row >> 5) * 32 * RQ + j * 32 + (row & 31);
    }

    // This thread, computed anew after the loop (so that nothing derived from it lives across it).
    static __device__ __forceinline__ int thread() {
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
        return t;
    }

    // The q of a thread's accumulators acc[.][j] and the p of acc[i][.][4 v + (0 .. 3)], within the
    // tile.
    static __device__ __forceinline__ int q_of(int thread, int j) {
        const int wave = thread >> 6, lane = thread & 63;
        return (wave / WP) * 32 * RQ + j * 32 + (lane & 31);
    }
    static __device__ __forceinline__ int p_of(int thread, int i, int v) {
        const int wave = thread >> 6, lane = thread & 63;
        return (wave % WP) * 32 * RP + i * 32 + 8 * v + 4 * (lane >> 5);
    }
};

// A workgroup's tile of tp x tq tiles: neighbouring workgroups go to different XCDs, each of
// which takes a run of tiles, in blocks of up to eight q-tiles by all p-tiles, so that those that
// run at a time on an XCD share rows of both operands in its L2.
__device__ __forceinline__ void tile_of(int id, int tp, int tq, int* p, int* q) {
    const int all = tp * tq, xcd = id & 7, per = all >> 3, rest = all & 7;
    const int t = xcd * per + (xcd < rest ? xcd : rest) + (id >> 3);
    const int band = t / (8 * tp), first = band * 8, height = tq - first < 8 ? tq - first : 8;
    const int in = t - band * 8 * tp;
    *p = in / height;
    *q = first + in % height;
}

}  // namespace kan
