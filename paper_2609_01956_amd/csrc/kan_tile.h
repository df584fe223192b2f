// kan_tile.h -- a workgroup's tile of out[q][p] = sum_k P[p][k] Q[q][k] on the matrix cores, both
// operands with k contiguous, in bf16 or fp32 with fp32 accumulation.
//
// A step takes 128 bytes of k (64 bf16, 32 fp32) of the tile's rows into LDS, straight from
// memory (16 bytes per lane, no registers between), two steps' buffers in turn: the next step's
// loads are in flight while this one's products run, one barrier per step.  In LDS a row's eight
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
    static constexpr int STAGE = (BP + BQ) * 128, BYTES = 2 * STAGE;
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

    // The products of the step in `src` (its lane's rows at pp and qq), while the next one's
    // loads go to `dst`.
    __device__ __forceinline__ void step(const char KAN_LDS* __restrict src,
                                         char KAN_LDS* __restrict dst, const TileRows& p,
                                         const TileRows& q, const uint32_t (&vp)[IP],
                                         const uint32_t (&vq)[IQ], bool more, bool past, int at,
                                         int wave, int pp, int qq, int half, int swz) {
        if (more) issue(p, q, vp, vq, past, at, dst, wave);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int chunk = ((2 * c + half) ^ swz) * 16;
            u32x4 a[RP], b[RQ];
#pragma unroll
            for (int i = 0; i < RP; ++i)
                a[i] = *(const u32x4 KAN_LDS*)(src + pp + i * 32 * 128 + chunk);
#pragma unroll
            for (int j = 0; j < RQ; ++j)
                b[j] = *(const u32x4 KAN_LDS*)(src + BP * 128 + qq + j * 32 * 128 + chunk);
#pragma unroll
            for (int i = 0; i < RP; ++i)
#pragma unroll
                for (int j = 0; j < RQ; ++j) multiply(a[i], b[j], acc[i][j]);
        }
    }

    // k_bytes: a multiple of 16.  lds: BYTES.
    __device__ __forceinline__ void run(char KAN_LDS* lds, const TileRows& p, const TileRows& q,
                                        int64_t k_from, int64_t k_bytes) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int j = 0; j < RQ; ++j) acc[i][j] = floatx16{};
        // a load's 64 lanes: eight rows of eight chunks, the chunk that stands there
        const int row = lane >> 3, chunk = (lane & 7) ^ row;
        uint32_t vp[IP], vq[IQ];
#pragma unroll
        for (int i = 0; i < IP; ++i) vp[i] = ((wave * IP + i) * 8 + row) * p.stride + chunk * 16;
#pragma unroll
        for (int i = 0; i < IQ; ++i) vq[i] = ((wave * IQ + i) * 8 + row) * q.stride + chunk * 16;
        const int pp = ((wave % WP) * 32 * RP + (lane & 31)) * 128;
        const int qq = ((wave / WP) * 32 * RQ + (lane & 31)) * 128;
        const int half = lane >> 5, swz = lane & 7;
        const int end = (int)(k_from + k_bytes);
        const int steps = (int)((k_bytes + 127) >> 7);
        int at = (int)k_from;
        issue(p, q, vp, vq, at + chunk * 16 >= end, at, lds, wave);
        for (int k = 0; k < steps; k += 2) {
            arrive();
            at += 128;
            step(lds, lds + STAGE, p, q, vp, vq, k + 1 < steps, at + chunk * 16 >= end, at, wave, pp,
                 qq, half, swz);
            if (k + 1 >= steps) break;
            arrive();
            at += 128;
            step(lds + STAGE, lds, p, q, vp, vq, k + 2 < steps, at + chunk * 16 >= end, at, wave, pp,
                 qq, half, swz);
        }
        arrive();
    }

    // The q of this lane's accumulators acc[.][j] and the p of acc[i][.][4 v + (0 .. 3)], within the tile.
    static __device__ __forceinline__ int q_of(int j) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        return (wave / WP) * 32 * RQ + j * 32 + (lane & 31);
    }
    static __device__ __forceinline__ int p_of(int i, int v) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
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
