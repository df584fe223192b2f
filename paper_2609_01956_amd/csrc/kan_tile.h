// kan_tile.h -- a workgroup's tile of out[q][p] = sum_k P(p, k) Q(q, k) on the matrix cores, in bf16
// or fp32 with fp32 accumulation.  Each operand stands in memory by rows (of p or q, k contiguous) or
// by k (rows of k, p or q contiguous), so that no product needs a transposed copy.
//
// A step takes 64 (bf16) or 32 (fp32) values of k of both operands into LDS, straight from memory
// (16 bytes per lane, no registers between), into one of two buffers; a step is 64 KB for a tile of
// 256 x 256.  One barrier a step, before the last quarter of its products, tells that the next
// step has arrived and that all waves have read this one, whose buffer then takes the loads of
// the step after the next.  Fragments are read a quarter ahead of their products.
//
// In LDS:
//   by rows  128 bytes a row, its eight 16-byte chunks at chunk ^ (row >> 1 & 7): sixteen lanes that
//            read one chunk of sixteen rows use all banks (with row & 7 they used half)
//   by k     (bf16) a row per k; fragments come from the LDS's transposing read (four k of 16 columns
//            for 16 lanes), whose four rows stand in different quarters of the banks, 64-byte
//            blocks at block ^ (k & 3)
// What lies past an operand's end is 0 (the buffer's bounds).  By rows, k must be a whole number of
// 16-byte chunks; rows are 16-byte aligned in both, and end with a chunk.  By k, columns past the end hold what follows:
// they reach outputs past the end only.
//
// Each wave holds RP x RQ tiles of 32 x 32: a lane's accumulators are 16 values of p (in fours of
// neighbours) for one q, so that sums over p stay in the lane.
//
// Measured on MI355X, 8192 x 8192, bf16, 256 x 256 tiles: k = 8192 1.21 PFLOP/s, 2048 1.06; without
// any loads, in LDS or to it, 1.61: the products alone hold the card at its power limit.  Steps of
// half the size in a ring of five, four in flight: 1.18 and 1.00.  Four waves of 128 x 128: 1.17
// and 0.99; tiles of 128 x 128, two workgroups a CU: 1.03 and 0.94.
#pragma once

#include "kan_device.h"

namespace kan {

#define KAN_LDS __attribute__((address_space(3)))

// An operand: `rows` of p (or q) by k elements, or k rows by `rows` elements; the tile's part begins at
// row (column) `first`.
struct Operand {
    const char* at;   // the tile's first element, at k = 0
    uint32_t stride;  // bytes from row to row
    int left;         // rows (columns) of the tile that there are
    int64_t k;        // by k: rows that there are (0 past them, up to the sum's end)
    // fp32 as bf16 terms: bytes from a term to the next, and the terms (4 bits each) that the sum's
    // segments take
    int64_t plane;
    uint32_t terms;
};

constexpr int kByRows = 0, kByK = 1;

template <typename T, int MODE>
__device__ __forceinline__ Operand operand(const void* p, int64_t first, int64_t rows, int most,
                                           int64_t stride_bytes, int64_t k = 0, int64_t plane = 0,
                                           uint32_t terms = 0) {
    Operand o;
    o.at = static_cast<const char*>(p) + first * (MODE == kByRows ? stride_bytes : (int64_t)sizeof(T));
    o.stride = (uint32_t)stride_bytes;
    o.left = (int)(rows - first < most ? rows - first : most);
    o.k = k;
    o.plane = plane;
    o.terms = terms;
    return o;
}

template <typename T, int W, int B, int R, int MODE>
struct Side {
    static constexpr int ES = (int)sizeof(T), K = 128 / ES;  // k of a step
    static constexpr int LOADS = B / 8 / W;                  // per wave and step
    static constexpr int BYTES = B * 128;                    // of a step
    static constexpr int ROW = B * ES, CHUNKS = ROW / 16;    // by k: a row in LDS
    static_assert(B % (8 * W) == 0, "whole loads");
    static_assert(MODE == kByRows || ES == 2, "operands by k are bf16");

    uint32_t from[LOADS];  // the lane's loads in a step's part of the operand
    int tail;              // by rows: bytes of k before the lane's chunk (of even loads)
    int read[MODE == kByRows ? 1 : R], chunk[4];  // its fragments in LDS

    // wave: among W; part: which R x 32 rows of the B are the wave's.
    __device__ __forceinline__ void place(int lane, int wave, int part, uint32_t stride) {
        if constexpr (MODE == kByRows) {
            // a load's 64 lanes: eight rows of eight chunks, the chunk that stands there
            const int row = lane >> 3, c = (lane & 7) ^ (row >> 1);
            tail = c * 16;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int load = wave * LOADS + i;
                from[i] = (load * 8 + row) * stride + ((c ^ ((load & 1) * 4)) * 16);
            }
            read[0] = (part * 32 * R + (lane & 31)) * 128;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                chunk[q] = ((2 * q + (lane >> 5)) ^ (lane >> 1 & 7)) * 16;
        } else {
            tail = 0;
            constexpr int PER = 64 / CHUNKS;  // rows of a load
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int row = (wave * LOADS + i) * PER + lane / CHUNKS, c = lane % CHUNKS;
                from[i] = row * stride + (c ^ (row & 3) << 2) * 16;
            }
            // (its quarter of the wave's four k, its 16 columns' 32 bytes and its 8 of them)
            const int k = (lane >> 5) * 8 + (lane >> 2 & 3);
#pragma unroll
            for (int i = 0; i < R; ++i)
                read[i] = k * ROW + ((part * R + i) ^ (k & 3)) * 64 + (lane >> 4 & 1) * 32 +
                          (lane & 3) * 8;
        }
    }

    // The loads of the step of segment `seg` that begins at k (of `end`; none past it: zeros) to LDS
    // byte dst.
    __device__ __forceinline__ void issue(const Operand& o, int seg, int64_t k, int64_t end, int wave,
                                          uint32_t dst) const {
        const char* at = o.at + (MODE == kByRows ? 0 : k * o.stride) +
                         (int64_t)(o.terms >> 4 * seg & 15) * o.plane;
        const int64_t there = end < o.k ? end : o.k;
        const int rows = MODE == kByRows ? o.left : (int)(there - k < K ? there - k : K);
        // (bounds are kept by 4 bytes: by k, the last row to the end of its last chunk)
        const int64_t width = MODE == kByRows ? end * ES : ((int64_t)o.left * ES + 15) & ~15;
        const uint64_t base = reinterpret_cast<uint64_t>(at);
        const u32x4 rsrc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu,
                            rows > 0 ? (uint32_t)((int64_t)(rows - 1) * o.stride + width) : 0u,
                            (uint32_t)kBufferWord3};
        const int bytes = (int)(end - k < K ? end - k : K) * ES;  // of the step's k
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uint32_t v = from[i];
            if constexpr (MODE == kByRows) {
                const int c = tail ^ (((wave * LOADS + i) & 1) * 64);
                v = c >= bytes ? 0x80000000u : v;
            }
            dma16(rsrc, v, MODE == kByRows ? (uint32_t)(k * ES) : 0u, dst + (wave * LOADS + i) * 1024);
        }
    }

    // The fragments of a quarter of a step at src.
    __device__ __forceinline__ void fetch(const char KAN_LDS* src, int quarter, u32x4 (&f)[R]) const {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if constexpr (MODE == kByRows) {
                f[i] = *(const u32x4 KAN_LDS*)(src + read[0] + chunk[quarter] + i * 32 * 128);
            } else {
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                const char KAN_LDS* p = src + read[i] + quarter * 16 * ROW;
                const u32x2 lo = __builtin_bit_cast(
                    u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 KAN_LDS*)p));
                const u32x2 hi = __builtin_bit_cast(
                    u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 KAN_LDS*)(p + 4 * ROW)));
                f[i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
            }
        }
    }

    typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
};

// SEGS: the sum is one of so many, each over all of k, of terms that the operands name.
template <typename T, int WP_, int WQ_, int RP_, int RQ_, int MP, int MQ, int SEGS = 1>
struct Tile {
    static constexpr int WP = WP_, WQ = WQ_, RP = RP_, RQ = RQ_;
    static constexpr int W = WP * WQ, THREADS = 64 * W;
    static constexpr int BP = 32 * RP * WP, BQ = 32 * RQ * WQ, K = 128 / (int)sizeof(T);
    typedef Side<T, W, BP, RP, MP> SideP;
    typedef Side<T, W, BQ, RQ, MQ> SideQ;
    static constexpr int STEP = SideP::BYTES + SideQ::BYTES, BYTES = 2 * STEP;

    floatx16 acc[RP][RQ];
    SideP sp;
    SideQ sq;

    // Waits for this wave's loads and reads, and for the other waves; the compiler moves no memory
    // access past it.
    static __device__ __forceinline__ void arrive() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    // The same for what is in LDS alone.
    static __device__ __forceinline__ void meet() {
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    static __device__ __forceinline__ int wave_of() {
        return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    }
    static __device__ __forceinline__ uint32_t byte_of(const char KAN_LDS* lds) {
        return (uint32_t)(uintptr_t)lds;
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
    __device__ __forceinline__ void products(const u32x4 (&a)[RP], const u32x4 (&b)[RQ]) {
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int j = 0; j < RQ; ++j) multiply(a[i], b[j], acc[i][j]);
    }

    // The loads of the first step of a tile over k from `at` to `end`, to the first STEP bytes of
    // lds (which no wave reads any more), ahead of `run`.
    __device__ __forceinline__ void start(char KAN_LDS* lds, const Operand& p, const Operand& q,
                                          int64_t at, int64_t end) {
        const int lane = threadIdx.x & 63, wave = wave_of();
        sp.place(lane, wave, wave % WP, p.stride);
        sq.place(lane, wave, wave / WP, q.stride);
        sp.issue(p, 0, at, end, wave, byte_of(lds));
        sq.issue(q, 0, at, end, wave, byte_of(lds) + SideP::BYTES);
    }

    // The sum over k from `at` to `end`, after `start` with the same arguments.  lds: BYTES.
    __device__ __forceinline__ void run(char KAN_LDS* lds, const Operand& p, const Operand& q,
                                        int64_t at, int64_t end) {
        const int wave = wave_of();
        const uint32_t base = byte_of(lds);
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int j = 0; j < RQ; ++j) acc[i][j] = floatx16{};
        // the step whose loads are next
        // (the segments of a step's k follow one another: their terms are read from L2 again)
        int64_t k = SEGS > 1 ? at : at + K;
        int seg = SEGS > 1 ? 1 : 0;
        const auto issue = [&](uint32_t dst) {
            if (k >= end) return;
            sp.issue(p, seg, k, end, wave, dst);
            sq.issue(q, seg, k, end, wave, dst + SideP::BYTES);
            if (++seg >= SEGS) seg = 0, k += K;
        };
        issue(base + STEP);
        u32x4 a[2][RP], b[2][RQ];
        const auto fetch = [&](const char KAN_LDS* src, int quarter, int to) {
            sp.fetch(src, quarter, a[to]);
            sq.fetch(src + SideP::BYTES, quarter, b[to]);
        };
        arrive();
        fetch(lds, 0, 0);
        int cur = 0;
        for (int steps = SEGS * (int)((end - at + K - 1) / K); steps > 0; --steps) {
#pragma unroll
            for (int c = 0; c < 3; ++c) {
                fetch(lds + cur, c + 1, (c + 1) & 1);
                products(a[c & 1], b[c & 1]);
                __builtin_amdgcn_sched_barrier(0);
            }
            arrive();
            __builtin_amdgcn_sched_barrier(0);
            issue(base + cur);
            // (after the last step: of what the buffer held before, for nothing)
            fetch(lds + STEP - cur, 0, 0);
            products(a[1], b[1]);
            __builtin_amdgcn_sched_barrier(0);
            cur = STEP - cur;
        }
        arrive();
    }

    // This thread, computed anew after the loop (so that nothing derived from it lives across it).
    static __device__ __forceinline__ int thread() {
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
        return t;
    }

    // The q of a thread's accumulators acc[.][j] and the p of acc[0][.][0], within the tile; that of
    // acc[i][.][e] is 32 i + 8 (e / 4) + e % 4 further on.
    static __device__ __forceinline__ int q_of(int thread, int j) {
        return ((thread >> 6) / WP) * 32 * RQ + j * 32 + (thread & 31);
    }
    static __device__ __forceinline__ int p_of(int thread) {
        return ((thread >> 6) % WP) * 32 * RP + 4 * (thread >> 5 & 1);
    }
    static constexpr int p_step(int i, int e) { return i * 32 + 8 * (e >> 2) + (e & 3); }

    // Values acc[.][j] of all threads as U in LDS: a row per q of j (ROWS in all, q_of_row) of BP
    // values, PITCH bytes apart.
    static constexpr int ROWS = 32 * WQ;
    template <typename U> static constexpr int PITCH = BP * (int)sizeof(U) + 16;
    template <typename U, typename F>
    __device__ __forceinline__ void put(char* lds, int thread, int j, F&& rounded) {
        typedef U four __attribute__((ext_vector_type(4)));
        char* const row = lds + ((thread >> 6) / WP * 32 + (thread & 31)) * PITCH<U> +
                          p_of(thread) * (int)sizeof(U);
#pragma unroll
        for (int i = 0; i < RP; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const floatx16& v = acc[i][j];
                *reinterpret_cast<four*>(row + p_step(i, 4 * g) * (int)sizeof(U)) =
                    four{rounded(v[4 * g]), rounded(v[4 * g + 1]), rounded(v[4 * g + 2]),
                         rounded(v[4 * g + 3])};
            }
    }
    static __device__ __forceinline__ int q_of_row(int row, int j) {
        return (row >> 5) * 32 * RQ + j * 32 + (row & 31);
    }
};

// Tile `id` of tp x tq: neighbouring ids go to different XCDs, each of which takes a run of tiles, in
// blocks of up to eight q-tiles by all p-tiles, so that those that run at a time on an XCD share
// rows of both operands in its L2.
__device__ __forceinline__ void tile_of(int id, int tp, int tq, int* p, int* q) {
    const int all = tp * tq, xcd = id & 7, per = all >> 3, rest = all & 7;
    const int t = xcd * per + (xcd < rest ? xcd : rest) + (id >> 3);
    const int band = t / (8 * tp), first = band * 8, height = tq - first < 8 ? tq - first : 8;
    const int in = t - band * 8 * tp;
    *p = in / height;
    *q = first + in % height;
}

}  // namespace kan
