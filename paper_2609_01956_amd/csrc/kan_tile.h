// kan_tile.h -- a workgroup's tile of out[q][p] = sum_k P(p, k) Q(q, k) on the matrix cores, in bf16
// or fp32 with fp32 accumulation.  Each operand stands in memory by rows (of p or q, k contiguous) or
// by k (rows of k, p or q contiguous), so that no product needs a transposed copy.
//
// A step takes 64 (bf16) or 32 (fp32) values of k of both operands into LDS, straight from memory
// (16 bytes per lane, no registers between), into one of two buffers; a step is 64 KB for a tile of
// 256 x 256.  One barrier a step, before the last quarter of its products, tells that the next
// step has arrived and that all waves have read this one, whose buffer then takes the loads of
// the step after the next.  Fragments are read a quarter ahead of their products, each read (and load)
// between two of them: in front of all, the reads keep the matrix cores waiting (8192 x 8192 x 8192
// 1.31 against 1.35 PFLOP/s).  A wave that waits at the barrier has a lower priority than one that
// goes on (2%).
//
// In LDS:
//   by rows  128 bytes a row, its eight 16-byte chunks at chunk ^ (row >> 1 & 7): sixteen lanes that
//            read one chunk of sixteen rows use all banks (with row & 7 they used half)
//   by k     (bf16) a row per k; fragments come from the LDS's transposing read (four k of 16 columns
//            for 16 lanes), whose four rows stand in different quarters of the banks, 64-byte
//            blocks at block ^ (k & 3)
// What lies past an operand's end is 0 (the buffer's bounds).  By rows, k must be a whole number of
// 16-byte chunks; rows are 16-byte aligned in both, and end with a chunk.  By k, columns past the end
// hold what follows: they reach outputs past the end only.
//
// Each wave holds RP x RQ tiles of 32 x 32: a lane's accumulators are 16 values of p (in fours of
// neighbours) for one q, so that sums over p stay in the lane.
//
// Measured on MI355X, random bf16, 256 x 256 tiles, with the head's sums of exponentials (PFLOP/s;
// of zeros, which take less power; a library's product of the same shape):
//   8192 x 8192 x k = 8192     1.32-1.35 (1.82; 1.61-1.64, of zeros 2.27)
//   8192 x 131072 x k = 2048   1.23-1.25 (1.59; 1.35-1.40, 1.61)
//   8192 x 32768 x k = 1024    1.13-1.17 (1.45; 1.29, 1.65)
// Random operands hold the card at its power limit, zeros show the waits that are left.  Per step the
// LDS gives 192 KB of fragments and takes 64 KB of loads, as many of its clocks as the matrix cores need.
// Tried: a ring of five steps of half the size, four in flight, 2-6% slower; four waves of 128 x 128,
// which read a third less, 7% slower in the products (their one wave a SIMD waits alone), and their
// accumulators leave the logits' sums no registers; the barrier after two or four products of its
// quarter 2 and 3% slower; tiles of 128 x 128, two workgroups a CU, 15%.
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

    // The loads of the step of segment `seg` that begins at k (of `end`; none past it: zeros): what
    // they have in common, and each, to the step at LDS byte dst.
    struct Loads {
        u32x4 rsrc;
        uint32_t at;
        int bytes;  // of the step's k
    };
    __device__ __forceinline__ Loads loads(const Operand& o, int seg, int64_t k, int64_t end) const {
        const char* at = o.at + (MODE == kByRows ? 0 : k * o.stride) +
                         (int64_t)(o.terms >> 4 * seg & 15) * o.plane;
        const int64_t there = end < o.k ? end : o.k;
        const int rows = MODE == kByRows ? (k < end ? o.left : 0) : (int)(there - k < K ? there - k : K);
        // (bounds are kept by 4 bytes: by k, the last row to the end of its last chunk)
        const int64_t width = MODE == kByRows ? end * ES : ((int64_t)o.left * ES + 15) & ~15;
        const uint64_t base = reinterpret_cast<uint64_t>(at);
        Loads l;
        l.rsrc = u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu,
                       rows > 0 ? (uint32_t)((int64_t)(rows - 1) * o.stride + width) : 0u,
                       (uint32_t)kBufferWord3};
        l.at = MODE == kByRows && k < end ? (uint32_t)(k * ES) : 0u;
        l.bytes = (int)(end - k < K ? end - k : K) * ES;
        return l;
    }
    __device__ __forceinline__ void issue(const Loads& l, int i, int wave, uint32_t dst) const {
        uint32_t v = from[i];
        if constexpr (MODE == kByRows) {
            const int c = tail ^ (((wave * LOADS + i) & 1) * 64);
            v = c >= l.bytes ? 0x80000000u : v;
        }
        dma16(l.rsrc, v, l.at, dst + (wave * LOADS + i) * 1024);
    }

    // Fragment i of a quarter of a step at src.
    __device__ __forceinline__ u32x4 fetch(const char KAN_LDS* src, int quarter, int i) const {
        if constexpr (MODE == kByRows) {
            return *(const u32x4 KAN_LDS*)(src + read[0] + chunk[quarter] + i * 32 * 128);
        } else {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            const char KAN_LDS* p = src + read[i] + quarter * 16 * ROW;
            const u32x2 lo = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 KAN_LDS*)p));
            const u32x2 hi = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 KAN_LDS*)(p + 4 * ROW)));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
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
    // The loads of the first step of a tile over k from `at` to `end`, to the first STEP bytes of
    // lds (which no wave reads any more), ahead of `run`.
    __device__ __forceinline__ void start(char KAN_LDS* lds, const Operand& p, const Operand& q,
                                          int64_t at, int64_t end) {
        const int lane = threadIdx.x & 63, wave = wave_of();
        sp.place(lane, wave, wave % WP, p.stride);
        sq.place(lane, wave, wave / WP, q.stride);
        const auto lp = sp.loads(p, 0, at, end);
        const auto lq = sq.loads(q, 0, at, end);
#pragma unroll
        for (int i = 0; i < SideP::LOADS; ++i) sp.issue(lp, i, wave, byte_of(lds));
#pragma unroll
        for (int i = 0; i < SideQ::LOADS; ++i) sq.issue(lq, i, wave, byte_of(lds) + SideP::BYTES);
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
        typename SideP::Loads lp;
        typename SideQ::Loads lq;
        const auto next = [&] {
            lp = sp.loads(p, seg, k, end);
            lq = sq.loads(q, seg, k, end);
            if (++seg >= SEGS) seg = 0, k += K;
        };
        constexpr int LOADS = SideP::LOADS + SideQ::LOADS;
        const auto issue = [&](int i, uint32_t dst) {
            if (i < SideP::LOADS) sp.issue(lp, i, wave, dst);
            else sq.issue(lq, i - SideP::LOADS, wave, dst + SideP::BYTES);
        };
        next();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) issue(i, base + STEP);
        u32x4 a[2][RP], b[2][RQ];
        const auto fetch = [&](const char KAN_LDS* src, int quarter, int to, int i) {
            if (i < RP) a[to][i] = sp.fetch(src, quarter, i);
            else b[to][i - RP] = sq.fetch(src + SideP::BYTES, quarter, i - RP);
        };
        arrive();
#pragma unroll
        for (int i = 0; i < RP + RQ; ++i) fetch(lds, 0, 0, i);
        int cur = 0;
        // (between the matrix instructions, which one after the other keep the matrix cores busy: the
        // reads of the next quarter, and the loads)
        constexpr int PRODUCTS = RP * RQ;
        for (int steps = SEGS * (int)((end - at + K - 1) / K); steps > 0; --steps) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c == 3) {
                    next();
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(0);
                    arrive();
                    __builtin_amdgcn_s_setprio(1);
                }
#pragma unroll
                for (int m = 0; m < PRODUCTS; ++m) {
                    // (after the last step: of what the buffer held before, for nothing)
#pragma unroll
                    for (int i = 0; i < RP + RQ; ++i)
                        if (turn_of(i, RP + RQ, PRODUCTS) == m)
                            fetch(c < 3 ? lds + cur : lds + STEP - cur, (c + 1) & 3, (c + 1) & 1, i);
                    if (c == 3) {
#pragma unroll
                        for (int i = 0; i < LOADS; ++i)
                            if (turn_of(i, LOADS, PRODUCTS) == m) issue(i, base + cur);
                    }
                    multiply(a[c & 1][m / RQ], b[c & 1][m % RQ], acc[m / RQ][m % RQ]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            cur = STEP - cur;
        }
        __builtin_amdgcn_s_setprio(0);
        arrive();
    }

    // Of n reads or loads between products, the product before which number i goes.
    static constexpr int turn_of(int i, int n, int products) {
        return n <= products ? i : i * products / n;
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
