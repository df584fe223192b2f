// kan_embed.hip -- rows of a table for tokens, scaled, and the gradient of the table.
//
//   y_b = scale table[t_b]
//   dtable_v = base_v + scale sum_{b: t_b = v} dy_b
//
// The gradient sorts the tokens (stable, by digits of up to nine bits), so that a row's sum has
// one order whatever runs when: for the same tokens, n and types the same bits.  Up to kRun entries
// are summed in rising order of b.  Tokens that occur more often are summed in chunks of kRun sorted
// entries first, each to a row of fp32 partial sums, which are then added in a fixed order; every
// row of the table is written once, from its own few entries or from its chunks' sums.
//
// All of it is bound by the memory where it is large.  65536 x 1024 bf16 rows of 50001 tokens: 32 us,
// 134 MB written at 4.2 TB/s while the table's rows come from it once and from the caches after.  The
// gradient of 65536 x 4096 bf16 for 131072 tokens, 367 us: 0.54 GB read and the rows that occur written
// in 160 us, the others in 170 (6.3 TB/s), sorting 30.  65536 x 256 fp32 for 50001, 58 us, is bound by
// what its six launches wait for: 25 us sort, 18 sum chunks, 5 + 7 join and write the rest.
#include <algorithm>

#include "kan_head.h"
#include "kan_ops.h"
#include "kan_rows.h"

namespace kan {

namespace {

constexpr int kLoads = 4;  // units in flight per lane

// V elements of a row of T in 16-byte units, in two steps: the loads, which no lane makes under a
// condition (a row's last unit is loaded where it ends with the row), and what they hold as fp32 (0
// past the row's end).
template <typename T, int V>
struct Piece {
    static constexpr int U = kVec<T>, N = V / U;
    u32x4 raw[N];
    __device__ __forceinline__ void issue(const T* row, int c, int n) {
        issue_units<0, true>(row, c, U, n, 0u, raw);
    }
    __device__ __forceinline__ void value(int c, int n, float (&v)[V]) {
        settle_units<0, true, T>(c, U, n, 0u, raw);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float u[U];
            widen(raw[k], u);
#pragma unroll
            for (int i = 0; i < U; ++i) v[k * U + i] = u[i];
        }
    }
};

// Four bf16: 8 bytes, so that a lane's columns fill 16 bytes of an fp32 row.
template <>
struct Piece<uint16_t, 4> {
    typedef uint64_t any __attribute__((aligned(2)));
    uint64_t raw;
    __device__ __forceinline__ void issue(const uint16_t* row, int c, int n) {
        if (n < 4) {
            raw = 0;
            for (int i = 0; i < 3; ++i)
                if (c + i < n) raw |= (uint64_t)row[c + i] << (16 * i);
            return;
        }
        raw = *reinterpret_cast<const any*>(row + min(c, n - 4));
    }
    __device__ __forceinline__ void value(int c, int n, float (&v)[4]) {
        const int past = n < 4 ? 0 : max(c + 4 - n, 0);
        const uint64_t r = raw >> (16 * past);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float((uint32_t)(r >> (16 * i)) << 16);
    }
};

// A workgroup's share of rows x units items: kLoads * 256 neighbours from an item on.
struct Share {
    int64_t row;  // of the first item
    uint32_t at;  // its unit in that row
    __device__ __forceinline__ Share(int64_t first, uint32_t units) {
        row = first / units;
        at = (uint32_t)(first - row * units);
    }
};

template <typename T, typename TP>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, uint32_t units) {
    constexpr int V = kVec<T>;
    const int64_t all = a.rows * units;
    for (int64_t first = (int64_t)blockIdx.x * 256 * kLoads; first < all;
         first += (int64_t)gridDim.x * 256 * kLoads) {
        const Share s(first, units);
        Piece<TP, V> piece[kLoads];
        int64_t row[kLoads], token[kLoads];
        int c[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const uint32_t j = s.at + u * 256 + threadIdx.x, r = j / units;
            row[u] = s.row + r;
            c[u] = (int)(j - r * units) * V;
            token[u] = row[u] < a.rows ? a.tokens[row[u]] : a.ignore;
        }
        // (tokens that are left out, or none, read the first row)
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const bool in = token[u] != a.ignore && token[u] >= 0 && token[u] < a.classes;
            piece[u].issue(static_cast<const TP*>(a.table) + (in ? token[u] * a.tstride : 0), c[u],
                           a.n);
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            if (row[u] >= a.rows) continue;
            float v[V];
            piece[u].value(c[u], a.n, v);
            const bool in = token[u] != a.ignore && token[u] >= 0 && token[u] < a.classes;
            const float none = token[u] == a.ignore ? 0.0f : __builtin_nanf("");
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = in ? v[i] * a.scale : none;
            store_unit<false>(static_cast<T*>(a.y) + row[u] * a.n, c[u], a.n, v);
        }
    }
}

// ------------------------------------------------------------ sorting

constexpr int kSortThreads = 1024, kSortWaves = 16;
// Entries of a workgroup: of one that sorts all in LDS, and of one tile of many.
constexpr int kSortFew = 4096, kSortTile = 2048;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
// Tiles up to which a pass also counts the next one's digits, per tile of its output.
constexpr int kCountTiles = 32;

struct Entry {
    uint32_t key, at;  // token (classes for none), place in the batch
};

__device__ __forceinline__ uint32_t key_of(int64_t token, int64_t ignore, int classes) {
    return token == ignore || token < 0 || token >= classes ? (uint32_t)classes : (uint32_t)token;
}

// Ranks of a tile's entries among those of their digit, in order: wave w holds the N * 64 entries
// from w N 64 on, a batch's lanes neighbours.  count: [kSortWaves][kDigits] in LDS;
// afterwards count[w][d] is the number of entries of digit d in waves before w, and total(d, n)
// has been called by one thread per digit with the tile's count of it.
template <int N, typename F>
__device__ __forceinline__ void rank_digits(uint32_t (*count)[kDigits], const uint32_t (&digit)[N],
                                            const bool (&live)[N], int bits, uint32_t (&rank)[N],
                                            F&& total) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, digits = 1 << bits;
    for (int i = threadIdx.x; i < kSortWaves * digits; i += kSortThreads)
        count[i >> bits][i & (digits - 1)] = 0;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < N; ++b) {
        uint64_t same = __ballot(live[b]);
        for (int k = 0; k < bits; ++k) {
            const uint64_t one = __ballot(digit[b] >> k & 1);
            same &= digit[b] >> k & 1 ? one : ~one;
        }
        const int before = __popcll(same & ((UINT64_C(1) << lane) - 1));
        if (live[b]) {
            const uint32_t seen = count[wave][digit[b]];
            rank[b] = seen + before;
            // (the lanes of a wave run together: all read before one of them writes)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (before == 0) count[wave][digit[b]] = seen + __popcll(same);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
        uint32_t sum = 0;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = count[w][d];
            count[w][d] = sum;
            sum += c;
        }
        total(d, sum);
    }
    __syncthreads();
}

// first[d] = sum of count[0 .. d), over kDigits values of a workgroup; count is left as it was.
__device__ __forceinline__ void digits_before(const uint32_t* count, uint32_t* first, int digits) {
    __shared__ uint32_t waves[kSortWaves];
    const int d = threadIdx.x, lane = d & 63;
    const uint32_t own = d < digits ? count[d] : 0;
    uint32_t sum = own;
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t v = __shfl_up(sum, o);
        if (lane >= o) sum += v;
    }
    if (lane == 63) waves[d >> 6] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < (d >> 6); ++w) before += waves[w];
    if (d < digits) first[d] = before + sum - own;
    __syncthreads();
}

// The first rows of the table, as they are where their tokens do not occur (base, or 0): written by
// workgroups beside those that sort, which leave most of the GPU and its memory idle.  In 16-byte
// units of memory, whatever the rows are.
struct Fill {
    const char* base;  // or null: 0
    char* to;
    int64_t bytes;        // of the table
    int64_t first, last;  // units: the one that holds the first byte is 0
    int groups;           // workgroups, the last ones of the launch
};
constexpr int kFillTurn = kLoads * kSortThreads;
__device__ __forceinline__ void fill_units(const Fill& f, int group) {
    const int head = (int)(reinterpret_cast<uintptr_t>(f.to) & 15);
    for (int64_t first = f.first + (int64_t)group * kFillTurn; first < f.last;
         first += (int64_t)f.groups * kFillTurn) {
        int64_t at[kLoads];
        bool whole[kLoads];
        u32x4 v[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int64_t u = first + k * kSortThreads + threadIdx.x;
            at[k] = u < f.last ? u * 16 - head : f.bytes;
            whole[k] = at[k] >= 0 && at[k] + 16 <= f.bytes;
            v[k] = u32x4{0, 0, 0, 0};
            if (f.base != nullptr && whole[k])
                v[k] = *unit_at(reinterpret_cast<const uint16_t*>(f.base + at[k]), 0);
        }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            if (whole[k]) {
                *reinterpret_cast<u32x4*>(f.to + at[k]) = v[k];
                continue;
            }
            for (int64_t b = at[k] < 0 ? 0 : at[k]; b < at[k] + 16 && b < f.bytes; b += 2)
                *reinterpret_cast<uint16_t*>(f.to + b) =
                    f.base == nullptr ? (uint16_t)0
                                      : *reinterpret_cast<const uint16_t*>(f.base + b);
        }
    }
}

struct SortArgs {
    const int64_t* tokens;  // the first pass's input, or null:
    const Entry* in;
    Entry* out;
    int64_t rows, ignore;
    int classes, shift, bits;
    uint32_t* hist;    // [tiles][kDigits] counts; after the scan, which is made if totals
    uint32_t* totals;  // ([kDigits], of all tiles) is not null: those of the tiles before
    uint32_t* next;    // the next pass's hist, to be added to, or null
    int next_bits;
    int tiles;
    int2* span;        // [classes + 1], to be cleared, and the later passes' hists
    int64_t later;     // (from `next` on)
    Fill fill;
};

__device__ __forceinline__ Entry entry_of(const SortArgs& a, int64_t i) {
    if (a.tokens == nullptr) return a.in[i];
    return Entry{key_of(a.tokens[i], a.ignore, a.classes), (uint32_t)i};
}

__device__ __forceinline__ void clear_spans(int2* span, int64_t n, int64_t first, int64_t step) {
    for (int64_t i = first; i < n; i += step) span[i] = int2{0, 0};
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(SortArgs a) {
    __shared__ uint32_t count[kDigits];
    if (a.span != nullptr)
        clear_spans(a.span, (int64_t)a.classes + 1, (int64_t)blockIdx.x * kSortThreads + threadIdx.x,
                    (int64_t)gridDim.x * kSortThreads);
    if (a.next != nullptr)
        for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < a.later;
             i += (int64_t)gridDim.x * kSortThreads)
            a.next[i] = 0;
    if ((int)blockIdx.x >= a.tiles) return;
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) count[d] = 0;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kSortTile / kSortThreads; ++b) {
        const int64_t i = (int64_t)blockIdx.x * kSortTile + b * kSortThreads + threadIdx.x;
        if (i < a.rows) atomicAdd(&count[entry_of(a, i).key >> a.shift & ((1 << a.bits) - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads)
        a.hist[(int64_t)blockIdx.x * kDigits + d] = count[d];
}

// Counts of the tiles before each, per digit, and of all.
__global__ void __launch_bounds__(64) sort_scan_kernel(SortArgs a) {
    const int d = blockIdx.x * 64 + threadIdx.x;
    uint32_t sum = 0;
    int t = 0;
    for (; t + 8 <= a.tiles; t += 8) {
        uint32_t c[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = a.hist[(int64_t)(t + k) * kDigits + d];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            a.hist[(int64_t)(t + k) * kDigits + d] = sum;
            sum += c[k];
        }
    }
    for (; t < a.tiles; ++t) {
        const uint32_t c = a.hist[(int64_t)t * kDigits + d];
        a.hist[(int64_t)t * kDigits + d] = sum;
        sum += c;
    }
    a.totals[d] = sum;
}

__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(SortArgs a) {
    __shared__ uint32_t count[kSortWaves][kDigits];
    __shared__ uint32_t all[kDigits], first[kDigits];
    __shared__ uint32_t next[kCountTiles * kDigits];
    constexpr int kBatches = kSortTile / kSortThreads;
    if ((int)blockIdx.x >= a.tiles) {
        fill_units(a.fill, blockIdx.x - a.tiles);
        return;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, digits = 1 << a.bits;
    if (a.next != nullptr)
        for (int i = threadIdx.x; i < a.tiles << a.next_bits; i += kSortThreads) next[i] = 0;
    Entry e[kBatches];
    uint32_t digit[kBatches], rank[kBatches];
    bool live[kBatches];
#pragma unroll
    for (int b = 0; b < kBatches; ++b) {
        const int64_t i = (int64_t)blockIdx.x * kSortTile + (wave * kBatches + b) * 64 + lane;
        live[b] = i < a.rows;
        e[b] = live[b] ? entry_of(a, i) : Entry{0, 0};
        digit[b] = e[b].key >> a.shift & (digits - 1);
    }
    uint32_t before = 0;  // entries of digit threadIdx.x in tiles before
    const int d = threadIdx.x;
    if (d < digits) {
        uint32_t sum = 0;
        if (a.totals != nullptr) {
            before = a.hist[(int64_t)blockIdx.x * kDigits + d];
            sum = a.totals[d];
        } else {
            for (int t0 = 0; t0 < a.tiles; t0 += 8) {
                uint32_t c[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    c[k] = t0 + k < a.tiles ? a.hist[(t0 + k) * kDigits + d] : 0u;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (t0 + k < (int)blockIdx.x) before += c[k];
                    sum += c[k];
                }
            }
        }
        all[d] = sum;
    }
    __syncthreads();
    digits_before(all, first, digits);
    if (d < digits) first[d] += before;
    rank_digits(count, digit, live, a.bits, rank, [](int, uint32_t) {});
#pragma unroll
    for (int b = 0; b < kBatches; ++b)
        if (live[b]) {
            const uint32_t to = first[digit[b]] + count[wave][digit[b]] + rank[b];
            a.out[to] = e[b];
            if (a.next != nullptr)
                atomicAdd(&next[(to / kSortTile << a.next_bits) +
                                (e[b].key >> (a.shift + a.bits) & ((1u << a.next_bits) - 1))],
                          1u);
        }
    if (a.next == nullptr) return;
    __syncthreads();
    // (sums of whole numbers: the same in any order)
    for (int i = threadIdx.x; i < a.tiles << a.next_bits; i += kSortThreads)
        if (next[i] != 0)
            atomicAdd(&a.next[(i >> a.next_bits) * kDigits + (i & ((1 << a.next_bits) - 1))],
                      next[i]);
}

// At most kSortFew entries: all passes in LDS by the first workgroup; others clear the spans.
__global__ void __launch_bounds__(kSortThreads) sort_few_kernel(SortArgs a, int passes) {
    __shared__ uint32_t count[kSortWaves][kDigits];
    __shared__ uint32_t all[kDigits], first[kDigits];
    __shared__ Entry hold[kSortFew];
    constexpr int kBatches = kSortFew / kSortThreads;
    const int groups = (int)gridDim.x - a.fill.groups;
    if ((int)blockIdx.x >= groups) {
        fill_units(a.fill, blockIdx.x - groups);
        return;
    }
    if (blockIdx.x > 0 || groups == 1)
        clear_spans(a.span, (int64_t)a.classes + 1,
                    (int64_t)(groups == 1 ? 0 : blockIdx.x - 1) * kSortThreads + threadIdx.x,
                    (int64_t)(groups == 1 ? 1 : groups - 1) * kSortThreads);
    if (blockIdx.x > 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Entry e[kBatches];
    uint32_t digit[kBatches], rank[kBatches];
    bool live[kBatches];
#pragma unroll
    for (int b = 0; b < kBatches; ++b) {
        const int i = (wave * kBatches + b) * 64 + lane;
        live[b] = i < a.rows;
        e[b] = live[b] ? entry_of(a, i) : Entry{0, 0};
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * a.bits, digits = 1 << a.bits;
#pragma unroll
        for (int b = 0; b < kBatches; ++b) digit[b] = e[b].key >> shift & (digits - 1);
        rank_digits(count, digit, live, a.bits, rank, [&](int d, uint32_t n) { all[d] = n; });
        digits_before(all, first, digits);
#pragma unroll
        for (int b = 0; b < kBatches; ++b)
            if (live[b]) hold[first[digit[b]] + count[wave][digit[b]] + rank[b]] = e[b];
        __syncthreads();
#pragma unroll
        for (int b = 0; b < kBatches; ++b)
            if (live[b]) e[b] = hold[(wave * kBatches + b) * 64 + lane];
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < kBatches; ++b)
        if (live[b]) a.out[(wave * kBatches + b) * 64 + lane] = e[b];
}

// ------------------------------------------------------------ sums

// The sorted entries are taken in chunks of kRun.  A token with at most kRun entries is summed, and its
// row written, by the chunk that it starts in; of one with more, each chunk leaves the sum of its part.
// With more than kRun kFan entries those sums are summed in groups of kFan next, and so on (level l:
// chunk_size(l) entries), so that whatever its share of the batch, a row is the sum of at most
// kRun entries or of about kFan sums.
constexpr int kRun = 16, kFan = 64, kLevels = 5;
__host__ __device__ constexpr int64_t chunk_size(int level) {
    int64_t n = kRun;
    for (int l = 0; l < level; ++l) n *= kFan;
    return n;
}

struct EmbedSumArgs {
    EmbedGradArgs g;
    const Entry* sorted;
    int2* span;            // [classes + 1] a token's entries: from, to
    float* part[kLevels];  // [2 chunks of the level][pitch] sums of a token's entries in a chunk: of
                           // one that starts in an earlier chunk or at its first entry, and of
                           // one that starts later (each with more entries than a chunk)
    int levels;            // that there are
    uint32_t pitch;        // floats of a sum
    uint32_t units;        // of 16 bytes of the table, a row
    int lanes;             // of a chunk: 64, 128 or 256
    int blocks;            // of 64 units, a row
    int heavy;             // the last launch: workgroups for tokens of more than kRun entries
    int64_t filled;        // 16-byte units of the table that have been filled
};

// The sums of a level's chunks c0 .. c1 of the token that starts at entry `start`, added in order.
template <int V>
__device__ __forceinline__ void add_parts(const EmbedSumArgs& a, int level, int c0, int c1,
                                          int start, uint32_t u, float (&s)[V]) {
    constexpr int U = 64 / V;  // (of 16 bytes, 16 loads)
    const int64_t size = chunk_size(level);
    for (int c = c0; c <= c1; c += U) {
        floatx4 p[U][V / 4];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int at = min(c + k, c1);
            const int64_t slot = 2 * (int64_t)at + (start > at * size ? 1 : 0);
#pragma unroll
            for (int i = 0; i < V / 4; ++i)
                p[k][i] = *reinterpret_cast<const floatx4*>(a.part[level] +
                                                            slot * a.pitch + u * V + 4 * i);
        }
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (c + k <= c1) {
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] += p[k][i / 4][i % 4];
            }
    }
}

template <int V>
__device__ __forceinline__ void store_part(const EmbedSumArgs& a, int level, int64_t slot, uint32_t u,
                                           const float (&s)[V]) {
    float* const out = a.part[level] + slot * a.pitch + u * V;
#pragma unroll
    for (int i = 0; i < V; i += 4)
        *reinterpret_cast<floatx4*>(out + i) = floatx4{s[i], s[i + 1], s[i + 2], s[i + 3]};
}

// A lane's V columns of a row.  FULL (rows of V columns at least, of which two lanes may write the
// same): the last lane's end with the row, so that no lane has a part of them; else Piece's.
template <typename T, int V, bool FULL>
struct Columns {
    Piece<T, V> piece;
    __device__ __forceinline__ void issue(const T* row, int c, int n) {
        if constexpr (!FULL) piece.issue(row, c, n);
        else if constexpr (V * sizeof(T) == 8)
            piece.raw = *reinterpret_cast<const typename Piece<T, V>::any*>(row + c);
        else
#pragma unroll
            for (int k = 0; k < Piece<T, V>::N; ++k)
                piece.raw[k] = *unit_at(row, c + k * kVec<T>);
    }
    __device__ __forceinline__ void value(int c, int n, float (&v)[V]) {
        piece.value(c, FULL ? c + V : n, v);
    }
    __device__ __forceinline__ void add(int c, int n, float (&s)[V]) {
        float v[V];
        value(c, n, v);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] += v[i];
    }
};
template <int V, bool FULL>
__device__ __forceinline__ int column_of(uint32_t unit, int n) {
    return FULL ? min((int)unit * V, n - V) : (int)unit * V;
}

// A row of the table: base + scale s.
template <bool FULL, bool PAST, typename TP, int V>
__device__ __forceinline__ void store_sum(const EmbedGradArgs& g, int64_t row, int c,
                                          const float (&s)[V], const float (&base)[V]) {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = __builtin_fmaf(s[i], g.scale, base[i]);
    store_unit<FULL, PAST>(static_cast<TP*>(g.dtable) + row * g.n, c, g.n, v);
}

// Spans, rows of few entries, and the first level's sums: a.lanes neighbouring lanes per chunk.
// What belongs to which row is uniform over them, so the loads of kRun entries are in flight at a
// time, under no condition.
template <typename T, typename TP, bool FULL, bool BASE>
__global__ void __launch_bounds__(256) embed_chunk_kernel(EmbedSumArgs a) {
    constexpr int V = kVec<TP>;
    const int64_t rows = a.g.rows, chunks = (rows + kRun - 1) / kRun;
    const int per = 256 / a.lanes, lane = threadIdx.x & 63, n = a.g.n;
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / a.lanes);
    for (int64_t chunk = (int64_t)blockIdx.x * per + team; chunk < chunks;
         chunk += (int64_t)gridDim.x * per) {
        const int64_t first = chunk * kRun;
        // lanes 0 .. 47: the entries of the chunk before, of the chunk, and of the next
        const int64_t mine = first + lane - kRun;
        const bool there = lane < 3 * kRun && mine >= 0 && mine < rows;
        const Entry e = there ? a.sorted[mine] : Entry{0xffffffffu, 0};
        const uint32_t left = __shfl_up(e.key, 1), right = __shfl_down(e.key, 1);
        if ((int)threadIdx.x % a.lanes < 64 && there && lane >= kRun && lane < 2 * kRun) {
            if (left != e.key) a.span[e.key].x = (int)mine;
            if (right != e.key) a.span[e.key].y = (int)mine + 1;
        }
        // bits of lanes: the first entry of a run of one token (48: what is past the window);
        // entries of tokens
        const uint64_t window = (UINT64_C(1) << 3 * kRun) - 1;
        const uint64_t starts = (__ballot(lane > 0 && left != e.key) & window) | ~window;
        const uint64_t tokens = __ballot(e.key < (uint32_t)a.g.classes);
        const auto start_after = [&](int l) { return __builtin_ctzll(starts >> l >> 1) + l + 1; };
        // the run at the chunk's first entry, if it started before; one of few entries is no business
        // of this chunk
        const uint32_t head = __builtin_amdgcn_readlane((int)e.key, kRun);
        const bool goes_on = !(starts >> kRun & 1), many = __popcll(__ballot(e.key == head)) > kRun;
        const int begin = goes_on && !many ? start_after(kRun) : kRun;
        if (begin >= 2 * kRun || !(tokens >> begin & 1)) continue;
        // the run that reaches past the chunk: its rest, if it is of few entries and starts here
        const int next = start_after(2 * kRun - 1);
        const int tail = 63 - __builtin_clzll((starts & ((UINT64_C(1) << 2 * kRun) - 1)) | 1);
        const int end = tail >= begin && next - tail <= kRun ? next : 2 * kRun;
        // entries to add, and those after which a sum is whole (or the chunk's share of it)
        const uint64_t live = tokens & ((UINT64_C(1) << end) - 1) & ~((UINT64_C(1) << begin) - 1);
        const uint64_t ends = live & (starts >> 1 | UINT64_C(1) << (end - 1));
        for (uint32_t u = threadIdx.x & (a.lanes - 1); u < a.units; u += a.lanes) {
            const int c = column_of<V, FULL>(u, n);
            float s[V] = {};
#pragma unroll 1
            for (int l0 = kRun; l0 < end; l0 += kRun) {
                Columns<T, V, FULL> v[kRun];
                Columns<TP, V, FULL> base[BASE ? kRun : 1];
#pragma unroll
                for (int i = 0; i < kRun; ++i) {
                    const int l = live >> (l0 + i) & 1 ? l0 + i : begin;
                    const uint32_t at = __builtin_amdgcn_readlane((int)e.at, l);
                    v[i].issue(static_cast<const T*>(a.g.dy) + at * a.g.dystride, c, n);
                    if constexpr (BASE) {
                        const uint32_t key = __builtin_amdgcn_readlane((int)e.key, l);
                        if (ends >> (l0 + i) & 1)
                            base[i].issue(static_cast<const TP*>(a.g.base) + (int64_t)key * n, c, n);
                    }
                }
#pragma unroll
                for (int i = 0; i < kRun; ++i) {
                    const int l = l0 + i;
                    if (!(live >> l & 1)) continue;
                    if (starts >> l & 1) {
#pragma unroll
                        for (int k = 0; k < V; ++k) s[k] = 0.0f;
                    }
                    v[i].add(c, n, s);
                    if (!(ends >> l & 1)) continue;
                    const uint32_t key = __builtin_amdgcn_readlane((int)e.key, l);
                    const uint64_t upto = starts & ((UINT64_C(2) << l) - 1);
                    const int from = upto >> kRun ? 63 - __builtin_clzll(upto) : -1;
                    if (from >= 0 && start_after(from) - from <= kRun) {
                        float w[V] = {};
                        if constexpr (BASE) base[i].value(c, n, w);
                        store_sum<FULL, false, TP>(a.g, key, c, s, w);
                    } else {
                        store_part(a, 0, 2 * chunk + (from > kRun ? 1 : 0), u, s);
                    }
                }
            }
        }
    }
}

// The sums of a later level's chunks from those of the level before, a workgroup for each 64 units: of
// either token (the one at the chunk's first entry, the one at its last) in four waves, a quarter of
// the sums in each.  (All in one wave: 8.4 us, so 4.9, for 64 chunks of 256 fp32; 17.9 and 8.6 for 64
// of 4096 bf16.)
constexpr int kJoinWaves = 4;  // of a token
template <int V>
__global__ void __launch_bounds__(128 * kJoinWaves) embed_join_kernel(EmbedSumArgs a, int level) {
    __shared__ float sums[2][kJoinWaves - 1][V][64];
    const int64_t rows = a.g.rows, size = chunk_size(level), fine = chunk_size(level - 1);
    const int64_t items = (rows + size - 1) / size * a.blocks;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slot = wave / kJoinWaves, share = wave % kJoinWaves;
    // short rows leave lanes over: each strand of them takes a part of the sums
    int width = 64;
    while (width >= 2 * (int)a.units) width /= 2;
    const int strands = 64 / width;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t chunk = item / a.blocks;
        const uint32_t u = (uint32_t)(item - chunk * a.blocks) * 64 + (lane & (width - 1));
        const int64_t first = chunk * size, end = first + size < rows ? first + size : rows;
        const uint32_t head = a.sorted[first].key, last = a.sorted[end - 1].key;
        const uint32_t k = slot == 0 ? head : last;
        bool live = k < (uint32_t)a.g.classes && !(slot == 1 && k == head);
        float s[V] = {};
        if (live) {
            const int2 span = a.span[k];
            live = span.y - span.x > size;
            if (live) {
                const int64_t from = span.x > first ? span.x : first, to = span.y < end ? span.y : end;
                const int c0 = (int)(from / fine), c1 = (int)((to - 1) / fine);
                const int all = (c1 - c0 + kJoinWaves) / kJoinWaves, q0 = c0 + share * all;
                const int q1 = min(q0 + all - 1, c1);
                const int each = (q1 - q0 + strands) / strands, mine = q0 + lane / width * each;
                if (u < a.units)
                    add_parts(a, level - 1, mine, min(mine + each - 1, q1), span.x, u, s);
                for (int o = width; o < 64; o *= 2)
#pragma unroll
                    for (int i = 0; i < V; ++i) s[i] += __shfl_xor(s[i], o);
            }
        }
        __syncthreads();  // (the sums of the item before are read)
        if (share > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) sums[slot][share - 1][i][lane] = s[i];
        }
        __syncthreads();
        if (share > 0 || !live || u >= a.units || lane >= width) continue;
#pragma unroll
        for (int q = 0; q < kJoinWaves - 1; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += sums[slot][q][i][lane];
        store_part(a, level, 2 * chunk + slot, u, s);
    }
}

// Rows of tokens with more than kRun entries (the first a.heavy workgroups, a wave for 64 units of the
// one that starts in a chunk), and of those that do not occur (the others).  PAST: stored past the caches.
template <typename TP, bool FULL, bool PAST>
__global__ void __launch_bounds__(256) embed_rest_kernel(EmbedSumArgs a) {
    constexpr int V = kVec<TP>;
    if ((int)blockIdx.x < a.heavy) {
        const int64_t rows = a.g.rows, items = (rows + kRun - 1) / kRun * a.blocks;
        for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items;
             item += (int64_t)a.heavy * 4) {
            const int64_t chunk = item / a.blocks;
            const uint32_t u = (uint32_t)(item - chunk * a.blocks) * 64 + (threadIdx.x & 63);
            // (with more than kRun entries it is the chunk's last one)
            const int64_t first = chunk * kRun, last = min(first + kRun, rows) - 1;
            const uint32_t key = a.sorted[last].key;
            if (key >= (uint32_t)a.g.classes) continue;
            const int2 span = a.span[key];
            const int count = span.y - span.x;
            if (count <= kRun || span.x < first) continue;
            int level = 0;
            while (level + 1 < a.levels && count > chunk_size(level + 1)) ++level;
            const int64_t size = chunk_size(level);
            if (u >= a.units) continue;
            const int c = column_of<V, FULL>(u, a.g.n);
            float s[V] = {}, w[V] = {};
            Columns<TP, V, FULL> base;
            if (a.g.base != nullptr)
                base.issue(static_cast<const TP*>(a.g.base) + (int64_t)key * a.g.n, c, a.g.n);
            add_parts(a, level, (int)(span.x / size), (int)((span.y - 1) / size), span.x, u, s);
            if (a.g.base != nullptr) base.value(c, a.g.n, w);
            store_sum<FULL, false, TP>(a.g, key, c, s, w);
        }
        return;
    }
    // the table as one run of aligned 16-byte units, whatever its rows are: stores of odd rows at their
    // own places take twice as long (109776 x 1153 fp32 in all 147 us, so 105)
    TP* const table = static_cast<TP*>(a.g.dtable);
    const int64_t total = (int64_t)a.g.classes * a.g.n;
    const int head = (int)((reinterpret_cast<uintptr_t>(table) & 15) / sizeof(TP));
    const int64_t units = (total + head + V - 1) / V, groups = gridDim.x - a.heavy;
    for (int64_t first = a.filled + (int64_t)(blockIdx.x - a.heavy) * 256 * kLoads; first < units;
         first += groups * 256 * kLoads) {
        // rows of the workgroup's elements, from that of the first one on
        const int64_t e0 = first * V - head, origin = e0 < 0 ? 0 : e0;
        const int64_t row0 = origin / a.g.n;
        const uint32_t at0 = (uint32_t)(origin - row0 * a.g.n);
        int64_t e[kLoads], row[kLoads];
        int from[kLoads], to[kLoads], turn[kLoads];  // a unit's elements, and the next row's first
        int2 one[kLoads], two[kLoads];               // spans of the first row and of the next
        uint32_t absent[kLoads];                     // bits: elements of rows that do not occur
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            e[u] = e0 + (int64_t)(u * 256 + (int)threadIdx.x) * V;
            from[u] = e[u] < 0 ? (int)-e[u] : 0;
            to[u] = (int)(total - e[u] < V ? total - e[u] : V);
            const uint32_t j = at0 + (uint32_t)(e[u] + from[u] - origin), r = j / (uint32_t)a.g.n;
            row[u] = row0 + r;
            turn[u] = (int)min((uint32_t)from[u] + a.g.n - (j - r * a.g.n), (uint32_t)V);
            one[u] = to[u] > from[u] ? a.span[row[u]] : int2{0, 1};
            two[u] = to[u] > turn[u] ? a.span[row[u] + 1] : int2{0, 1};
        }
        const auto bits = [](int lo, int hi) { return hi > lo ? (1u << hi) - (1u << lo) : 0u; };
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            absent[u] = (one[u].x == one[u].y ? bits(from[u], min(turn[u], to[u])) : 0u) |
                        (two[u].x == two[u].y ? bits(turn[u], min(turn[u] + a.g.n, to[u])) : 0u);
            // (rows shorter than a unit)
            for (int at = turn[u] + a.g.n, k = 2; at < to[u]; at += a.g.n, ++k) {
                const int2 span = a.span[row[u] + k];
                if (span.x == span.y) absent[u] |= bits(at, min(at + a.g.n, to[u]));
            }
        }
        constexpr uint32_t FULL_UNIT = (1u << V) - 1;
        u32x4 base[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            base[u] = u32x4{0, 0, 0, 0};
            if (a.g.base != nullptr && absent[u] == FULL_UNIT)
                base[u] = *unit_at(static_cast<const TP*>(a.g.base) + e[u], 0);
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            if (absent[u] == FULL_UNIT) {
                u32x4* const to = reinterpret_cast<u32x4*>(table + e[u]);
                if (PAST) __builtin_nontemporal_store(base[u], to);
                else *to = base[u];
            } else if (absent[u] != 0) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (absent[u] >> i & 1)
                        table[e[u] + i] =
                            a.g.base == nullptr ? TP(0) : static_cast<const TP*>(a.g.base)[e[u] + i];
            }
        }
    }
}

// ------------------------------------------------------------ plans

int64_t div_up(int64_t v, int64_t by) { return (v + by - 1) / by; }
int groups_of(int64_t n) { return (int)std::min<int64_t>(n, kMaxGroups); }

// Workgroups of each kind in the last launch: they go on by strides.
constexpr int kRestGroups = 1 << 13;
constexpr int kJoinGroups = 1 << 16;
// Bytes (read and written) of the table that a pass of sorting may fill beside it, what one launch
// sorts taking about two passes' time; workgroups of such a launch.  4096 x 1024 bf16 of 131072 tokens:
// without 71 us, 32 MB 67, 64 MB 61, 96 MB 55; 65536 x 256 fp32 of 50001 62, 59, 59, 59; with a base,
// 30001 x 1001 of 50001, 122, 120, 124, 127.
constexpr int64_t kFillBytes = INT64_C(48) << 20;
constexpr int kFillGroups = 256;

struct EmbedGradPlan {
    Entry* list[2];
    uint32_t *hist, *totals;
    int2* span;
    float* part[kLevels];
    int levels, tiles, passes;
    int bits;   // of a pass
    int hists;  // passes' counts side by side, or 1: one for all
    size_t bytes;
};

EmbedGradPlan embed_grad_plan(int64_t rows, int32_t classes, int32_t n, void* ws) {
    EmbedGradPlan p = {};
    char* const base = static_cast<char*>(ws);
    const auto take = [&](int64_t bytes) {
        char* const at = base == nullptr ? nullptr : base + p.bytes;
        p.bytes += (size_t)(div_up(bytes, 256) * 256);
        return at;
    };
    int bits = 0;
    while (classes >> bits) ++bits;  // (of the keys 0 .. classes)
    p.passes = (int)div_up(bits, kDigitBits);
    p.bits = (int)div_up(bits, p.passes);
    p.tiles = (int)div_up(rows, kSortTile);
    const bool few = rows <= kSortFew;
    p.hists = p.tiles <= kCountTiles ? p.passes : 1;
    p.span = reinterpret_cast<int2*>(take(((int64_t)classes + 1) * 8));
    for (int i = 0; i < (few ? 1 : 2); ++i)
        p.list[i] = reinterpret_cast<Entry*>(take(rows * (int64_t)sizeof(Entry)));
    if (!few) {
        p.hist = reinterpret_cast<uint32_t*>(take((int64_t)p.hists * p.tiles * kDigits * 4));
        p.totals = reinterpret_cast<uint32_t*>(take(kDigits * 4));
    }
    for (; p.levels < kLevels && rows > chunk_size(p.levels); ++p.levels)
        p.part[p.levels] = reinterpret_cast<float*>(
            take(2 * div_up(rows, chunk_size(p.levels)) * (div_up(n, 8) * 8) * 4));
    return p;
}

#define KAN_TRY(...)                          \
    do {                                      \
        const hipError_t e_ = (__VA_ARGS__);  \
        if (e_ != hipSuccess) return e_;      \
    } while (0)

template <typename T, typename TP>
hipError_t embed(const EmbedArgs& a, hipStream_t s) {
    const uint32_t units = (uint32_t)div_up(a.n, kVec<T>);
    embed_kernel<T, TP><<<groups_of(div_up(a.rows * units, 256 * kLoads)), 256, 0, s>>>(a, units);
    return hipGetLastError();
}

template <typename T, typename TP>
hipError_t embed_grad(const EmbedGradArgs& g, void* ws, hipStream_t s) {
    const EmbedGradPlan p = embed_grad_plan(g.rows, g.classes, g.n, ws);
    SortArgs a = {};
    a.tokens = g.tokens;
    a.out = p.list[0];
    a.rows = g.rows;
    a.ignore = g.ignore;
    a.classes = g.classes;
    a.bits = a.next_bits = p.bits;
    a.tiles = p.tiles;
    a.span = p.span;
    // (in place, rows of tokens that do not occur stay as they are)
    const int64_t bytes = (int64_t)g.classes * g.n * (int64_t)sizeof(TP);
    const int64_t units =
        g.base == g.dtable ? 0 : div_up(bytes + (reinterpret_cast<uintptr_t>(g.dtable) & 15), 16);
    a.fill = Fill{static_cast<const char*>(g.base), static_cast<char*>(g.dtable), bytes, 0, 0, 0};
    const auto fill_next = [&](int sorting, int passes) {
        a.fill.first = a.fill.last;
        a.fill.last =
            std::min(units, a.fill.first + passes * kFillBytes / (g.base == nullptr ? 16 : 32));
        a.fill.groups = (int)std::min<int64_t>(div_up(a.fill.last - a.fill.first, kFillTurn),
                                               kFillGroups - sorting);
    };
    const int clear = (int)std::min<int64_t>(div_up((int64_t)g.classes + 1, 4 * kSortThreads), 1024);
    if (g.rows <= kSortFew) {
        const int groups = clear == 1 ? 1 : clear + 1;
        fill_next(1, 2);
        sort_few_kernel<<<groups + a.fill.groups, kSortThreads, 0, s>>>(a, p.passes);
        KAN_TRY(hipGetLastError());
    } else {
        const int64_t hist = (int64_t)p.tiles * kDigits;
        a.later = (p.hists - 1) * hist;
        for (int i = 0; i < p.passes; ++i) {
            a.out = p.list[i & 1];
            a.hist = p.hist + (p.hists > 1 ? i * hist : 0);
            a.next = p.hists > 1 && i + 1 < p.passes ? a.hist + hist : nullptr;
            if (i == 0 || p.hists == 1) {
                const int groups = i == 0 ? std::max(clear, p.tiles) : p.tiles;
                sort_count_kernel<<<groups, kSortThreads, 0, s>>>(a);
                KAN_TRY(hipGetLastError());
            }
            if (p.tiles > kCountTiles) {
                a.totals = p.totals;
                sort_scan_kernel<<<kDigits / 64, 64, 0, s>>>(a);
                KAN_TRY(hipGetLastError());
            }
            // (beside the sort of more tiles it has not been tried: the last launch writes those rows)
            if (p.tiles <= kCountTiles) fill_next(p.tiles, 1);
            sort_scatter_kernel<<<p.tiles + a.fill.groups, kSortThreads, 0, s>>>(a);
            KAN_TRY(hipGetLastError());
            a.tokens = nullptr;
            a.span = nullptr;
            a.in = a.out;
            a.shift += p.bits;
        }
    }
    EmbedSumArgs e = {};
    e.g = g;
    e.sorted = a.out;
    e.span = p.span;
    e.levels = p.levels;
    e.pitch = (uint32_t)(div_up(g.n, 8) * 8);
    e.units = (uint32_t)div_up(g.n, kVec<TP>);
    e.lanes = 64;
    e.blocks = (int)div_up(e.units, 64);
    for (int l = 0; l < p.levels; ++l) e.part[l] = p.part[l];
    while (e.lanes < 256 && (uint32_t)e.lanes < e.units) e.lanes *= 2;
    const int per = 256 / e.lanes;
    // (in place no column may have two writers)
    const bool whole = g.n % kVec<TP> == 0;
    const bool full = g.n >= kVec<TP> && (whole || g.base != g.dtable);
    if (g.rows > 0) {
        const int groups = groups_of(div_up(div_up(g.rows, kRun), per));
        const auto chunks = g.base != nullptr
                                ? full ? embed_chunk_kernel<T, TP, true, true>
                                       : embed_chunk_kernel<T, TP, false, true>
                                : full ? embed_chunk_kernel<T, TP, true, false>
                                       : embed_chunk_kernel<T, TP, false, false>;
        chunks<<<groups, 256, 0, s>>>(e);
        KAN_TRY(hipGetLastError());
    }
    for (int l = 1; l < p.levels; ++l) {
        embed_join_kernel<kVec<TP>>
            <<<(int)std::min<int64_t>(div_up(g.rows, chunk_size(l)) * e.blocks, kJoinGroups),
               128 * kJoinWaves, 0, s>>>(e, l);
        KAN_TRY(hipGetLastError());
    }
    if (g.rows > kRun)
        e.heavy = (int)std::min<int64_t>(div_up(div_up(g.rows, kRun) * e.blocks, 4), kRestGroups);
    e.filled = a.fill.last;
    const int64_t rest = div_up(units - e.filled, 256 * kLoads);
    const int groups = e.heavy + (int)std::min<int64_t>(rest, kRestGroups);
    if (groups == 0) return hipSuccess;
    const bool past = (int64_t)g.classes * g.n * (int64_t)sizeof(TP) >= kPastCaches;
    const auto others = past ? full ? embed_rest_kernel<TP, true, true>
                                    : embed_rest_kernel<TP, false, true>
                             : full ? embed_rest_kernel<TP, true, false>
                                    : embed_rest_kernel<TP, false, false>;
    others<<<groups, 256, 0, s>>>(e);
    return hipGetLastError();
}

}  // namespace

size_t embed_grad_workspace(int64_t rows, int32_t classes, int32_t n) {
    return embed_grad_plan(rows, classes, n, nullptr).bytes;
}

hipError_t launch_embed(bool bf16, bool bf16_table, const EmbedArgs& a, hipStream_t s) {
    if (!bf16) return embed<float, float>(a, s);
    return bf16_table ? embed<uint16_t, uint16_t>(a, s) : embed<uint16_t, float>(a, s);
}
hipError_t launch_embed_grad(bool bf16, bool bf16_table, const EmbedGradArgs& a, void* ws,
                             hipStream_t s) {
    if (!bf16) return embed_grad<float, float>(a, ws, s);
    return bf16_table ? embed_grad<uint16_t, uint16_t>(a, ws, s)
                      : embed_grad<uint16_t, float>(a, ws, s);
}

}  // namespace kan
