// kan_embed.hip -- rows of a table for tokens, scaled, and the gradient of the table.
//
//   y_b = scale table[t_b]
//   dtable_v = base_v + scale sum_{b: t_b = v} dy_b   (in rising order of b)
//
// The gradient sorts the tokens (stable, by digits of up to nine bits), so that a row's sum has
// one order whatever runs when.  Tokens that occur often are summed in chunks of kRun sorted
// entries first, each to a row of fp32 partial sums; then every row of the table is written once,
// from its own few entries or from its chunks' sums.
#include <algorithm>

#include "kan_head.h"
#include "kan_ops.h"
#include "kan_rows.h"

namespace kan {

namespace {

constexpr int kLoads = 4;  // units in flight per lane

// V elements of a table's row from column c on, as fp32 (0 past the row's end).
template <typename TP, int V>
__device__ __forceinline__ void load_row(const TP* row, int c, int n, float (&v)[V]) {
    constexpr int U = kVec<TP>;
    if (c + V <= n) {
#pragma unroll
        for (int k = 0; k < V / U; ++k) {
            float u[U];
            widen(*unit_at(row, c + k * U), u);
#pragma unroll
            for (int i = 0; i < U; ++i) v[k * U + i] = u[i];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i] = 0.0f;
        if (c + i < n) {
            if constexpr (sizeof(TP) == 2) v[i] = __uint_as_float((uint32_t)row[c + i] << 16);
            else v[i] = row[c + i];
        }
    }
}

template <typename TP, int V>
__device__ __forceinline__ void store_row(TP* row, int c, int n, const float (&v)[V]) {
    constexpr int U = kVec<TP>;
#pragma unroll
    for (int k = 0; k < V / U; ++k) {
        float u[U];
#pragma unroll
        for (int i = 0; i < U; ++i) u[i] = v[k * U + i];
        if (c + k * U < n) store_unit<false>(row, c + k * U, n, u);
    }
}

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
        float v[kLoads][V];
        int64_t row[kLoads], token[kLoads];
        int c[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const uint32_t j = s.at + u * 256 + threadIdx.x, r = j / units;
            row[u] = s.row + r;
            c[u] = (int)(j - r * units) * V;
            token[u] = row[u] < a.rows ? a.tokens[row[u]] : a.ignore;
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const bool in = token[u] != a.ignore && token[u] >= 0 && token[u] < a.classes;
            if (in) {
                load_row(static_cast<const TP*>(a.table) + token[u] * a.tstride, c[u], a.n, v[u]);
#pragma unroll
                for (int i = 0; i < V; ++i) v[u][i] *= a.scale;
            } else {
                const float none = token[u] == a.ignore ? 0.0f : __builtin_nanf("");
#pragma unroll
                for (int i = 0; i < V; ++i) v[u][i] = none;
            }
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (row[u] < a.rows)
                store_unit<false>(static_cast<T*>(a.y) + row[u] * a.n, c[u], a.n, v[u]);
    }
}

// ------------------------------------------------------------ sorting

constexpr int kSortThreads = 1024, kSortWaves = 16, kSortTile = 4096;
constexpr int kBatches = kSortTile / kSortThreads;  // per wave, of 64 neighbours
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;

struct Entry {
    uint32_t key, at;  // token (classes for none), place in the batch
};

__device__ __forceinline__ uint32_t key_of(int64_t token, int64_t ignore, int classes) {
    return token == ignore || token < 0 || token >= classes ? (uint32_t)classes : (uint32_t)token;
}

// Ranks of a tile's entries among those of their digit, in order: wave w holds the kBatches * 64
// entries from w kBatches 64 on, a batch's lanes neighbours.  count: [kSortWaves][kDigits] in LDS;
// afterwards count[w][d] is the number of entries of digit d in waves before w, and total(d, n)
// has been called by one thread per digit with the tile's count of it.
template <typename F>
__device__ __forceinline__ void rank_digits(uint32_t (*count)[kDigits], const uint32_t (&digit)[kBatches],
                                            const bool (&live)[kBatches], int bits,
                                            uint32_t (&rank)[kBatches], F&& total) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, digits = 1 << bits;
    for (int i = threadIdx.x; i < kSortWaves * digits; i += kSortThreads)
        count[i >> bits][i & (digits - 1)] = 0;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kBatches; ++b) {
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

struct SortArgs {
    const int64_t* tokens;  // the first pass's input, or null:
    const Entry* in;
    Entry* out;
    int64_t rows, ignore;
    int classes, shift, bits;
    uint32_t* hist;   // [tiles][kDigits]: counts; before a scatter that follows `scan`: those of
    uint32_t* totals; // tiles before, and [kDigits] counts of all; null: no scan
    int tiles;
    int2* span;       // [classes + 1], to be cleared
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
    if ((int)blockIdx.x >= a.tiles) return;
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) count[d] = 0;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kBatches; ++b) {
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
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, digits = 1 << a.bits;
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
            for (int t = 0; t < a.tiles; ++t) {
                const uint32_t c = a.hist[(int64_t)t * kDigits + d];
                if (t < (int)blockIdx.x) before += c;
                sum += c;
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
        if (live[b]) a.out[first[digit[b]] + count[wave][digit[b]] + rank[b]] = e[b];
}

// At most kSortTile entries: all passes in LDS by the first workgroup; the others clear the spans.
__global__ void __launch_bounds__(kSortThreads) sort_few_kernel(SortArgs a, int bits_all) {
    __shared__ uint32_t count[kSortWaves][kDigits];
    __shared__ uint32_t all[kDigits], first[kDigits];
    __shared__ Entry hold[kSortTile];
    if (blockIdx.x > 0 || gridDim.x == 1)
        clear_spans(a.span, (int64_t)a.classes + 1,
                    (int64_t)(gridDim.x == 1 ? 0 : blockIdx.x - 1) * kSortThreads + threadIdx.x,
                    (int64_t)(gridDim.x == 1 ? 1 : gridDim.x - 1) * kSortThreads);
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
    for (int shift = 0; shift < bits_all; shift += kDigitBits) {
        const int bits = min(kDigitBits, bits_all - shift), digits = 1 << bits;
#pragma unroll
        for (int b = 0; b < kBatches; ++b) digit[b] = e[b].key >> shift & (digits - 1);
        rank_digits(count, digit, live, bits, rank, [&](int d, uint32_t n) { all[d] = n; });
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

// Tokens with more entries than this are summed in chunks of as many.
constexpr int kRun = 32;

struct EmbedSumArgs {
    EmbedGradArgs g;
    const Entry* sorted;
    int2* span;   // [classes + 1] a token's entries: from, to
    float* part;  // [2 chunks][units V] sums of the entries of a token that has more than kRun, in
                  // a chunk: one that starts in an earlier chunk or at its first entry, and one
                  // that starts later
    uint32_t units;
};

template <typename T, int V>
__device__ __forceinline__ void add_rows(const EmbedSumArgs& a, int from, int to, int c,
                                         float (&s)[V]) {
    for (int i = from; i < to; i += 4) {
        float v[4][V];
        uint32_t at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) at[u] = a.sorted[min(i + u, to - 1)].at;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            load_row(static_cast<const T*>(a.g.dy) + at[u] * a.g.dystride, c, a.g.n, v[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i + u >= to) break;
#pragma unroll
            for (int k = 0; k < V; ++k) s[k] += v[u][k];
        }
    }
}

// Spans, and the chunks' sums: a workgroup per chunk.
template <typename T>
__global__ void __launch_bounds__(256) embed_chunk_kernel(EmbedSumArgs a) {
    constexpr int V = kVec<T>;
    const int64_t rows = a.g.rows;
    for (int64_t chunk = blockIdx.x; chunk * kRun < rows; chunk += gridDim.x) {
        const int64_t first = chunk * kRun;
        const int lane = threadIdx.x & 63;
        // the chunk's keys (every wave), those of the chunks around it
        const auto key = [&](int64_t i) {
            return i < 0 || i >= rows ? 0xffffffffu : a.sorted[i].key;
        };
        const int64_t mine = first + lane - kRun;  // lanes: the chunk before, the chunk
        const uint32_t k0 = key(mine), k1 = key(first + kRun + (lane & (kRun - 1)));
        if (threadIdx.x >= kRun && threadIdx.x < 64 && mine < rows) {
            if (key(mine - 1) != k0) a.span[k0].x = (int)mine;
            if (key(mine + 1) != k0) a.span[k0].y = (int)mine + 1;
        }
        // runs of one key that reach into the chunk: the one at its first entry, and one that
        // reaches past its last
#pragma unroll
        for (int slot = 0; slot < 2; ++slot) {
            const uint32_t k = __builtin_amdgcn_readlane((int)k0, slot == 0 ? kRun : 63);
            const uint32_t head = __builtin_amdgcn_readlane((int)k0, kRun);
            if (k >= (uint32_t)a.g.classes || (slot == 1 && k == head)) continue;
            const uint64_t here = __ballot(k0 == k);
            const int in = __popcll(here >> kRun), before = __popcll(here & 0xffffffffu);
            const int after = __popcll(__ballot(k1 == k) & 0xffffffffu);
            if (in + before + after <= kRun) continue;
            const int from = (int)first + __builtin_ctzll(here >> kRun);
            for (uint32_t u = threadIdx.x; u < a.units; u += 256) {
                float s[V] = {};
                add_rows<T, V>(a, from, from + in, u * V, s);
                float* const out = a.part + ((2 * chunk + slot) * a.units + u) * V;
#pragma unroll
                for (int i = 0; i < V; i += 4)
                    *reinterpret_cast<floatx4*>(out + i) =
                        floatx4{s[i], s[i + 1], s[i + 2], s[i + 3]};
            }
        }
    }
}

template <typename T, typename TP>
__global__ void __launch_bounds__(256) embed_sum_kernel(EmbedSumArgs a) {
    constexpr int V = kVec<T>;
    const int64_t all = (int64_t)a.g.classes * a.units;
    for (int64_t first = (int64_t)blockIdx.x * 256; first < all;
         first += (int64_t)gridDim.x * 256) {
        const Share s(first, a.units);
        const uint32_t j = s.at + threadIdx.x, r = j / a.units;
        const int64_t row = s.row + r;
        const uint32_t u = j - r * a.units;
        if (row >= a.g.classes) continue;
        const int2 span = a.span[row];
        const bool in_place = a.g.base == a.g.dtable;
        if (span.x == span.y && in_place) continue;
        float v[V] = {};
        if (span.y - span.x <= kRun) {
            add_rows<T, V>(a, span.x, span.y, u * V, v);
        } else {
            const int c0 = span.x / kRun, c1 = (span.y - 1) / kRun;
            constexpr int U = 8;
            for (int c = c0; c <= c1; c += U) {
                floatx4 p[U][V / 4];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int at = min(c + k, c1);
                    const int slot = 2 * at + (span.x > at * kRun ? 1 : 0);
#pragma unroll
                    for (int i = 0; i < V / 4; ++i)
                        p[k][i] = *reinterpret_cast<const floatx4*>(
                            a.part + ((int64_t)slot * a.units + u) * V + 4 * i);
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if (c + k > c1) break;
#pragma unroll
                    for (int i = 0; i < V; ++i) v[i] += p[k][i / 4][i % 4];
                }
            }
        }
        float b[V] = {};
        if (a.g.base != nullptr)
            load_row(static_cast<const TP*>(a.g.base) + row * a.g.n, (int)u * V, a.g.n, b);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = __builtin_fmaf(v[i], a.g.scale, b[i]);
        store_row(static_cast<TP*>(a.g.dtable) + row * a.g.n, (int)u * V, a.g.n, v);
    }
}

// ------------------------------------------------------------ plans

int64_t div_up(int64_t v, int64_t by) { return (v + by - 1) / by; }
int groups_of(int64_t n) { return (int)std::min<int64_t>(n, kMaxGroups); }

struct EmbedGradPlan {
    Entry* list[2];
    uint32_t *hist, *totals;
    int2* span;
    float* part;
    int tiles, bits, passes;
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
    while (classes >> p.bits) ++p.bits;  // (of the keys 0 .. classes)
    p.passes = (int)div_up(p.bits, kDigitBits);
    p.tiles = (int)div_up(rows, kSortTile);
    const bool few = p.tiles <= 1;
    p.span = reinterpret_cast<int2*>(take(((int64_t)classes + 1) * 8));
    for (int i = 0; i < (few ? 1 : 2); ++i)
        p.list[i] = reinterpret_cast<Entry*>(take(rows * (int64_t)sizeof(Entry)));
    if (!few) {
        p.hist = reinterpret_cast<uint32_t*>(take((int64_t)p.tiles * kDigits * 4));
        p.totals = reinterpret_cast<uint32_t*>(take(kDigits * 4));
    }
    if (rows > kRun)
        p.part = reinterpret_cast<float*>(take(2 * div_up(rows, kRun) * (div_up(n, 8) * 8) * 4));
    return p;
}

#define KAN_TRY(...)                          \
    do {                                      \
        const hipError_t e_ = (__VA_ARGS__);  \
        if (e_ != hipSuccess) return e_;      \
    } while (0)

// Tiles from which the counts before each are summed by a launch of its own.
constexpr int kScanTiles = 64;

template <typename T, typename TP>
hipError_t embed(const EmbedArgs& a, hipStream_t s) {
    const uint32_t units = (uint32_t)div_up(a.n, kVec<T>);
    embed_kernel<T, TP><<<groups_of(div_up(a.rows * units, 256 * kLoads)), 256, 0, s>>>(a, units);
    return hipGetLastError();
}

template <typename T, typename TP>
hipError_t embed_grad(const EmbedGradArgs& g, void* ws, hipStream_t s) {
    const EmbedGradPlan p = embed_grad_plan(g.rows, g.classes, g.n, ws);
    SortArgs a = {g.tokens, nullptr, p.list[0], g.rows, g.ignore, g.classes, 0, p.bits,
                  p.hist, nullptr, p.tiles, p.span};
    const int clear = (int)std::min<int64_t>(div_up((int64_t)g.classes + 1, 4 * kSortThreads), 1024);
    if (p.tiles <= 1) {
        sort_few_kernel<<<clear == 1 ? 1 : clear + 1, kSortThreads, 0, s>>>(a, p.bits);
        KAN_TRY(hipGetLastError());
    } else {
        for (int i = 0; i < p.passes; ++i) {
            a.out = p.list[i & 1];
            a.bits = std::min(kDigitBits, p.bits - a.shift);
            a.totals = nullptr;
            sort_count_kernel<<<i == 0 ? std::max(clear, p.tiles) : p.tiles, kSortThreads, 0, s>>>(a);
            KAN_TRY(hipGetLastError());
            if (p.tiles > kScanTiles) {
                a.totals = p.totals;
                sort_scan_kernel<<<kDigits / 64, 64, 0, s>>>(a);
                KAN_TRY(hipGetLastError());
            }
            sort_scatter_kernel<<<p.tiles, kSortThreads, 0, s>>>(a);
            KAN_TRY(hipGetLastError());
            a.tokens = nullptr;
            a.span = nullptr;
            a.in = a.out;
            a.shift += kDigitBits;
        }
    }
    const EmbedSumArgs e = {g, a.out, p.span, p.part, (uint32_t)div_up(g.n, kVec<T>)};
    if (g.rows > 0) {
        embed_chunk_kernel<T><<<groups_of(div_up(g.rows, kRun)), 256, 0, s>>>(e);
        KAN_TRY(hipGetLastError());
    }
    embed_sum_kernel<T, TP><<<groups_of(div_up((int64_t)g.classes * e.units, 256)), 256, 0, s>>>(e);
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
