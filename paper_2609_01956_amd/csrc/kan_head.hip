// kan_head.hip -- log probabilities of given tokens under a linear head over a long vocabulary,
// without its logits in memory, and their gradient.
//
//   z_bv = scale x_b . w_v,  m = max_v z_bv,  s = sum_v exp(z_bv - m)
//   logp_b = z_bt - m - log s,  best_b = the lowest v with z_bv = m
//   dz_bv = dlogp_b ([v = t_b] - p_bv),  p = exp(z - m - log s)
//   dx = scale dz W,  dW = scale dz^T X
//
// Forward.  Many rows: tiles of 256 x 256 logits (kan_tile.h) on the matrix cores, each reduced in
// registers to its rows' maximum, sum and best class, 8 bytes (and 4) a row and tile; a second kernel
// joins a row's parts.  The workgroups stay, one a CU, and begin a tile's loads before the tile
// ahead of it is reduced.  8192 x 2048 -> 131072 bf16 3.6 ms, 1.22 PFLOP/s; 2001 x 1001 -> 50001, whose
// rows have to be copied first (37 us), 250 us, six turns of the GPU by big tiles and a seventh by
// small ones.  Up to 32 (64) rows: weights straight from memory into 16 x 16 products, x in LDS, bound
// by the reads (1 x 1024 -> 131072 bf16 45 us, 6.0 TB/s).  Few tiles: sums over parts of k in memory.
//
// Gradient.  The logits' tiles again, as dz in memory, 512 MB of it (and of copied weights) at a
// time, of which the two products are made: dx over the classes, dW over the rows, in the same
// tiles, where too few fill the GPU over parts of k that are added after it.  That dz is written once
// and read twice takes less than to make the logits twice: at 8192 x 2048 -> 131072 bf16 the three
// products take 1.05, 0.89 and 0.89 ms for each quarter of the classes, 11.3 ms in all, 1.17 PFLOP/s.
// Few rows: both products in one pass over the weights on the vector ALUs; up to 64 in fp32: dz by the
// forward's kernel of few rows.
#include "kan_head.h"

#include <algorithm>

#include "kan_ops.h"
#include "kan_rows.h"
#include "kan_tile.h"

namespace kan {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f, kLn2Low = -1.904654299957768e-9f;  // their sum
constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kNoIndex = 0x7fffffff;

// exp(t) with the roundings of t log2 e and of the constant: off by at most 1e-7 + 7.3e-8 |t|.
__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(t * kLog2e); }
// To 2^-22 of the value (t above -1e5): what the argument's rounding left out as a factor.
__device__ __forceinline__ float exp_exact(float t) {
    const float h = t * kLog2e, e = __builtin_amdgcn_exp2f(h);
    return __builtin_fmaf(e, __builtin_fmaf(-h, kLn2Low, __builtin_fmaf(-h, kLn2, t)), e);
}
// 1 - exp(t), to 2^-22 of it near t = 0, where the difference would lose what p nearly 1 leaves (nine
// terms of the series: the tenth is below 2^-29 of the sum).
__device__ __forceinline__ float one_less_exp(float t) {
    if (!(__builtin_fabsf(t) <= 0.5f)) return 1.0f - exp_exact(__builtin_fmaxf(t, -1e4f));
    float s = 1.0f;
#pragma unroll
    for (int k = 9; k >= 2; --k) s = __builtin_fmaf(s, t * (1.0f / k), 1.0f);
    return -t * s;
}
// What a maximum is subtracted as: rows (so far) without any class stay at 0.
__device__ __forceinline__ float anchor(float m) { return m == kNegInf ? 0.0f : m; }

// A row's running maximum, sum of exp(z - m), and the lowest class at the maximum.
struct Best {
    float m, s;
    int at;
};
__device__ __forceinline__ Best join(const Best& a, const Best& b) {
    Best c;
    c.m = __builtin_fmaxf(a.m, b.m);
    const float o = anchor(c.m);
    c.s = a.s * exp_of(__builtin_fmaxf(a.m - o, -200.0f)) +
          b.s * exp_of(__builtin_fmaxf(b.m - o, -200.0f));
    c.at = a.m > b.m ? a.at : b.m > a.m ? b.at : min(a.at, b.at);
    return c;
}
__device__ __forceinline__ Best from_lane(const Best& a, int mask) {
    return Best{__shfl_xor(a.m, mask), __shfl_xor(a.s, mask), __shfl_xor(a.at, mask)};
}

// Where a launch leaves a row's parts.
struct Parts {
    float2* sums;  // [parts][rows] m and s
    int* best;     // [parts][rows], or null
    float* target; // [rows] the target's logit
};
__device__ __forceinline__ void leave(const Parts& o, int64_t part, int64_t rows, int64_t row,
                                      const Best& b) {
    o.sums[part * rows + row] = float2{b.m, b.s};
    if (o.best != nullptr) o.best[part * rows + row] = b.at;
}

// fp32 operands of large products go through the matrix cores as bf16 terms: a value is the sum of
// three of 8 bits each, h + m + l (exact for |v| above 2^-109), and a product
// h h' + h m' + m h' + m m' + h l' + l h': what is left out is below 2^-25 of it.  So six segments of k
// in bf16, at sixteen times the fp32 instruction's rate, the small ones first.  The term h stands
// twice, as it is for the last segment, and 0 where it is infinite or NaN for the others, so that
// such values enter the sum once, as they would in fp32.
constexpr int kTerms = 4, kSegments = 6;  // h, h where finite, m, l
constexpr uint32_t kTermsP = 0x012213, kTermsQ = 0x021231;
constexpr uint32_t kTermsDz = 0x010120;   // dz, as Q: h, m, l

template <typename T, int S> using BigLogits = Tile<T, 2, 4, 4, 2, kByRows, kByRows, S>;  // 256 x 256
template <typename T, int S> using SmallLogits = Tile<T, 2, 2, 2, 2, kByRows, kByRows, S>;  // 128 x 128

// The tiles of rows x classes logits.
struct LogitArgs {
    const void *x, *w;
    int64_t rows, xstride, wstride;  // bytes from row to row
    int classes;                     // of this launch, from class `first` on
    int first;
    int k;                           // elements of a row, with its padding
    int tp, tq;
    float scale;
    const int64_t* targets;
    int64_t xplane, wplane;          // bytes from term to term (fp32 as bf16 terms), else 0
};

// Each workgroup's tiles, one after the other: ready(tile, p, q) with the products of tile (p, q),
// after ahead() there has begun the next one's loads, which from then on own the first Tl::STEP bytes
// of lds.
template <typename T, typename Tl, typename F>
__device__ __forceinline__ void for_tiles(const LogitArgs& a, char* lds, F&& ready) {
    char KAN_LDS* const to = (char KAN_LDS*)lds;
    const int tiles = a.tp * a.tq;
    int tp, tq;
    Operand p, q;
    const auto find = [&](int id) {
        tile_of(id, a.tp, a.tq, &tp, &tq);
        p = operand<T, kByRows>(a.w, (int64_t)tp * Tl::BP, a.classes, Tl::BP, a.wstride, 0, a.wplane,
                                kTermsP);
        q = operand<T, kByRows>(a.x, (int64_t)tq * Tl::BQ, a.rows, Tl::BQ, a.xstride, 0, a.xplane,
                                kTermsQ);
    };
    Tl t;
    find(blockIdx.x);
    t.start(to, p, q, 0, a.k);
    for (int id = blockIdx.x; id < tiles; id += gridDim.x) {
        t.run(to, p, q, 0, a.k);
        const int here_p = tp, here_q = tq;
        ready(t, here_p, here_q, [&] {
            if (id + (int)gridDim.x >= tiles) return;
            find(id + gridDim.x);
            t.start(to, p, q, 0, a.k);
        });
    }
}

// Makes acc the logits over c, with c > 0 returned, and those of classes past the end `none`.
template <typename Tl>
__device__ __forceinline__ float settle(Tl& t, const LogitArgs& a, int p0, int tid, float none) {
    if (a.scale > 0.0f && p0 + Tl::BP <= a.classes) return a.scale;
    const int classes = a.classes - p0 - Tl::p_of(tid);
#pragma unroll
    for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
        for (int j = 0; j < Tl::RQ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                t.acc[i][j][e] = Tl::p_step(i, e) < classes ? t.acc[i][j][e] * a.scale : none;
    return 1.0f;
}

struct HeadTileArgs {
    LogitArgs z;
    Parts out;
    int64_t part;  // of the first tile
};

// Bound by the matrix cores; what the logits cost after the products is four operations and an
// exponential each, while the next tile's first loads are on their way.
template <typename T, typename Tl, bool BEST>
__global__ void __launch_bounds__(Tl::THREADS, 2) head_tile_kernel(HeadTileArgs h) {
    __shared__ __attribute__((aligned(128))) char lds[Tl::BYTES];
    const LogitArgs& a = h.z;
    Best* const red = reinterpret_cast<Best*>(lds + Tl::STEP);  // [WP][BQ]
    static_assert(Tl::STEP + Tl::WP * Tl::BQ * (int)sizeof(Best) <= Tl::BYTES, "LDS");
    for_tiles<T, Tl>(a, lds, [&](Tl& t, int tp, int tq, auto&& ahead) {
        const int tid = Tl::thread(), p0 = tp * Tl::BP, p1 = p0 + Tl::p_of(tid);
        const int64_t q0 = (int64_t)tq * Tl::BQ;
        int64_t target[Tl::RQ];
#pragma unroll
        for (int j = 0; j < Tl::RQ; ++j) {
            const int64_t row = q0 + Tl::q_of(tid, j);
            target[j] = row < a.rows ? a.targets[row] : -1;
            target[j] = target[j] < a.first ? -1 : target[j] - a.first;
        }
        ahead();
        const float scale = settle(t, a, p0, tid, kNegInf);
#pragma unroll
        for (int j = 0; j < Tl::RQ; ++j) {
            const int64_t row = q0 + Tl::q_of(tid, j);
            if (target[j] >= p0 && target[j] < p0 + Tl::BP && target[j] < a.classes) {
                const int p = (int)target[j] - p1;
#pragma unroll
                for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (p == Tl::p_step(i, e)) h.out.target[row] = t.acc[i][j][e] * scale;
            }
            Best b = {kNegInf, 0.0f, kNoIndex};
#pragma unroll
            for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if (BEST) b.at = t.acc[i][j][e] > b.m ? Tl::p_step(i, e) : b.at;
                    b.m = __builtin_fmaxf(b.m, t.acc[i][j][e]);
                }
            if (BEST && b.at == kNoIndex) {  // (nothing above -infinity: its first class there)
#pragma unroll
                for (int i = Tl::RP - 1; i >= 0; --i)
#pragma unroll
                    for (int e = 15; e >= 0; --e)
                        if (t.acc[i][j][e] == kNegInf && p1 + Tl::p_step(i, e) < a.classes)
                            b.at = Tl::p_step(i, e);
            }
            if (BEST && b.at != kNoIndex) b.at += p1 + a.first;
            b.m *= scale;
            // (a logit less m with one rounding)
            const float o = -anchor(b.m);
#pragma unroll
            for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    b.s += exp_of(__builtin_fmaf(t.acc[i][j][e], scale, o));
            b = join(b, from_lane(b, 32));
            if ((tid & 63) < 32) red[((tid >> 6) % Tl::WP) * Tl::BQ + Tl::q_of(tid, j)] = b;
        }
        Tl::meet();
        for (int q = tid; q < Tl::BQ; q += Tl::THREADS) {
            if (q0 + q >= a.rows) break;
            Best b = red[q];
#pragma unroll
            for (int i = 1; i < Tl::WP; ++i) b = join(b, red[i * Tl::BQ + q]);
            leave(h.out, h.part + tp, a.rows, q0 + q, b);
        }
        Tl::meet();
    });
}

// ------------------------------------------------------------ the gradient's rows

struct HeadGradTileArgs {
    LogitArgs z;
    const float *stats, *dlogp;
    int64_t ignore;
    int all;          // classes
    void* dz;         // [rows][zstride], 0 past the classes; of fp32 as terms, kDzTerms of them
    int64_t zstride;  // elements, a multiple of 16 bytes
    int64_t zwidth;   // of a row that may be written
    int64_t zplane;   // elements from term to term
};
constexpr int kDzTerms = 3;

// What a row's dz is made of: dz = d ([v = target] - exp(z - m - logs)).
struct RowGrad {
    float m, logs, d;
    int target;  // from the launch's first class on
};
__device__ __forceinline__ RowGrad row_grad(const HeadGradTileArgs& g, int64_t row) {
    // (rows that have no gradient: p = 0, whatever their logits are)
    RowGrad r = {__builtin_huge_valf(), 0.0f, 0.0f, -1};
    if (row >= g.z.rows) return r;
    const int64_t c = g.z.targets[row];
    const float m = g.stats[2 * row], logs = g.stats[2 * row + 1], d = g.dlogp[row];
    if (c == g.ignore) return r;
    // (a target that is no class, NaN and infinite logits show in the row's gradient)
    r.d = c < 0 || c >= g.all || m != m || m == -kNegInf || logs != logs ? __builtin_nanf("") : d;
    if (m == kNegInf && logs == kNegInf && r.d == r.d) {
        r.d = 0.0f;
        return r;
    }
    r.m = m;
    r.logs = logs;
    r.target = (int)c - g.z.first;
    return r;
}
// -d p for the logit less m (of which its scale's rounding is the only one: m + logs taken off at once
// would cost p |m| 2^-24 of it).  Where bf16 follows, which hides the rounding of the exponential's
// argument, log2 e and logs are in that argument's one operation.
template <bool EXACT>
__device__ __forceinline__ float dz_of(const RowGrad& r, float t) {
    return -r.d * (EXACT ? exp_exact(__builtin_fmaxf(t - r.logs, -1e4f))
                         : __builtin_amdgcn_exp2f(__builtin_fmaxf(
                               __builtin_fmaf(t, kLog2e, -r.logs * kLog2e), -1e4f)));
}

// dz of the target for the logit less m.  (By the series in bf16 too: with p near 1, d - d p keeps few
// bits of 1 - p or none, 0 for m = 30 and logs = 7.6e-7.)
__device__ __forceinline__ float target_of(const RowGrad& r, float t) {
    return r.d * one_less_exp(t - r.logs);
}

// ------------------------------------------------------------ few rows

// Elements [k, k + 16 bytes) of a row of n, 0 past its end.
template <typename T>
__device__ __forceinline__ u32x4 chunk_of(const T* row, int k, int n) {
    constexpr int V = kVec<T>;
    if (k + V <= n) return *unit_at(row, k);
    u32x4 r = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (k + i >= n) continue;
        if constexpr (sizeof(T) == 2) r[i / 2] |= (uint32_t)row[k + i] << (16 * (i % 2));
        else r[i] = __float_as_uint(row[k + i]);
    }
    return r;
}

struct HeadThinArgs {
    const void *x, *w;
    int rows;
    int64_t xstride, wstride;  // elements
    int classes, n;
    float scale;
    const int64_t* targets;
    Parts out;
};
constexpr int kThinWaves = 8;
constexpr int kThinLds = 64 << 10;  // bytes of x in LDS at a time (128 KB: one workgroup a CU, slower)

// Rows of weights straight from memory into the matrix instruction, x from LDS: bound by the reads of
// the weights.  NT: groups of 16 rows.  WHAT: the rows' parts, with the best class, or dz in fp32,
// [classes][16 NT].  SPLIT: the waves share one group of 16 classes and split k.
enum { kLogp, kBest, kDz };
template <typename T, int NT, int WHAT, bool SPLIT>
__global__ void __launch_bounds__(64 * kThinWaves) head_thin_kernel(HeadThinArgs a,
                                                                    HeadGradTileArgs grad,
                                                                    float* dz) {
    constexpr bool BEST = WHAT == kBest;
    constexpr int V = kVec<T>, ROWS = 16 * NT;
    constexpr int SLICE = kThinLds / ROWS / 16 & ~7;  // chunks of a row in LDS at a time
    constexpr int TURN = SPLIT ? 1 : kThinWaves;  // groups of 16 classes of a workgroup at a time
    extern __shared__ __attribute__((aligned(128))) char lds[];
    __shared__ Best red[kThinWaves][ROWS];
    static_assert(kThinLds + sizeof(red) <= 160 << 10, "LDS of a CU");
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r16 = lane & 15, quad = lane >> 4;
    const int row0 = blockIdx.y * ROWS, rows = min(a.rows - row0, ROWS);
    const T* const x = static_cast<const T*>(a.x) + row0 * a.xstride;
    const T* const w = static_cast<const T*>(a.w);
    const int chunks = (a.n + V - 1) / V;
    const int width = min((chunks + 7) & ~7, SLICE);  // chunks per row in LDS, a multiple of 8
    const auto fill = [&](int c0) {
        for (int i = threadIdx.x; i < ROWS * width; i += 64 * kThinWaves) {
            const int row = i / width, c = i - row * width;
            u32x4 v = {0, 0, 0, 0};
            if (row < rows && (c0 + c) < chunks)
                v = chunk_of(x + row * a.xstride, (c0 + c) * V, a.n);
            *reinterpret_cast<u32x4*>(lds + ((size_t)row * width + (c ^ (row & 7))) * 16) = v;
        }
    };
    Best best[NT];
    int64_t target[NT];
    RowGrad of[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        best[t] = Best{kNegInf, 0.0f, kNoIndex};
        target[t] = WHAT != kDz && t * 16 + r16 < rows ? a.targets[row0 + t * 16 + r16] : -1;
        if (WHAT == kDz) of[t] = row_grad(grad, row0 + t * 16 + r16);
    }
    const bool once = chunks <= width;
    if (once) {
        fill(0);
        __syncthreads();
    }
    const int groups = (a.classes + 15) >> 4;
    // (all waves of a workgroup take the same turns: x comes in slices between barriers)
    for (int g0 = blockIdx.x * TURN; g0 < groups; g0 += gridDim.x * TURN) {
        const int p0 = (SPLIT ? g0 : g0 + wave) * 16;
        const T* const row = w + (int64_t)min(p0 + r16, a.classes - 1) * a.wstride;
        // (fp32: several sums, each of a part of the products, so that roundings add up less)
        constexpr int SUMS = sizeof(T) == 2 ? 1 : NT <= 2 ? 4 : 2;
        floatx4 all[NT][SUMS] = {};
        for (int c0 = 0; c0 < chunks; c0 += width) {
            if (!once) {
                __syncthreads();
                fill(c0);
                __syncthreads();
            }
            const auto product = [&](int c, u32x4 wv) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int r = t * 16 + r16;
                    const u32x4 xv = *reinterpret_cast<const u32x4*>(
                        lds + ((size_t)r * width + ((c + quad) ^ (r & 7))) * 16);
                    if constexpr (sizeof(T) == 2) {
                        all[t][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, wv), __builtin_bit_cast(bf16x8, xv),
                            all[t][0], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            all[t][i % SUMS] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                                __uint_as_float(wv[i]), __uint_as_float(xv[i]), all[t][i % SUMS], 0,
                                0, 0);
                    }
                }
            };
            // this wave's chunks of the slice: whole ones in all four quarters of the wave first
            const int here = min(width, chunks - c0), each = ((here + 31) >> 5) * 4;
            int c = SPLIT ? min(wave * each, here) : 0;
            const int end = SPLIT ? min(c + each, here) : here;
            const int full = min(end, (a.n / V - c0) & ~3);
            constexpr int U = 8;
            for (; c + 4 * U <= full; c += 4 * U) {
                u32x4 wv[U];
#pragma unroll
                for (int u = 0; u < U; ++u) wv[u] = *unit_at(row, (c0 + c + 4 * u + quad) * V);
#pragma unroll
                for (int u = 0; u < U; ++u) product(c + 4 * u, wv[u]);
            }
            for (; c < full; c += 4) product(c, *unit_at(row, (c0 + c + quad) * V));
            for (; c < end; c += 4) {
                const int at = c0 + c + quad;
                product(c, at < chunks ? chunk_of(row, at * V, a.n) : u32x4{0, 0, 0, 0});
            }
        }
        floatx4 acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            acc[t] = all[t][0];
            if constexpr (SUMS > 1) acc[t] += all[t][1];
            if constexpr (SUMS > 2) acc[t] += all[t][2] + all[t][3];
        }
        if constexpr (SPLIT) {
            // (the only group of the workgroup: its sums may stand where x did)
            floatx4* const sums = reinterpret_cast<floatx4*>(lds);
            __syncthreads();
#pragma unroll
            for (int t = 0; t < NT; ++t) sums[(wave * NT + t) * 64 + lane] = acc[t];
            __syncthreads();
            if (wave != 0) break;
#pragma unroll
            for (int t = 0; t < NT; ++t)
                for (int i = 1; i < kThinWaves; ++i) acc[t] += sums[(i * NT + t) * 64 + lane];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (WHAT == kDz) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int p = p0 + quad * 4 + i;
                    const float v = __builtin_fmaf(acc[t][i], a.scale, -of[t].m);
                    float y = dz_of<true>(of[t], v);
                    if (p == of[t].target) y = target_of(of[t], v);
                    if (p < a.classes) dz[((int64_t)p * NT + t) * 16 + r16] = y;
                }
                continue;
            }
            float m = best[t].m;
            int at = best[t].at;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int p = p0 + quad * 4 + i;
                const float z = p < a.classes ? acc[t][i] * a.scale : kNegInf;
                if (p == target[t] && p < a.classes) a.out.target[row0 + t * 16 + r16] = z;
                if (BEST && (z > m || (z == kNegInf && at == kNoIndex && p < a.classes))) at = p;
                m = __builtin_fmaxf(m, z);
                acc[t][i] = z;
            }
            const float o = anchor(m);
            float s = best[t].s * exp_of(__builtin_fmaxf(best[t].m - o, -200.0f));
#pragma unroll
            for (int i = 0; i < 4; ++i) s += exp_of(acc[t][i] - o);
            best[t] = Best{m, s, at};
        }
    }
    if (WHAT == kDz) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        best[t] = join(best[t], from_lane(best[t], 16));
        best[t] = join(best[t], from_lane(best[t], 32));
        if (quad == 0) red[wave][t * 16 + r16] = best[t];
    }
    __syncthreads();
    const int row = threadIdx.x;
    if (row < rows) {
        Best b = red[0][row];
        for (int i = 1; i < kThinWaves; ++i) b = join(b, red[i][row]);
        leave(a.out, blockIdx.x, a.rows, row0 + row, b);
    }
}

// ------------------------------------------------------------ parts into rows

struct HeadJoinArgs {
    Parts in;
    int64_t rows;
    int parts, classes, lanes;  // lanes (a power of two, at most 64) neighbouring rows
    const int64_t* targets;
    int64_t ignore;
    float *logp, *stats;
    int64_t* best;
};
__global__ void __launch_bounds__(256) head_join_kernel(HeadJoinArgs a) {
    __shared__ Best red[256];
    const int r = threadIdx.x & (a.lanes - 1), strand = threadIdx.x / a.lanes, strands = 256 / a.lanes;
    const int64_t row = (int64_t)blockIdx.x * a.lanes + r;
    Best b = {kNegInf, 0.0f, kNoIndex};
    if (row < a.rows) {
        for (int i = strand; i < a.parts; i += strands) {
            const float2 v = a.in.sums[(int64_t)i * a.rows + row];
            b = join(b, Best{v.x, v.y,
                             a.in.best != nullptr ? a.in.best[(int64_t)i * a.rows + row] : kNoIndex});
        }
    }
    red[threadIdx.x] = b;
    for (int n = 128; n >= a.lanes; n >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < n) red[threadIdx.x] = join(red[threadIdx.x], red[threadIdx.x + n]);
    }
    if (strand != 0 || row >= a.rows) return;
    b = red[r];
    // (a tile takes m = +infinity from sums that are finite before the scale, which leaves it an s of 0)
    const float logs = b.m == -kNegInf ? __builtin_nanf("") : logf(b.s);
    const int64_t t = a.targets[row];
    float lp = 0.0f;
    if (t != a.ignore) {
        lp = __builtin_nanf("");
        if (t >= 0 && t < a.classes)
            lp = b.m == kNegInf && b.s == 0.0f ? kNegInf : a.in.target[row] - b.m - logs;
    }
    a.logp[row] = lp;
    a.stats[2 * row] = b.m;
    a.stats[2 * row + 1] = logs;
    if (a.best != nullptr) a.best[row] = b.at == kNoIndex ? 0 : b.at;
}

// ------------------------------------------------------------ gradient

template <typename T>
__device__ __forceinline__ T rounded(float v) {
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return v;
}

// Four neighbours, `left` of them within the row.
template <typename T>
__device__ __forceinline__ void store_four(T* at, int64_t left, const T (&v)[4]) {
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (left >= 4) {
        *reinterpret_cast<four*>(at) = four{v[0], v[1], v[2], v[3]};
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < left) at[i] = v[i];
}

// dz of the tiles in bf16, or in bf16 terms of fp32 (TERMS): the operand of the products that follow.
// Its rows go through LDS, so that they are stored by whole lines, while the next tile's first
// loads are on their way.
template <typename Tl, bool TERMS>
__global__ void __launch_bounds__(Tl::THREADS, 2) head_grad_kernel(HeadGradTileArgs g) {
    typedef uint16_t T;
    constexpr int V = kVec<T>, U = Tl::BP / V, PITCH = Tl::template PITCH<T>;
    constexpr int AT = Tl::STEP, NEED = AT + Tl::ROWS * PITCH;
    __shared__ __attribute__((aligned(128))) char lds[NEED > Tl::BYTES ? NEED : Tl::BYTES];
    const LogitArgs& a = g.z;
    for_tiles<T, Tl>(a, lds, [&](Tl& t, int tp, int tq, auto&& ahead) {
        const int tid = Tl::thread(), p0 = tp * Tl::BP, p1 = p0 + Tl::p_of(tid);
        const int64_t q0 = (int64_t)tq * Tl::BQ;
        RowGrad row[Tl::RQ];
#pragma unroll
        for (int j = 0; j < Tl::RQ; ++j) row[j] = row_grad(g, q0 + Tl::q_of(tid, j));
        ahead();
        const float scale = settle(t, a, p0, tid, kNegInf);
#pragma unroll
        for (int j = 0; j < Tl::RQ; ++j) {
            const RowGrad& r = row[j];
            const float o = -r.m;
            const bool here = r.target >= p0 && r.target < p0 + Tl::BP;
            const int target = r.target - p1;
            float own = 0.0f;  // the target's logit, then its dz
            if (here) {
#pragma unroll
                for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        own = target == Tl::p_step(i, e) ? t.acc[i][j][e] : own;
                own = target_of(r, __builtin_fmaf(own, scale, o));
            }
#pragma unroll
            for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    t.acc[i][j][e] = dz_of<TERMS>(r, __builtin_fmaf(t.acc[i][j][e], scale, o));
            if (here) {
#pragma unroll
                for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        t.acc[i][j][e] = target == Tl::p_step(i, e) ? own : t.acc[i][j][e];
            }
            if (p0 + Tl::BP > a.classes) {
                const int classes = a.classes - p1;
#pragma unroll
                for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (Tl::p_step(i, e) >= classes) t.acc[i][j][e] = 0.0f;
            }
#pragma unroll 1
            for (int term = 0; term < (TERMS ? kDzTerms : 1); ++term) {
                t.template put<T>(lds + AT, tid, j, [](float v) { return rounded<T>(v); });
                Tl::meet();
                T* const dz = static_cast<T*>(g.dz) + term * g.zplane;
                for (int u = tid; u < Tl::ROWS * U; u += Tl::THREADS) {
                    const int r = u / U, p = (u % U) * V;
                    const int64_t q = q0 + Tl::q_of_row(r, j);
                    if (q < a.rows && p0 + p < g.zwidth)
                        *reinterpret_cast<u32x4*>(dz + q * g.zstride + p0 + p) =
                            *reinterpret_cast<const u32x4*>(lds + AT + r * PITCH +
                                                            p * (int)sizeof(T));
                }
                Tl::meet();
                if (!TERMS) break;
                // (what the term left out)
#pragma unroll
                for (int i = 0; i < Tl::RP; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        t.acc[i][j][e] -= bf16_to_f32(f32_to_bf16(t.acc[i][j][e]));
            }
        }
    });
}

// out[q][p] = scale (sum over k of P(p, k) Q(q, k) + acc), or acc (+)= the sum over a split's k.
struct ProductArgs {
    const void *p, *q;
    int64_t pstride, qstride;  // bytes
    int64_t np, nq, k;
    int64_t pk, qk;            // rows of an operand that stands by k
    int64_t pplane, qplane;    // bytes from term to term (fp32 as bf16 terms), else 0
    uint32_t qterms;
    int64_t k_split;           // k of a split
    int tp, tq;
    float* acc;  // [splits][nq][np], or null
    bool add;    // to what acc holds
    void* out;   // [nq][np], or null
    float scale;
};

// (the operands in bf16 or as bf16 terms; O: of the result)
template <typename O, typename Tl, int MP, int MQ>
__global__ void __launch_bounds__(Tl::THREADS, 2) head_product_kernel(ProductArgs a) {
    typedef uint16_t T;
    constexpr int U = Tl::BP / 4, PITCH = Tl::template PITCH<float>, NEED = Tl::ROWS * PITCH;
    __shared__ __attribute__((aligned(128))) char lds[NEED > Tl::BYTES ? NEED : Tl::BYTES];
    const int tiles = a.tp * a.tq, split = blockIdx.x / tiles;
    int tp, tq;
    tile_of(blockIdx.x - split * tiles, a.tp, a.tq, &tp, &tq);
    const int64_t q0 = (int64_t)tq * Tl::BQ, p0 = (int64_t)tp * Tl::BP;
    const int64_t k0 = split * a.k_split, k1 = a.k - k0 < a.k_split ? a.k : k0 + a.k_split;
    if (k0 >= a.k) return;  // (a last piece that is shorter: nothing to add)
    const Operand p = operand<T, MP>(a.p, p0, a.np, Tl::BP, a.pstride, a.pk, a.pplane,
                                         kTermsP);
    const Operand q = operand<T, MQ>(a.q, q0, a.nq, Tl::BQ, a.qstride, a.qk, a.qplane,
                                         a.qterms);
    Tl t;
    t.start((char KAN_LDS*)lds, p, q, k0, k1);
    t.run((char KAN_LDS*)lds, p, q, k0, k1);
    const int tid = Tl::thread();
#pragma unroll
    for (int j = 0; j < Tl::RQ; ++j) {
        t.template put<float>(lds, tid, j, [](float v) { return v; });
        Tl::meet();
        for (int u = tid; u < Tl::ROWS * U; u += Tl::THREADS) {
            const int r = u / U, c = (u % U) * 4;
            const int64_t row = q0 + Tl::q_of_row(r, j), left = a.np - p0 - c;
            if (row >= a.nq || left <= 0) continue;
            const floatx4 v = *reinterpret_cast<const floatx4*>(lds + r * PITCH + c * 4);
            float o[4] = {v[0], v[1], v[2], v[3]};
            float* const acc = a.acc + (split * a.nq + row) * a.np + p0 + c;
            if (a.add) {
                if (left >= 4) {
                    typedef float four __attribute__((ext_vector_type(4), aligned(4)));
                    const four w = *reinterpret_cast<const four*>(acc);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] += w[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < left) o[e] += acc[e];
                }
            }
            if (a.out == nullptr) {
                store_four(acc, left, o);
                continue;
            }
            O w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = rounded<O>(o[e] * a.scale);
            store_four(static_cast<O*>(a.out) + row * a.np + p0 + c, left, w);
        }
        Tl::meet();
    }
}

// Few rows: both products at once, each weight read and each of its gradients written once, on the
// vector ALUs (two fused multiply-adds per weight and row).  A lane holds four columns of x and of
// dx, R rows of them; a wave goes through its classes, the dz of four of them in a lane each, and
// the waves of a workgroup add their dx through LDS.
constexpr int kOuterRows = 16, kOuterWaves = 4;
struct HeadOuterArgs {
    const void *x, *w;
    const float* dz;           // [classes][kOuterRows]
    int64_t xstride, wstride;  // elements
    int rows, classes, n;
    int each;                  // classes of a wave
    const int64_t* targets;
    int64_t ignore;
    float scale;
    float* part;               // [workgroups of a column block][rows][n], or null
    void* dw;                  // or null
};
// Four columns of a row (0 past its end), at any alignment.
template <typename T>
struct Four {
    typedef T any __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    any v;
    __device__ __forceinline__ void load(const T* row, int left) {
        v = any{};
        if (left >= 4) {
            v = *reinterpret_cast<const any*>(row);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < left) v[i] = row[i];
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 2) return bf16_to_f32(v[i]);
        else return v[i];
    }
};

template <typename T, int R>
__global__ void __launch_bounds__(64 * kOuterWaves) head_outer_kernel(HeadOuterArgs a, int blocks) {
    constexpr int U = R == 16 ? 4 : 8;  // classes in flight
    __shared__ float sums[kOuterWaves][R][256];
    static_assert(kOuterRows == 16, "four classes' dz a wave");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int block = blockIdx.x % blocks, slice = blockIdx.x / blocks;
    const int c = (block * 64 + lane) * 4, left = a.n - c;
    float x[R][4], dx[R][4] = {};
#pragma unroll
    for (int r = 0; r < R; ++r) {
        Four<T> v;
        // (nothing of what ignored rows hold)
        const bool live = r < a.rows && a.targets[r] != a.ignore;
        v.load(static_cast<const T*>(a.x) + (live ? r * a.xstride + c : 0), live ? left : 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[r][i] = v.get(i);
    }
    const int64_t first = ((int64_t)slice * kOuterWaves + wave) * a.each;
    const int64_t last = first + a.each < a.classes ? first + a.each : a.classes;
    for (int64_t p = first; p < last; p += U) {
        Four<T> w[U];
        float dz[U / 4];
#pragma unroll
        for (int q = 0; q < U / 4; ++q) {
            const int64_t at = p + 4 * q + (lane >> 4);
            dz[q] = a.dz[(at < last ? at : p) * kOuterRows + (lane & 15)];
        }
        if (a.part != nullptr) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                w[u].load(static_cast<const T*>(a.w) + (p + u < last ? p + u : p) * a.wstride + c,
                          left);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= last) break;
            float g[4] = {};
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float d = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(
                    (int)__float_as_uint(dz[u / 4]), (u % 4) * 16 + r));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (a.part != nullptr) dx[r][i] = __builtin_fmaf(d, w[u].get(i), dx[r][i]);
                    g[i] = __builtin_fmaf(d, x[r][i], g[i]);
                }
            }
            if (a.dw != nullptr && left > 0) {
                T o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = rounded<T>(g[i] * a.scale);
                store_four(static_cast<T*>(a.dw) + (p + u) * a.n + c, left, o);
            }
        }
    }
    if (a.part == nullptr) return;
#pragma unroll
    for (int r = 0; r < R; ++r)
        *reinterpret_cast<floatx4*>(&sums[wave][r][lane * 4]) =
            floatx4{dx[r][0], dx[r][1], dx[r][2], dx[r][3]};
    __syncthreads();
    const int at = block * 256 + threadIdx.x;
    if (at >= a.n) return;
    for (int r = 0; r < a.rows; ++r) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < kOuterWaves; ++k) s += sums[k][r][threadIdx.x];
        a.part[((int64_t)slice * a.rows + r) * a.n + at] = s;
    }
}

// out = scale times the sum of many parts of few values: 16 lanes a value, each a sixteenth of the
// parts.
template <typename T>
__global__ void __launch_bounds__(256) head_gather_kernel(const float* part, int parts, int64_t n,
                                                          float scale, T* out) {
    __shared__ float sums[16][17];
    const int v = threadIdx.x & 15, strand = threadIdx.x >> 4;
    for (int64_t first = (int64_t)blockIdx.x * 16; first < n; first += (int64_t)gridDim.x * 16) {
        float s = 0.0f;
        if (first + v < n)
            for (int k = strand; k < parts; k += 16) s += part[k * n + first + v];
        __syncthreads();
        sums[strand][v] = s;
        __syncthreads();
        if (threadIdx.x < 16 && first + v < n) {
            s = 0.0f;
            for (int k = 0; k < 16; ++k) s += sums[k][v];
            out[first + v] = rounded<T>(s * scale);
        }
    }
}

// out = scale times the sum of the splits, in their order.
template <typename T>
__global__ void __launch_bounds__(256) head_sum_kernel(const float* acc, int splits, int64_t n,
                                                       float scale, T* out) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n;
         i += (int64_t)gridDim.x * 1024) {
        typedef float four __attribute__((ext_vector_type(4), aligned(4)));
        const int64_t left = n - i;
        float s[4] = {};
        for (int k = 0; k < splits; ++k) {
            const float* const at = acc + k * n + i;
            if (left >= 4) {
                const four v = *reinterpret_cast<const four*>(at);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] += v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < left) s[e] += at[e];
            }
        }
        T r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = rounded<T>(s[e] * scale);
        store_four(out + i, left, r);
    }
}

// The logit of a class (before the scale) from its sums over k in parts.
__device__ __forceinline__ float sum_of(const float* z, int splits, int64_t step) {
    float s = z[0];
    for (int k = 1; k < splits; ++k) s += z[k * step];
    return s;
}

struct HeadRowsArgs {
    const float* z;  // [splits][rows][classes] sums over k
    int splits;
    int64_t rows;
    int classes;
    float scale;
    const int64_t* targets;
    int64_t ignore;
    float *logp, *stats;
    int64_t* best;
};

// Few tiles: the logits' sums, which were made in parts of k, to what is asked; a row per wave, or
// per workgroup (WHOLE), four classes of a lane at a time.
template <bool WHOLE>
__global__ void __launch_bounds__(256) head_rows_kernel(HeadRowsArgs a) {
    constexpr int U = 4, LANES = WHOLE ? 256 : 64;
    __shared__ Best waves[4];
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t row = WHOLE ? (int64_t)blockIdx.x
                              : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.rows) return;
    const float* const z = a.z + row * a.classes;
    const int64_t step = a.rows * a.classes;
    Best b = {kNegInf, 0.0f, kNoIndex};
    for (int c = lane; c < a.classes; c += U * LANES) {
        float v[U] = {};
        for (int k = 0; k < a.splits; ++k)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] += z[k * step + min(c + u * LANES, a.classes - 1)];
        // (a NaN adds to the sum alone)
        Best here = {kNegInf, 0.0f, kNoIndex};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = c + u * LANES < a.classes;
            v[u] = in ? v[u] * a.scale : kNegInf;
            if (in && (v[u] > here.m || (v[u] == here.m && here.at == kNoIndex)))
                here.at = c + u * LANES;
            here.m = __builtin_fmaxf(here.m, v[u]);
        }
        b = join(b, here);
#pragma unroll
        for (int u = 0; u < U; ++u) b.s += exp_of(v[u] - anchor(b.m));
    }
    for (int o = 1; o < 64; o *= 2) b = join(b, from_lane(b, o));
    if (WHOLE) {
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = b;
        __syncthreads();
        b = join(join(waves[0], waves[1]), join(waves[2], waves[3]));
    }
    if (lane != 0) return;
    const float logs = logf(b.s);
    const int64_t t = a.targets[row];
    float lp = 0.0f;
    if (t != a.ignore) {
        lp = __builtin_nanf("");
        if (t >= 0 && t < a.classes)
            lp = b.m == kNegInf && b.s == 0.0f
                     ? kNegInf
                     : sum_of(z + t, a.splits, step) * a.scale - b.m - logs;
    }
    a.logp[row] = lp;
    a.stats[2 * row] = b.m;
    a.stats[2 * row + 1] = logs;
    if (a.best != nullptr) a.best[row] = b.at == kNoIndex ? 0 : b.at;
}

// dz of eight classes of a row from c0 on, as head_grad_kernel leaves it.
template <bool TERMS>
__device__ __forceinline__ void leave_dz(const HeadGradTileArgs& g, int64_t row, int c0, float (&y)[8]) {
    uint16_t* out = static_cast<uint16_t*>(g.dz) + row * g.zstride + c0;
    for (int term = 0; term < (TERMS ? kDzTerms : 1); ++term, out += g.zplane) {
        const u32x4 h = narrow(y);
        *reinterpret_cast<u32x4*>(out) = h;
        float w[8];
        widen(h, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] -= w[k];
    }
}

// The same for the gradient: dz as head_grad_kernel leaves it, 16 bytes a lane.
template <bool TERMS>
__global__ void __launch_bounds__(256) head_dz_kernel(HeadGradTileArgs g, const float* z, int splits) {
    const LogitArgs& a = g.z;
    const uint32_t units = (uint32_t)(g.zstride / 8);
    const int64_t all = a.rows * units, step = a.rows * a.classes;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all;
         i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / units;
        const int c0 = (int)(i - row * units) * 8;
        const RowGrad r = row_grad(g, row);
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = c0 + k;
            y[k] = 0.0f;
            if (c >= a.classes) continue;
            const float v = sum_of(z + row * a.classes + c, splits, step);
            const float t = __builtin_fmaf(v, a.scale, -r.m);
            y[k] = c == r.target ? target_of(r, t) : dz_of<TERMS>(r, t);
        }
        leave_dz<TERMS>(g, row, c0, y);
    }
}

// Up to 64 rows' dz in fp32, [classes][pitch], as terms by rows.
__global__ void __launch_bounds__(256) head_turn_kernel(HeadGradTileArgs g, const float* dz, int pitch) {
    const int64_t all = g.zstride / 8 * pitch;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all;
         i += (int64_t)gridDim.x * 256) {
        const int64_t unit = i / pitch;
        const int row = (int)(i - unit * pitch), c0 = (int)unit * 8;
        if (row >= g.z.rows) continue;
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            y[k] = c0 + k < g.z.classes ? dz[(int64_t)(c0 + k) * pitch + row] : 0.0f;
        leave_dz<true>(g, row, c0, y);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) head_zero_kernel(T* out, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
        out[i] = T(0);
}

// ------------------------------------------------------------ rows laid out for the tiles

// Rows of n elements to be laid out as rows of `to` elements (a multiple of 16 bytes), 0 past n; 0
// throughout for rows whose target is `ignore` (targets null: none).  x null: no rows.
struct Rows {
    const void* x;
    int64_t stride, rows;
    int n, to;
    void* out;
    const int64_t* targets;
    int64_t ignore;
    int groups;  // workgroups that do it
};
// Of two in one launch the one that this workgroup does, and its place among those that do.
__device__ __forceinline__ const Rows& rows_of(const Rows& a, const Rows& b, int* group) {
    const bool first = (int)blockIdx.x < a.groups;
    *group = first ? blockIdx.x : blockIdx.x - a.groups;
    return first ? a : b;
}

// Copied.
template <typename T>
__global__ void __launch_bounds__(256) head_pack_kernel(Rows one, Rows two) {
    constexpr int V = kVec<T>;
    int group;
    const Rows& r = rows_of(one, two, &group);
    const int units = r.to / V;
    const int64_t all = r.rows * units;
    for (int64_t i = (int64_t)group * 256 + threadIdx.x; i < all; i += (int64_t)r.groups * 256) {
        const int64_t row = i / units;
        const int c = (int)(i - row * units) * V;
        u32x4 v = {0, 0, 0, 0};
        if (r.targets == nullptr || r.targets[row] != r.ignore)
            v = chunk_of(static_cast<const T*>(r.x) + row * r.stride, c, r.n);
        *reinterpret_cast<u32x4*>(static_cast<T*>(r.out) + row * r.to + c) = v;
    }
}

// fp32 as kTerms terms.
__global__ void __launch_bounds__(256) head_terms_kernel(Rows one, Rows two) {
    int group;
    const Rows& r = rows_of(one, two, &group);
    const int units = r.to / 8;
    const int64_t all = r.rows * units;
    for (int64_t i = (int64_t)group * 256 + threadIdx.x; i < all; i += (int64_t)r.groups * 256) {
        const int64_t row = i / units;
        const int c = (int)(i - row * units) * 8;
        float v[8] = {}, finite[8];
        if (r.targets == nullptr || r.targets[row] != r.ignore) {
            const float* const x = static_cast<const float*>(r.x) + row * r.stride;
            const u32x4 a = chunk_of(x, c, r.n), b = chunk_of(x, c + 4, r.n);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(a[k]), v[4 + k] = __uint_as_float(b[k]);
        }
        u32x4* const at =
            reinterpret_cast<u32x4*>(static_cast<uint16_t*>(r.out) + row * r.to + c);
        const int64_t plane = r.rows * r.to / 8;
        u32x4 h = narrow(v);
        float w[8];
        widen(h, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // (a finite value whose rounding is infinite: the largest instead)
            const bool is = __builtin_fabsf(v[k]) < __builtin_huge_valf();
            if (is && __builtin_fabsf(w[k]) == __builtin_huge_valf())
                w[k] = __builtin_copysignf(3.38953139e38f, v[k]);
            finite[k] = is ? w[k] : 0.0f;
        }
        at[0] = narrow(w);
        at[plane] = narrow(finite);
#pragma unroll
        for (int t = 2; t < kTerms; ++t) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = finite[k] == 0.0f ? 0.0f : v[k] - finite[k];
            h = narrow(v);
            at[t * plane] = h;
            widen(h, finite);
        }
    }
}

// ------------------------------------------------------------ plans

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t div_up(int64_t v, int64_t by) { return (v + by - 1) / by; }

// Device memory handed out piece by piece (from null: sizes alone).
struct Arena {
    char* base;
    size_t at = 0;
    template <typename T = char>
    T* take(int64_t bytes) {
        char* p = base == nullptr ? nullptr : base + at;
        at += (size_t)up(bytes, 256);
        return reinterpret_cast<T*>(p);
    }
};

constexpr int kBig = 256, kSmall = 128;  // a tile's sides
// Rows up to which the weights are read once, past the tiles: 32; 64 where the tiles would need a
// copy of the weights or, in fp32, multiply 128 rows (64 x 1024 -> 131072 bf16 61 us, by tiles 50;
// 64 x 1024 -> 50001 fp32 91, by tiles 131).
constexpr int kThinRows = 32, kThinMost = 64;
// fp32 rows up to which that is done in groups of kThinMost where the tiles would need a copy of the
// weights and terms do not pay: 156 x 935 -> 35856 169 us, by tiles 277; without a copy tiles are
// as fast at 65 rows and faster above (256 x 1024 -> 50001 252 us against 302).
constexpr int kThinGroups = 256;
// Bytes of a piece's intermediate tensors.
constexpr int64_t kPieceBytes = INT64_C(512) << 20;
constexpr int64_t kPieceClasses = 1 << 20, kPieceTiles = 1 << 20;
constexpr int kFillTiles = 256;  // tiles that occupy the GPU

// Microseconds that `groups` tiles of `steps` steps take, by measured rates: a big tile (one a CU)
// 1.65 us a step, two small ones a CU 1.04, one 0.7, 4.2 times that on the fp32 instruction; what
// comes before and after the steps 8 and 5.
double tile_time(bool big, int64_t groups, int64_t steps, int es) {
    const double step = (big ? 1.65 : groups > kFillTiles ? 1.04 : 0.7) * (es == 4 ? 4.2 : 1.0);
    return (double)div_up(groups, big ? kFillTiles : 2 * kFillTiles) * (steps * step + (big ? 8 : 5));
}
int64_t tiles_of(int64_t a, int64_t b, bool big) {
    const int side = big ? kBig : kSmall;
    return div_up(a, side) * div_up(b, side);
}
// Steps of k in `segments` segments; es: bytes of the operands' elements.
int64_t steps_of(int64_t k, int es, bool terms) {
    return div_up(k, 128 / es) * (terms ? kSegments : 1);
}

// How many of `wide` (classes) by `rows` products big tiles make: all, none, or as many as fill the
// GPU some whole turns, with small tiles for the rest in a second launch.
struct Mix {
    int64_t big;  // of wide: a multiple of kBig, or all
    double time;
};
constexpr double kSecondLaunch = 4.0;
Mix mix_of(int64_t rows, int64_t wide, int64_t k, int es, bool terms) {
    const int64_t steps = steps_of(k, es, terms), tiles = tiles_of(rows, wide, true);
    Mix m = {wide, tile_time(true, tiles, steps, es)};
    const auto offer = [&](int64_t big, double time) {
        if (time < m.time) m = {big, time};
    };
    offer(0, tile_time(false, tiles_of(rows, wide, false), steps, es));
    const int64_t high = div_up(rows, kBig), big = tiles / kFillTiles * kFillTiles / high * kBig;
    if (big > 0 && big < wide)
        offer(big, tile_time(true, big / kBig * high, steps, es) + kSecondLaunch +
                       tile_time(false, tiles_of(rows, wide - big, false), steps, es));
    return m;
}
// The tiles along `wide`.
int64_t parts_of(int64_t big, int64_t wide) { return div_up(big, kBig) + div_up(wide - big, kSmall); }

constexpr int64_t kTermRows = 384;
// fp32 operands as bf16 terms: what making them costs (12 bytes of memory traffic an element) is
// regained by the product with about kTermRows rows of the other operand, and where a tile a CU or
// less leaves the time to its steps of k.
bool by_terms(const HeadShape& s) {
    if (s.es != 4) return false;
    return s.rows * s.classes >= kTermRows * (s.rows + s.classes) ||
           (s.n >= 64 && tiles_of(s.rows, s.classes, false) <= kFillTiles);
}

// A product out[nq][np] over k: its tiles, and how k is split where they are few.
struct ProductPlan {
    bool big;
    double time;
    int tp, splits;
    int64_t k_split;
    int64_t rest;  // of nq: the first row that small tiles make in a second launch, or nq
};
// The least of the time for the tiles and, with k in splits, for their sums (written and read at
// about 4.5 TB/s, one more launch).
ProductPlan product_plan(int64_t np, int64_t nq, int64_t k, bool terms) {
    ProductPlan p = {};
    const int es = 2;
    const int64_t step = 128 / es, steps = div_up(k, step);
    double least = 0.0;
    for (const bool big : {true, false}) {
        const int64_t tiles = tiles_of(np, nq, big);
        // (1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 15, ..: a few are enough)
        const int64_t most = std::min({steps, steps_of(k, es, terms) / 4,
                                       8 * kFillTiles / std::max<int64_t>(1, tiles)});
        for (int64_t splits = 1; splits == 1 || splits <= std::min<int64_t>(most, 2 * kFillTiles);
             splits += std::max<int64_t>(1, splits / 4)) {
            const double time =
                tile_time(big, tiles * splits, steps_of(div_up(k, splits), es, terms), es) +
                (splits > 1 ? 4.0 + 2.0 * splits * np * nq * 4 / 4.5e6 : 0.0);
            if (least > 0.0 && time >= least) continue;
            least = time;
            p.big = big;
            p.splits = (int)splits;
        }
    }
    const Mix mix = mix_of(np, nq, k, es, terms);
    p.rest = nq;
    if (mix.big > 0 && mix.big < nq && mix.time < least) {
        least = mix.time;
        p.big = true;
        p.splits = 1;
        p.rest = mix.big;
    }
    p.time = least;
    const int b = p.big ? kBig : kSmall;
    p.tp = (int)div_up(np, b);
    p.k_split = div_up(steps, p.splits) * step;
    p.splits = (int)div_up(k, p.k_split);
    return p;
}

// Few tiles with a long k: the logits' sums over parts of k, in memory, rather than the tiles' own
// logits (8 us: the launch that reads them).  0: no.
constexpr int64_t kSumsBytes = INT64_C(64) << 20;
ProductPlan sums_plan(int64_t rows, int64_t classes, int64_t k, bool terms) {
    ProductPlan p = {};
    const int es = 2;
    if (tiles_of(rows, classes, true) > kFillTiles) return p;
    const double own = mix_of(rows, classes, k, es, terms).time;
    p = product_plan(classes, rows, k, terms);
    if (p.time + 8.0 >= own || p.splits * rows * classes * 4 > kSumsBytes) p.splits = 0;
    return p;
}

struct HeadPlan {
    bool thin, terms;
    int64_t parts;
    int64_t piece;      // classes
    int to;             // elements of a packed row
    Parts out;
    void *xp, *wp;      // packed rows, or null
    ProductPlan pz;     // splits > 0: the logits' sums
    float* z;
    size_t bytes;
};

// Few classes and a long k: a workgroup for each 16 classes.
bool thin_split(const HeadShape& s) {
    return div_up(s.classes, 16) <= 2 * kFillTiles && div_up(s.n, 16 / s.es) >= 64;
}
int thin_groups(const HeadShape& s) {
    return (int)std::min<int64_t>(div_up(div_up(s.classes, 16), thin_split(s) ? 1 : kThinWaves),
                                  2 * kFillTiles);
}
HeadPlan head_plan(const HeadShape& s, void* ws) {
    HeadPlan p = {};
    Arena arena = {static_cast<char*>(ws)};
    p.thin = s.rows <= (s.es == 2 && s.ws ? kThinRows : kThinMost) ||
             (s.es == 4 && !s.ws && s.rows <= kThinGroups && !by_terms(s));
    p.terms = !p.thin && by_terms(s);
    p.to = (int)up(s.n, p.terms ? 8 : 16 / s.es);
    const int64_t packed = (int64_t)p.to * (p.terms ? kTerms * 2 : s.es);  // bytes of a row
    const bool xp = p.terms || !s.xs, wp = p.terms || !s.ws;
    if (p.thin) {
        p.parts = thin_groups(s);
    } else {
        int64_t most = kPieceTiles / div_up(s.rows, kSmall) * kSmall / kBig * kBig;
        if (wp) most = std::min(most, std::max<int64_t>(kPieceBytes / packed / kBig * kBig, kBig));
        p.piece = up(div_up(s.classes, div_up(s.classes, most)), kBig);
        for (int64_t first = 0; first < s.classes; first += p.piece) {
            const int64_t here = std::min<int64_t>(s.classes - first, p.piece);
            p.parts += parts_of(mix_of(s.rows, here, s.n, p.terms ? 2 : s.es, p.terms).big, here);
        }
        if (xp) p.xp = arena.take(s.rows * packed);
        if (wp) p.wp = arena.take(p.piece * packed);
        if (p.piece >= s.classes && (p.terms || s.es == 2))
            p.pz = sums_plan(s.rows, s.classes, s.n, p.terms);
        if (p.pz.splits > 0) {
            p.z = arena.take<float>((int64_t)p.pz.splits * s.rows * s.classes * 4);
            p.bytes = arena.at;
            return p;
        }
    }
    p.out.sums = arena.take<float2>(p.parts * s.rows * 8);
    p.out.best = arena.take<int>(p.parts * s.rows * 4);
    p.out.target = arena.take<float>(s.rows * 4);
    p.bytes = arena.at;
    return p;
}

int grid_of(int64_t items, int per) { return (int)std::min<int64_t>(div_up(items, per), 1 << 16); }

// Rows copied (T), or as terms of fp32 ones, both in one launch.
template <typename T>
hipError_t pack(bool terms, Rows one, Rows two, hipStream_t st) {
    for (Rows* r : {&one, &two})
        r->groups = r->x == nullptr ? 0 : grid_of(r->rows * (r->to / (terms ? 8 : kVec<T>)), 256);
    const int groups = one.groups + two.groups;
    if (groups == 0) return hipSuccess;
    if (terms) head_terms_kernel<<<groups, 256, 0, st>>>(one, two);
    else head_pack_kernel<T><<<groups, 256, 0, st>>>(one, two);
    return hipGetLastError();
}

#define KAN_TRY(...)                          \
    do {                                      \
        const hipError_t e_ = (__VA_ARGS__);  \
        if (e_ != hipSuccess) return e_;      \
    } while (0)

template <typename T, int NT, int WHAT>
hipError_t thin(const HeadShape& s, const HeadThinArgs& a, const HeadGradTileArgs& g, float* dz,
                hipStream_t st) {
    const bool split = thin_split(s);
    const int chunks = (int)div_up(a.n, kVec<T>), slice = kThinLds / (16 * NT) / 16 & ~7;
    // (x, and the waves' sums after it)
    const size_t lds = std::max((size_t)16 * NT * std::min((chunks + 7) & ~7, slice) * 16,
                                (size_t)(split ? kThinWaves * NT * 1024 : 0));
    const auto kernel =
        split ? head_thin_kernel<T, NT, WHAT, true> : head_thin_kernel<T, NT, WHAT, false>;
    const dim3 groups(thin_groups(s), (unsigned)div_up(a.rows, 16 * NT));
    kernel<<<groups, 64 * kThinWaves, lds, st>>>(a, g, dz);
    return hipGetLastError();
}
template <typename T, int WHAT>
hipError_t thin(const HeadShape& s, const HeadThinArgs& a, hipStream_t st) {
    const HeadGradTileArgs none = {};
    const int64_t rows = div_up(a.rows, div_up(a.rows, kThinMost));  // of workgroups' own
    return rows <= 16   ? thin<T, 1, WHAT>(s, a, none, nullptr, st)
           : rows <= 32 ? thin<T, 2, WHAT>(s, a, none, nullptr, st)
           : rows <= 48 ? thin<T, 3, WHAT>(s, a, none, nullptr, st)
                        : thin<T, 4, WHAT>(s, a, none, nullptr, st);
}
HeadThinArgs thin_args(const HeadShape& s, const void* x, const void* w, float scale,
                       const int64_t* targets) {
    HeadThinArgs t = {};
    t.x = x;
    t.w = w;
    t.rows = (int)s.rows;
    t.xstride = s.xstride;
    t.wstride = s.wstride;
    t.classes = s.classes;
    t.n = s.n;
    t.scale = scale;
    t.targets = targets;
    return t;
}

// Workgroups that are resident together: one of a big tile on a CU, or two of a small one.
int resident(int tiles, bool big) { return std::min(tiles, big ? kFillTiles : 2 * kFillTiles); }

// launch(z, classes before, are its tiles big) for the first `big` classes, and for the rest.
template <typename F>
hipError_t by_tiles(const LogitArgs& all, int64_t big, F&& launch) {
    for (const bool first : {true, false}) {
        const int64_t from = first ? 0 : big, here = first ? big : all.classes - big;
        if (here == 0) continue;
        const int side = first ? kBig : kSmall;
        LogitArgs z = all;
        z.w = static_cast<const char*>(all.w) + from * all.wstride;
        z.first = (int)(all.first + from);
        z.classes = (int)here;
        z.tp = (int)div_up(here, side);
        z.tq = (int)div_up(all.rows, side);
        KAN_TRY(launch(z, from, first));
    }
    return hipSuccess;
}

template <typename T, typename Tl>
hipError_t logit_tiles(const HeadTileArgs& a, bool best, bool big, hipStream_t st) {
    const int groups = resident(a.z.tp * a.z.tq, big);
    if (best) head_tile_kernel<T, Tl, true><<<groups, Tl::THREADS, 0, st>>>(a);
    else head_tile_kernel<T, Tl, false><<<groups, Tl::THREADS, 0, st>>>(a);
    return hipGetLastError();
}
template <typename T, int S>
hipError_t logit_tiles(const HeadTileArgs& a, const void* best, bool big, hipStream_t st) {
    return big ? logit_tiles<T, BigLogits<T, S>>(a, best != nullptr, true, st)
               : logit_tiles<T, SmallLogits<T, S>>(a, best != nullptr, false, st);
}

// O: the type of the call (of its operands, in fp32 as bf16 terms, and its results).
template <typename O, int MP, int MQ>
hipError_t product(const ProductPlan& p, const ProductArgs& all, hipStream_t st) {
    constexpr int S = sizeof(O) == 4 ? kSegments : 1;
    typedef Tile<uint16_t, 2, 4, 4, 2, MP, MQ, S> Big;
    typedef Tile<uint16_t, 2, 2, 2, 2, MP, MQ, S> Small;
    const int64_t rest = std::min(p.rest, all.nq);
    ProductArgs a = all;
    a.nq = rest;
    a.k_split = p.k_split;
    a.tp = p.tp;
    a.tq = (int)div_up(rest, p.big ? kBig : kSmall);
    const int groups = a.tp * a.tq * p.splits;
    if (p.big) head_product_kernel<O, Big, MP, MQ><<<groups, Big::THREADS, 0, st>>>(a);
    else head_product_kernel<O, Small, MP, MQ><<<groups, Small::THREADS, 0, st>>>(a);
    KAN_TRY(hipGetLastError());
    if (rest == all.nq) return hipSuccess;
    a.q = static_cast<const char*>(all.q) + rest * (MQ == kByRows ? all.qstride : 2);
    a.nq = all.nq - rest;
    a.tp = (int)div_up(all.np, kSmall);
    a.tq = (int)div_up(a.nq, kSmall);
    if (all.out != nullptr) a.out = static_cast<O*>(all.out) + rest * all.np;
    if (all.acc != nullptr) a.acc = all.acc + rest * all.np;
    head_product_kernel<O, Small, MP, MQ><<<a.tp * a.tq, Small::THREADS, 0, st>>>(a);
    return hipGetLastError();
}

// The sums over k of a launch's logits, in parts: [splits][rows][classes].
template <typename O>
hipError_t sums(const ProductPlan& p, const LogitArgs& z, float* out, hipStream_t st) {
    ProductArgs r = {};
    r.p = z.w;
    r.q = z.x;
    r.pstride = z.wstride;
    r.qstride = z.xstride;
    r.pplane = z.wplane;
    r.qplane = z.xplane;
    r.qterms = kTermsQ;
    r.np = z.classes;
    r.nq = z.rows;
    r.k = z.k;
    r.acc = out;
    return product<O, kByRows, kByRows>(p, r, st);
}

template <typename T>
hipError_t head(const HeadShape& s, const HeadArgs& a, void* ws, hipStream_t st) {
    HeadPlan p = head_plan(s, ws);
    if (a.best == nullptr) p.out.best = nullptr;
    if (p.thin) {
        HeadThinArgs t = thin_args(s, a.x, a.w, a.scale, a.targets);
        t.out = p.out;
        KAN_TRY(a.best != nullptr ? thin<T, kBest>(s, t, st) : thin<T, kLogp>(s, t, st));
    } else {
        HeadTileArgs t = {};
        const int es = p.terms ? 2 : s.es;
        t.z.x = p.xp != nullptr ? p.xp : a.x;
        t.z.xstride = (p.xp != nullptr ? p.to : s.xstride) * es;
        t.z.wstride = (p.wp != nullptr ? p.to : s.wstride) * es;
        t.z.xplane = p.terms ? s.rows * p.to * es : 0;
        t.z.rows = s.rows;
        t.z.k = p.to;
        t.z.scale = a.scale;
        t.z.targets = a.targets;
        t.out = p.out;
        for (int64_t first = 0; first < s.classes; first += p.piece) {
            const int64_t here = std::min<int64_t>(s.classes - first, p.piece);
            t.z.first = (int)first;
            t.z.classes = (int)here;
            t.z.w = static_cast<const char*>(a.w) + first * s.wstride * s.es;
            Rows x = {}, w = {};
            if (p.xp != nullptr && first == 0) x = {a.x, s.xstride, s.rows, s.n, p.to, p.xp};
            if (p.wp != nullptr) {
                w = {t.z.w, s.wstride, here, s.n, p.to, p.wp};
                t.z.w = p.wp;
                t.z.wplane = p.terms ? here * p.to * es : 0;
            }
            KAN_TRY(pack<T>(p.terms, x, w, st));
            if (p.pz.splits > 0) {
                KAN_TRY(sums<T>(p.pz, t.z, p.z, st));
                const HeadRowsArgs r = {p.z, p.pz.splits, s.rows, s.classes, a.scale, a.targets,
                                        a.ignore, a.logp, a.stats, a.best};
                if (s.classes >= 512) head_rows_kernel<true><<<(int)s.rows, 256, 0, st>>>(r);
                else head_rows_kernel<false><<<(int)div_up(s.rows, 4), 256, 0, st>>>(r);
                return hipGetLastError();
            }
            KAN_TRY(by_tiles(t.z, mix_of(s.rows, here, s.n, es, p.terms).big,
                             [&](const LogitArgs& z, int64_t, bool big) {
                                 const HeadTileArgs part = {z, t.out, t.part};
                                 t.part += z.tp;
                                 return p.terms
                                            ? logit_tiles<uint16_t, kSegments>(part, a.best, big, st)
                                            : logit_tiles<T, 1>(part, a.best, big, st);
                             }));
        }
    }
    HeadJoinArgs j = {p.out, s.rows, (int)p.parts, s.classes, 1, a.targets, a.ignore, a.logp, a.stats,
                      a.best};
    while (j.lanes < 64 && div_up(s.rows, j.lanes) > 4 * kFillTiles) j.lanes *= 2;
    head_join_kernel<<<(int)div_up(s.rows, j.lanes), 256, 0, st>>>(j);
    return hipGetLastError();
}

struct HeadGradPlan {
    bool few, terms;
    int blocks, slices, each;  // few rows: column blocks, workgroups of each, classes of a wave
    int64_t piece, zstride;  // classes; elements
    int to;
    void *xp, *wp;           // packed rows, or null
    void* dz;
    int thin;                // groups of 16 rows whose dz are made in fp32 first, at z; or 0
    float *dx, *dw, *z;      // sums over k in parts, or null
    ProductPlan px, pw, pz;  // (pz.splits > 0: the logits')
    size_t bytes;
};

HeadGradPlan head_grad_plan(const HeadShape& s, bool dx, bool dw, void* ws) {
    HeadGradPlan p = {};
    Arena arena = {static_cast<char*>(ws)};
    // (16 rows of bf16: 326 us against the tiles' 240 at 1024 -> 131072, bound by the multiply-adds)
    p.few = s.rows <= (s.es == 2 ? kOuterRows / 2 : kOuterRows);
    if (p.few) {
        // (about 1024 workgroups, each wave at least 16 classes)
        p.blocks = (int)div_up(s.n, 256);
        const int64_t most = std::max<int64_t>(1, 4 * kFillTiles / p.blocks);
        p.each = (int)std::max<int64_t>(16, div_up(s.classes, most * kOuterWaves));
        p.slices = (int)div_up(s.classes, (int64_t)p.each * kOuterWaves);
        p.z = arena.take<float>((int64_t)s.classes * kOuterRows * 4);
        if (dx) p.dx = arena.take<float>((int64_t)p.slices * s.rows * s.n * 4);
        p.bytes = arena.at;
        return p;
    }
    p.terms = s.es == 4;  // (three products of each)
    p.to = (int)up(s.n, 8);
    const int64_t packed = (int64_t)p.to * (p.terms ? kTerms : 1) * 2;  // bytes of a row
    const int zes = (p.terms ? kDzTerms : 1) * 2;                       // and of a logit
    const bool wp = p.terms || !s.ws;
    // as few pieces as their dz (and packed weights) and launches allow, of one size
    const int64_t row = zes * s.rows + (wp ? packed : 0);
    int64_t most = std::min(kPieceClasses, kPieceTiles / div_up(s.rows, kSmall) * kSmall);
    most = std::min(most, std::max<int64_t>(kPieceBytes / row / kBig * kBig, kBig));
    p.piece = up(div_up(s.classes, div_up(s.classes, most)), kBig);
    p.zstride = std::min(p.piece, up(s.classes, 64));
    const int64_t here = std::min<int64_t>(p.piece, s.classes);
    // (a copy without what ignored rows hold: 0 times it need not be 0)
    if (p.terms || !s.xs || dw) p.xp = arena.take(s.rows * packed);
    // (weights read once in fp32, not six times as terms: 22 x 1004 -> 44307 149 us, so
    // 70 and 5; their terms are dx's alone then)
    if (p.terms && s.rows <= kThinMost) p.thin = (int)div_up(s.rows, 16);
    if (wp && (dx || p.thin == 0)) p.wp = arena.take(p.piece * packed);
    p.dz = arena.take(s.rows * p.zstride * zes);
    if (p.thin > 0) {
        p.z = arena.take<float>(p.piece * p.thin * 16 * 4);
    } else if (p.piece >= s.classes) {
        p.pz = sums_plan(s.rows, s.classes, s.n, p.terms);
    }
    if (p.pz.splits > 0) p.z = arena.take<float>((int64_t)p.pz.splits * s.rows * s.classes * 4);
    if (dx) {
        p.px = product_plan(s.n, s.rows, p.zstride, p.terms);
        if (p.px.splits > 1 || p.piece < s.classes)
            p.dx = arena.take<float>((int64_t)p.px.splits * s.rows * s.n * 4);
    }
    if (dw) {
        p.pw = product_plan(s.n, here, s.rows, p.terms);
        if (p.pw.splits > 1) p.dw = arena.take<float>((int64_t)p.pw.splits * here * s.n * 4);
    }
    p.bytes = arena.at;
    return p;
}

template <typename O>
hipError_t gradient_tiles(const HeadGradTileArgs& g, bool big, hipStream_t st) {
    constexpr bool TERMS = sizeof(O) == 4;
    typedef BigLogits<uint16_t, TERMS ? kSegments : 1> Big;
    typedef SmallLogits<uint16_t, TERMS ? kSegments : 1> Small;
    const int groups = resident(g.z.tp * g.z.tq, big);
    if (big) head_grad_kernel<Big, TERMS><<<groups, Big::THREADS, 0, st>>>(g);
    else head_grad_kernel<Small, TERMS><<<groups, Small::THREADS, 0, st>>>(g);
    return hipGetLastError();
}

// (many parts of few values go over 16 lanes a value: 62 parts of 1442 values 37 us in one lane each; 15
// of a million 26 us, so 10)
template <typename T>
hipError_t sum(const float* acc, int splits, int64_t n, float scale, void* out, hipStream_t st) {
    if (splits >= 12 && n < kFillTiles * 1024)
        head_gather_kernel<T><<<grid_of(n, 16), 256, 0, st>>>(acc, splits, n, scale,
                                                              static_cast<T*>(out));
    else
        head_sum_kernel<T><<<grid_of(n, 1024), 256, 0, st>>>(acc, splits, n, scale,
                                                             static_cast<T*>(out));
    return hipGetLastError();
}

template <typename T>
hipError_t head_grad_few(const HeadShape& s, const HeadGradArgs& a, const HeadGradPlan& p,
                         hipStream_t st) {
    HeadGradTileArgs g = {};
    g.z.rows = s.rows;
    g.z.targets = a.targets;
    g.stats = a.stats;
    g.dlogp = a.dlogp;
    g.ignore = a.ignore;
    g.all = s.classes;
    KAN_TRY(thin<T, 1, kDz>(s, thin_args(s, a.x, a.w, a.scale, a.targets), g, p.z, st));
    const HeadOuterArgs o = {a.x, a.w, p.z, s.xstride, s.wstride, (int)s.rows, s.classes, s.n, p.each,
                             a.targets, a.ignore, a.scale, p.dx, a.dw};
    auto kernel = s.rows <= 4 ? head_outer_kernel<T, 4> : head_outer_kernel<T, 8>;
    if constexpr (sizeof(T) == 4)
        if (s.rows > 8) kernel = head_outer_kernel<T, kOuterRows>;
    kernel<<<p.blocks * p.slices, 64 * kOuterWaves, 0, st>>>(o, p.blocks);
    KAN_TRY(hipGetLastError());
    if (p.dx == nullptr) return hipSuccess;
    return sum<T>(p.dx, p.slices, s.rows * s.n, a.scale, a.dx, st);
}

template <typename T>
hipError_t head_grad(const HeadShape& s, const HeadGradArgs& a, void* ws, hipStream_t st) {
    if (s.rows == 0) {
        if (a.dw == nullptr) return hipSuccess;
        const int64_t n = (int64_t)s.classes * s.n;
        head_zero_kernel<T><<<grid_of(n, 256), 256, 0, st>>>(static_cast<T*>(a.dw), n);
        return hipGetLastError();
    }
    const HeadGradPlan p = head_grad_plan(s, a.dx != nullptr, a.dw != nullptr, ws);
    if (p.few) return head_grad_few<T>(s, a, p, st);
    const bool terms = p.terms;
    const int es = 2;  // bytes of an operand's element
    HeadGradTileArgs g = {};
    g.z.x = p.xp != nullptr ? p.xp : a.x;
    g.z.xstride = (p.xp != nullptr ? p.to : s.xstride) * es;
    g.z.wstride = (p.wp != nullptr ? p.to : s.wstride) * es;
    g.z.xplane = terms ? s.rows * p.to * es : 0;
    g.z.rows = s.rows;
    g.z.k = p.to;
    g.z.scale = a.scale;
    g.z.targets = a.targets;
    g.stats = a.stats;
    g.dlogp = a.dlogp;
    g.ignore = a.ignore;
    g.all = s.classes;
    g.dz = p.dz;
    g.zstride = p.zstride;
    g.zplane = s.rows * p.zstride;
    const int64_t zbytes = p.zstride * es;
    for (int64_t first = 0; first < s.classes; first += p.piece) {
        const int64_t here = std::min<int64_t>(s.classes - first, p.piece);
        g.z.w = static_cast<const char*>(a.w) + first * s.wstride * s.es;
        g.z.first = (int)first;
        g.z.classes = (int)here;
        Rows x = {}, w = {};
        if (p.xp != nullptr && first == 0)
            x = {a.x, s.xstride, s.rows, s.n, p.to, p.xp, a.targets, a.ignore};
        if (p.wp != nullptr) {
            w = {g.z.w, s.wstride, here, s.n, p.to, p.wp};
            g.z.w = p.wp;
            g.z.wplane = terms ? here * p.to * es : 0;
        }
        KAN_TRY(pack<T>(terms, x, w, st));
        if (p.thin > 0) {
            if constexpr (sizeof(T) == 4) {
                HeadShape part = s;
                part.classes = (int)here;
                const HeadThinArgs t =
                    thin_args(part, a.x, static_cast<const char*>(a.w) + first * s.wstride * s.es,
                              a.scale, a.targets);
                KAN_TRY(p.thin == 2   ? thin<T, 2, kDz>(part, t, g, p.z, st)
                        : p.thin == 3 ? thin<T, 3, kDz>(part, t, g, p.z, st)
                                      : thin<T, 4, kDz>(part, t, g, p.z, st));
                head_turn_kernel<<<grid_of(p.zstride / 8 * p.thin * 16, 256), 256, 0, st>>>(
                    g, p.z, p.thin * 16);
                KAN_TRY(hipGetLastError());
            }
        } else if (p.pz.splits > 0) {
            KAN_TRY(sums<T>(p.pz, g.z, p.z, st));
            head_dz_kernel<sizeof(T) == 4>
                <<<grid_of(s.rows * (p.zstride / 8), 256), 256, 0, st>>>(g, p.z, p.pz.splits);
            KAN_TRY(hipGetLastError());
        } else {
            KAN_TRY(by_tiles(g.z, mix_of(s.rows, here, s.n, es, terms).big,
                             [&](const LogitArgs& z, int64_t from, bool big) {
                                 HeadGradTileArgs part = g;
                                 part.z = z;
                                 part.dz = static_cast<uint16_t*>(p.dz) + from;
                                 part.zwidth = p.zstride - from;
                                 return gradient_tiles<T>(part, big, st);
                             }));
        }
        ProductArgs r = {};
        r.q = p.dz;
        r.qstride = zbytes;
        r.qplane = terms ? g.zplane * es : 0;
        r.qterms = kTermsDz;
        r.np = s.n;
        r.scale = a.scale;
        if (a.dx != nullptr) {
            const bool last = first + p.piece >= s.classes, whole = p.px.splits == 1 && last;
            r.p = g.z.w;
            r.pstride = g.z.wstride;
            r.pplane = g.z.wplane;
            r.nq = s.rows;
            r.k = up(here, 16 / es);  // (whole chunks of dz's rows, which are 0 past the classes)
            r.pk = here;
            r.acc = p.dx;
            r.add = first > 0;
            r.out = whole ? a.dx : nullptr;
            KAN_TRY(product<T, kByK, kByRows>(p.px, r, st));
            if (last && !whole)
                KAN_TRY(sum<T>(p.dx, p.px.splits, s.rows * s.n, a.scale, a.dx, st));
        }
        if (a.dw != nullptr) {
            char* const out = static_cast<char*>(a.dw) + first * s.n * s.es;
            r.p = p.xp;
            r.pstride = g.z.xstride;
            r.pplane = g.z.xplane;
            r.nq = here;
            r.k = r.pk = r.qk = s.rows;
            r.acc = p.dw;
            r.add = false;
            r.out = p.pw.splits == 1 ? out : nullptr;
            KAN_TRY(product<T, kByK, kByK>(p.pw, r, st));
            if (p.pw.splits > 1) KAN_TRY(sum<T>(p.dw, p.pw.splits, here * s.n, a.scale, out, st));
        }
    }
    return hipSuccess;
}

}  // namespace

size_t head_workspace(const HeadShape& s) {
    return s.rows == 0 ? 0 : head_plan(s, nullptr).bytes;
}
size_t head_grad_workspace(const HeadShape& s, bool dx, bool dw) {
    return s.rows == 0 ? 0 : head_grad_plan(s, dx, dw, nullptr).bytes;
}
hipError_t launch_head(const HeadShape& s, const HeadArgs& a, void* ws, hipStream_t st) {
    return s.es == 2 ? head<uint16_t>(s, a, ws, st) : head<float>(s, a, ws, st);
}
hipError_t launch_head_grad(const HeadShape& s, const HeadGradArgs& a, void* ws, hipStream_t st) {
    return s.es == 2 ? head_grad<uint16_t>(s, a, ws, st) : head_grad<float>(s, a, ws, st);
}

}  // namespace kan
