// kan_norm.hip -- layer norm over the last dimension, with the residual sum before it,
// and its gradient.
//
//   h = x (+ r),  mu = mean_i h,  rstd = 1 / sqrt(mean_i (h - mu)^2 + eps),
//   y = (h - mu) rstd w + b
//   xh = (h - mu) rstd,  g = dy w,
//   dx = rstd (g - mean_i g - xh mean_i(g xh)) (+ dh),
//   dw = sum_rows dy xh,  db = sum_rows dy
//
// Both are bound by HBM: about ten operations per element moved.  A row stays in the
// registers of the lanes that share it, so it is read once, and its variance is the mean
// of squared differences from a mean that is corrected by the mean difference (no
// cancellation, and no rounding of the sum, where the centre is far from 0).  Rows up to 32
// 16-byte units share a wave with others; up to 1024 elements a wave takes a row; above,
// as many waves as give each lane 16 elements (32 from 8193 on), which join their sums through
// LDS; above kNormRegRow elements a row no longer fits and is read again for each step (from
// L2).  The weight gradients are summed in registers over all rows that a workgroup takes (its
// lanes keep their columns from row to row), joined over the workgroup through LDS, written
// once per workgroup and summed in a fixed order by a second launch (a single workgroup
// writes the gradients): deterministic, no atomics.
// All sums and statistics are fp32; y, h and dx are rounded once, when stored (y from the
// sum x + r before its rounding to h).
//
// Measured on MI355X: forward 65536 x 784 bf16 43.7 us (4.7 TB/s), 16384 x 8192 bf16 with the
// residual 198 us (5.4 TB/s); gradient 16384 x 8192 bf16 with dh 216 us (5.0 TB/s), 30001 x 1001
// bf16 with dh 50.9 us (4.7 TB/s), 16384 x 256 fp32 15.5-16.4 us (3.1-3.3 TB/s, both launches,
// outputs at hand).  fp32: forward 65536 x 784 80 us, 16384 x 12288 321 us (5.1 and 5.0 TB/s),
// gradient 16384 x 8192 307 us (5.3 TB/s), but 16384 x 12288 661 us (3.7 TB/s): above 8192 columns
// its 32 elements per lane spill 74 registers.  Rows that are read again: 16384 x 20000 forward
// 1326 us in fp32 and 1109 in bf16 (2.0 and 1.2 TB/s of the bytes that have to move), 8192 x 20000
// fp32 gradient 1376 us (1.4 TB/s): they load one element per lane.  Loads of the next row ahead
// of time did not help where they were tried, at two units per lane (30001 x 1001: 58.9 us against
// 52.3): the other waves hide them, and the registers cost some of those.
#include "kan_ops.h"
#include "kan_rows.h"

namespace kan {

namespace {

constexpr int kMaxWaves = 8;

// How a workgroup takes rows.
enum Mode {
    kShared,  // 64 >> shift rows in each wave, one unit per lane (32 lanes a row at most)
    kWave,    // a row in each wave (33 units or more)
    kGroup,   // a.waves waves a row, as many rows as eight waves take
};

// Where a lane works.
template <int M>
struct Place {
    int lane, wave;
    int first, waves;  // kGroup: the waves of the row
    int lanes;         // lanes that share a row, within the wave
    int slot;          // this lane's place among all lanes of the row
    int stride;        // lanes of the row, over all waves
    int rows;          // rows a workgroup takes at a time
    int sub;           // this lane's row among them
    __device__ __forceinline__ Place(int shift, int waves_) : waves(waves_) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lanes = M == kShared ? 1 << shift : 64;
        if (M == kGroup) {
            rows = (int)(blockDim.x >> 6) / waves;
            sub = wave / waves;
        } else {
            rows = M == kShared ? (int)blockDim.x >> shift : (int)blockDim.x >> 6;
            sub = M == kShared ? (int)threadIdx.x >> shift : wave;
        }
        first = M == kGroup ? sub * waves : 0;
        stride = M == kGroup ? 64 * waves : lanes;
        slot = M == kShared ? lane & (lanes - 1)
               : M == kWave ? lane
                            : (wave - first) * 64 + lane;
    }

    // Sums over the lanes of a row (all lanes of the workgroup call).  kGroup: `red` is a
    // buffer that no wave still reads (the callers alternate two).
    __device__ __forceinline__ void sum(float& a, float& b, float (*red)[2]) const {
        if (M == kShared) {
            a = group_sum(a, lanes);
            b = group_sum(b, lanes);
            return;
        }
        a = wave_sum(a);
        b = wave_sum(b);
        if (M == kWave) return;
        if (lane == 0) {
            red[wave][0] = a;
            red[wave][1] = b;
        }
        __syncthreads();
        a = b = 0.0f;
        for (int w = 0; w < waves; ++w) {
            a += red[first + w][0];
            b += red[first + w][1];
        }
    }
};

// The variance from the mean square q around a rounded mean that is e off: q - e^2, which
// takes away next to nothing (and never all but rounding: e is a rounding of the mean).  A q
// past fp32 stays infinite: rstd is 0.
__device__ __forceinline__ float spread(float q, float e) {
    return q == __builtin_huge_valf() ? q : q - __builtin_fminf(e * e, q);
}

// (one unit in the last place; the bare instruction takes a subnormal v, as rows of little
// spread have without eps, for 0)
__device__ __forceinline__ float inverse_root(float v) { return rsqrtf(v); }

template <int N>
__device__ __forceinline__ void clear_units(u32x4 (&raw)[N]) {
#pragma unroll
    for (int u = 0; u < N; ++u) raw[u] = u32x4{0u, 0u, 0u, 0u};
}

template <int M> constexpr int kThreads = M == kGroup ? 64 * kMaxWaves : 256;
constexpr int kGradThreads = 64 * kMaxWaves;

// C units per lane, of which the first FC are full in every lane.
template <typename T, typename TP, int M, int C, int FC>
__global__ void __launch_bounds__(kThreads<M>) norm_kernel(NormArgs a) {
#pragma clang fp contract(off)  // (differences are from the rounded mean: exact near it)
    constexpr int V = kVec<T>;
    constexpr bool kSub = M == kShared;
    __shared__ float red[2][kMaxWaves][2];
    const Place<M> p(a.shift, a.waves);
    const int n = a.n, col0 = p.slot * V, step = p.stride * V;
    const float inv_n = 1.0f / (float)n;
    float w[C][V], b[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_params<kSub>(static_cast<const TP*>(a.w), col0 + c * step, n, 1.0f, w[c]);
        load_params<kSub>(static_cast<const TP*>(a.b), col0 + c * step, n, 0.0f, b[c]);
    }
    for (int64_t r0 = (int64_t)blockIdx.x * p.rows; r0 < a.rows;
         r0 += (int64_t)gridDim.x * p.rows) {
        const int64_t row = r0 + p.sub;
        if (M == kWave && row >= a.rows) break;
        // (past the last row nothing is stored; the first row's values stand in)
        const bool live = M == kWave || row < a.rows;
        const int nl = live ? n : 0;
        const int64_t at = live ? row * n : 0;
        float v[C][V];
        u32x4 rx[C], rr[C];
        issue_units<FC, kSub>(static_cast<const T*>(a.x) + at, col0, step, n, 0u, rx);
        if (a.res != nullptr)
            issue_units<FC, kSub>(static_cast<const T*>(a.res) + at, col0, step, n, 0u, rr);
        else
            clear_units(rr);
        settle_units<FC, kSub, T>(col0, step, n, 0u, rx);
        settle_units<FC, kSub, T>(col0, step, n, 0u, rr);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float r[V];
            widen(rx[c], v[c]);
            widen(rr[c], r);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] += r[i];
        }
        if (a.h != nullptr && live) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (c < FC) store_unit<true>(static_cast<T*>(a.h) + at, col0 + c * step, n, v[c]);
                else store_unit<false>(static_cast<T*>(a.h) + at, col0 + c * step, n, v[c]);
            }
        }
        float s = 0.0f, q = 0.0f, e = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) s += v[c][i];
        p.sum(s, e, red[0]);
        const float mu = s * inv_n;
        e = 0.0f;
        StaticFor<0, C>::run([&](auto c) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = (c < FC) || col0 + c * step + i < n ? v[c][i] - mu : 0.0f;
                v[c][i] = d;
                e += d;
                q = __builtin_fmaf(d, d, q);
            }
        });
        p.sum(q, e, red[1]);
        // what the rounding of the sum left out of the mean (e / n, its rounding taken back once:
        // it is all that y keeps of a constant row)
        const float e0 = e * inv_n;
        e = __builtin_fmaf(__builtin_fmaf(-e0, (float)n, e), inv_n, e0);
        const float rstd = inverse_root(spread(q * inv_n, e) + a.eps);
        if (a.mean != nullptr && live && p.slot == 0) {
            a.mean[row] = mu + e;
            a.rstd[row] = rstd;
        }
        StaticFor<0, C>::run([&](auto c) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                v[c][i] = __builtin_fmaf((v[c][i] - e) * rstd, w[c][i], b[c][i]);
            if (M == kGroup && !live) return;
            store_unit<(c < FC) && M != kShared>(static_cast<T*>(a.y) + at, col0 + c * step, nl,
                                                 v[c]);
        });
    }
}

// Rows that do not fit in registers: one workgroup per row, read three times.
template <typename T, typename TP>
__global__ void __launch_bounds__(512) norm_long_kernel(NormArgs a) {
#pragma clang fp contract(off)
    __shared__ float red[2][kMaxWaves][2];
    const Place<kGroup> p(0, 8);
    const int n = a.n;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * n;
        const T* res = a.res ? static_cast<const T*>(a.res) + row * n : nullptr;
        auto value = [&](int i) {
            return Storage<T>::load(x + i) + (res ? Storage<T>::load(res + i) : 0.0f);
        };
        float s = 0.0f, q = 0.0f, e = 0.0f;
        for (int i = threadIdx.x; i < n; i += 512) s += value(i);
        p.sum(s, e, red[0]);
        const float mu = s / (float)n;
        e = 0.0f;
        for (int i = threadIdx.x; i < n; i += 512) {
            const float d = value(i) - mu;
            e += d;
            q = __builtin_fmaf(d, d, q);
        }
        p.sum(q, e, red[1]);
        e /= (float)n;
        const float rstd = inverse_root(spread(q / (float)n, e) + a.eps);
        if (a.mean != nullptr && threadIdx.x == 0) {
            a.mean[row] = mu + e;
            a.rstd[row] = rstd;
        }
        for (int i = threadIdx.x; i < n; i += 512) {
            const float v = value(i);
            if (a.h != nullptr) Storage<T>::store(static_cast<T*>(a.h) + row * n + i, v);
            const float w = a.w ? Storage<TP>::load(static_cast<const TP*>(a.w) + i) : 1.0f;
            const float b = a.b ? Storage<TP>::load(static_cast<const TP*>(a.b) + i) : 0.0f;
            Storage<T>::store(static_cast<T*>(a.y) + row * n + i,
                              __builtin_fmaf((v - mu - e) * rstd, w, b));
        }
    }
}

// What a row's gradient reads.
template <typename T, int C>
struct GradRow {
    u32x4 h[C], dy[C], dh[C];
    float mu, rstd;
    template <int FC, bool TINY>
    __device__ __forceinline__ void issue(const NormGradArgs& a, int64_t row, int col0, int step) {
        const int64_t at = row * a.n;
        issue_units<FC, TINY>(static_cast<const T*>(a.h) + at, col0, step, a.n, 0u, h);
        issue_units<FC, TINY>(static_cast<const T*>(a.dy) + at, col0, step, a.n, 0u, dy);
        if (a.dh != nullptr)
            issue_units<FC, TINY>(static_cast<const T*>(a.dh) + at, col0, step, a.n, 0u, dh);
        else
            clear_units(dh);
        mu = a.mean[row];
        rstd = a.rstd[row];
    }
    // What stands in for a row past the last one adds nothing to the sums.
    __device__ __forceinline__ void keep(bool live) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[c][i] = live ? h[c][i] : 0u;
                dy[c][i] = live ? dy[c][i] : 0u;
            }
        mu = live ? mu : 0.0f;
        rstd = live ? rstd : 0.0f;
    }
};

template <typename T, typename TP, int M, int C, int FC>
__global__ void __launch_bounds__(kGradThreads) norm_grad_kernel(NormGradArgs a) {
    constexpr int V = kVec<T>;
    constexpr bool kSub = M == kShared;
    __shared__ float red[2][kMaxWaves][2];
    extern __shared__ __attribute__((aligned(16))) float join[];  // where a workgroup takes several rows
    const Place<M> p(a.shift, a.waves);
    const int n = a.n, col0 = p.slot * V, step = p.stride * V;
    const float inv_n = 1.0f / (float)n;
    float w[C][V], dw[C][V], db[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_params<kSub>(static_cast<const TP*>(a.w), col0 + c * step, n, 1.0f, w[c]);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[c][i] = db[c][i] = 0.0f;
    }
    const int64_t stride = (int64_t)gridDim.x * p.rows;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * p.rows; r0 < a.rows; r0 += stride, turn ^= 1) {
        const int64_t row = r0 + p.sub;
        if (M == kWave && row >= a.rows) break;
        const bool live = M == kWave || row < a.rows;
        GradRow<T, C> cur;
        cur.template issue<FC, kSub>(a, live ? row : 0, col0, step);
        settle_units<FC, kSub, T>(col0, step, n, 0u, cur.h);
        settle_units<FC, kSub, T>(col0, step, n, 0u, cur.dy);
        if (M != kWave) cur.keep(live);
        const float mu = cur.mu, rstd = cur.rstd;
        float s1 = 0.0f, s2 = 0.0f;
        // (past the row's end dy is 0, and with it all that is summed)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float h[V], dy[V];
            widen(cur.h[c], h);
            widen(cur.dy[c], dy);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (h[i] - mu) * rstd;
                const float g = dy[i] * w[c][i];
                dw[c][i] = __builtin_fmaf(dy[i], xh, dw[c][i]);
                db[c][i] += dy[i];
                s1 += g;
                s2 = __builtin_fmaf(g, xh, s2);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        p.sum(s1, s2, red[turn]);
        s1 *= inv_n;
        s2 *= inv_n;
        settle_units<FC, kSub, T>(col0, step, n, 0u, cur.dh);
        // xh and g are formed again from the 16-byte units, which take half or less of the
        // registers that they would take as fp32
#pragma unroll
        for (int c = 0; c < C; ++c) {
            asm volatile("" : "+v"(cur.h[c]), "+v"(cur.dy[c]), "+v"(cur.dh[c]));
            float h[V], dy[V], d[V];
            widen(cur.h[c], h);
            widen(cur.dy[c], dy);
            widen(cur.dh[c], d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (h[i] - mu) * rstd, g = dy[i] * w[c][i];
                d[i] = __builtin_fmaf(rstd, g - s1 - xh * s2, d[i]);
            }
            if (a.dx != nullptr && live) {
                T* dx = static_cast<T*>(a.dx) + row * n;
                if (c < FC) store_unit<true>(dx, col0 + c * step, n, d);
                else store_unit<false>(dx, col0 + c * step, n, d);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (a.dw == nullptr && a.db == nullptr) return;
    // This workgroup's sums, [2][workgroups][n] (or, of a single one, the gradients): over the
    // rows of a wave by lanes, over the rows of the workgroup through LDS, [rows][columns of
    // the lanes].
    const int rows = M == kGroup ? p.rows : kMaxWaves, mine = M == kGroup ? p.sub : p.wave;
    const int span = C * step;
    for (int k = 0; k < 2; ++k) {
        float(&acc)[C][V] = k == 0 ? dw : db;
        float* part = a.part + ((int64_t)k * gridDim.x + blockIdx.x) * n;
        TP* grad = static_cast<TP*>(k == 0 ? a.dw : a.db);
        const bool direct = a.part == nullptr;
        if (direct && grad == nullptr) continue;
        if (M == kShared)
            for (int o = p.lanes; o < 64; o *= 2)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[0][i] += __shfl_xor(acc[0][i], o);
        if (rows == 1 && !direct) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const float u[4] = {acc[c][i], acc[c][i + 1], acc[c][i + 2], acc[c][i + 3]};
                    store_unit<false>(part, col0 + c * step + i, n, u);
                }
            continue;
        }
        if (rows == 1) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (col0 + c * step + i < n)
                        Storage<TP>::store(grad + col0 + c * step + i, acc[c][i]);
            continue;
        }
        if (k == 1) __syncthreads();
        if (p.lane < p.lanes) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < V; i += 4)
                    *reinterpret_cast<floatx4*>(join + mine * span + col0 + c * step + i) =
                        floatx4{acc[c][i], acc[c][i + 1], acc[c][i + 2], acc[c][i + 3]};
        }
        __syncthreads();
        for (int j = threadIdx.x; j < n; j += blockDim.x) {
            float t = join[j];
            for (int r = 1; r < rows; ++r) t += join[r * span + j];
            if (direct) Storage<TP>::store(grad + j, t);
            else part[j] = t;
        }
    }
}

// dx of rows that do not fit in registers: one workgroup per row, read twice.
template <typename T, typename TP>
__global__ void __launch_bounds__(512) norm_grad_long_kernel(NormGradArgs a) {
    __shared__ float red[2][kMaxWaves][2];
    const Place<kGroup> p(0, 8);
    const int n = a.n;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const T* h = static_cast<const T*>(a.h) + row * n;
        const T* dy = static_cast<const T*>(a.dy) + row * n;
        const float mu = a.mean[row], rstd = a.rstd[row];
        auto grad = [&](int i) {
            const float w = a.w ? Storage<TP>::load(static_cast<const TP*>(a.w) + i) : 1.0f;
            return Storage<T>::load(dy + i) * w;
        };
        float s1 = 0.0f, s2 = 0.0f;
        for (int i = threadIdx.x; i < n; i += 512) {
            const float g = grad(i);
            s1 += g;
            s2 = __builtin_fmaf(g, (Storage<T>::load(h + i) - mu) * rstd, s2);
        }
        p.sum(s1, s2, red[turn]);
        s1 /= (float)n;
        s2 /= (float)n;
        for (int i = threadIdx.x; i < n; i += 512) {
            const float xh = (Storage<T>::load(h + i) - mu) * rstd;
            const float d =
                a.dh ? Storage<T>::load(static_cast<const T*>(a.dh) + row * n + i) : 0.0f;
            Storage<T>::store(static_cast<T*>(a.dx) + row * n + i,
                              __builtin_fmaf(rstd, grad(i) - s1 - xh * s2, d));
        }
    }
}

// Partial weight gradients of the same rows: a lane per column, the rows split over
// gridDim.y.
template <typename T, typename TP>
__global__ void __launch_bounds__(256) norm_grad_columns_kernel(NormGradArgs a) {
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (col >= a.n) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float dy = Storage<T>::load(static_cast<const T*>(a.dy) + row * a.n + col);
        const float xh =
            (Storage<T>::load(static_cast<const T*>(a.h) + row * a.n + col) - a.mean[row]) *
            a.rstd[row];
        dw = __builtin_fmaf(dy, xh, dw);
        db += dy;
    }
    if (a.part == nullptr) {
        if (a.dw != nullptr) Storage<TP>::store(static_cast<TP*>(a.dw) + col, dw);
        if (a.db != nullptr) Storage<TP>::store(static_cast<TP*>(a.db) + col, db);
        return;
    }
    a.part[(int64_t)blockIdx.y * a.n + col] = dw;
    a.part[((int64_t)gridDim.y + blockIdx.y) * a.n + col] = db;
}

// dw (blockIdx.y 0) and db (1) from the workgroups' sums, in a fixed order: 16 columns
// per workgroup, 64 lanes of each column over the parts, eight loads in flight.
template <typename TP>
__global__ void __launch_bounds__(1024) norm_params_kernel(const float* part, int parts, int n,
                                                           TP* dw, TP* db) {
    __shared__ float sums[16][65];
    TP* out = blockIdx.y == 0 ? dw : db;
    if (out == nullptr) return;
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int col = blockIdx.x * 16 + c;
    const float* src = part + (int64_t)blockIdx.y * parts * n;
    float s = 0.0f, t[8] = {};
    if (col < n) {
        int k = g;
        for (; k + 7 * 64 < parts; k += 8 * 64)
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] += src[(int64_t)(k + j * 64) * n + col];
        for (; k < parts; k += 64) s += src[(int64_t)k * n + col];
    }
    s += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
    sums[c][g] = s;
    __syncthreads();
    // (a wave adds one column)
    const int wave = threadIdx.x >> 6;
    s = wave_sum(sums[wave][threadIdx.x & 63]);
    if ((threadIdx.x & 63) == 0 && blockIdx.x * 16 + wave < n)
        Storage<TP>::store(out + blockIdx.x * 16 + wave, s);
}

constexpr int kLongParts = 64;

}  // namespace

NormPlan norm_plan(int64_t rows, int32_t n, int es, bool grad) {
    NormPlan p = {};
    const int V = 16 / es;
    int64_t per = 1, most = 2048;
    p.threads = 512;
    if (n > kNormRegRow) {
        p.waves = 0;
    } else if (n <= 1024) {
        p.waves = 1;
        p.threads = grad ? kGradThreads : 256;
        while (V << p.shift < n && p.shift < 6) ++p.shift;
        per = p.threads >> p.shift;
        p.units = p.shift < 6 || n <= 64 * V ? 1 : (n <= 512 ? 8 : 16) / V;
    } else {
        // 16 elements per lane, 32 where eight waves need them
        p.units = (n <= 8192 ? 16 : 32) / V;
        p.waves = (n + 64 * V * p.units - 1) / (64 * V * p.units);
        per = 8 / p.waves;
        p.threads = (int)(64 * p.waves * per);
    }
    // Workgroups of the gradient: each leaves a row of partial sums, so no more than keep the
    // memory busy, of eight waves (with the joining launch: 16384 x 256 fp32 512 workgroups
    // 15.9 us, 768 17.4; 16384 x 1024 fp32 256 42.6 us, 384 44.8, 512 45.4).
    if (grad) most = p.units == 1 ? 512 : p.waves == 1 ? 256 : n <= 8192 ? 512 : 256;
    // (the weight gradients' join: the columns of all lanes of the workgroup's waves that take
    // different rows)
    if (grad && per > 1 && p.waves > 0)
        p.lds = sizeof(float) * p.units * V *
                (p.waves > 1 || p.units > 1 ? p.threads : kMaxWaves << p.shift);
    // (few rows: one workgroup, whose sums are the gradients: 16 x 784 bf16 11-12 us against
    // 15.4 with the joining launch)
    if (grad && rows <= 3 * per && p.waves > 0) most = 1;
    const int64_t need = (rows + per - 1) / per;
    p.blocks = (int)(need < most ? need : most);
    p.parts = p.waves == 0 ? (int)(rows < kLongParts ? rows : kLongParts) : p.blocks;
    return p;
}

namespace {

// f(integral constants M, C, FC) for a plan's kernel.  At more than one unit per lane a row
// has more than half of the lanes' columns (whole waves share it): the first half of the
// units is full.
template <typename T, typename F>
void norm_dispatch(const NormPlan& p, F&& f) {
    constexpr int V = kVec<T>;
    auto go = [&](auto mode, auto units) {
        constexpr int C = decltype(units)::value;
        f(mode, units, std::integral_constant<int, C / 2>{});
    };
    using std::integral_constant;
    if (p.shift < 6 && p.waves == 1)
        go(integral_constant<int, kShared>{}, integral_constant<int, 1>{});
    else if (p.units == 1)
        go(integral_constant<int, kWave>{}, integral_constant<int, 1>{});
    else if (p.waves > 1 && p.units == 32 / V)
        go(integral_constant<int, kGroup>{}, integral_constant<int, 32 / V>{});
    else if (p.waves > 1)
        go(integral_constant<int, kGroup>{}, integral_constant<int, 16 / V>{});
    else if (p.units == 16 / V)
        go(integral_constant<int, kWave>{}, integral_constant<int, 16 / V>{});
    else if constexpr (V == 4)
        go(integral_constant<int, kWave>{}, integral_constant<int, 2>{});
}

template <typename T, typename TP>
hipError_t norm_forward(const NormPlan& p, const NormArgs& a, hipStream_t s) {
    if (p.waves == 0) {
        norm_long_kernel<T, TP><<<p.blocks, 512, 0, s>>>(a);
        return hipGetLastError();
    }
    norm_dispatch<T>(p, [&](auto m, auto c, auto fc) {
        norm_kernel<T, TP, decltype(m)::value, decltype(c)::value, decltype(fc)::value>
            <<<p.blocks, p.threads, 0, s>>>(a);
    });
    return hipGetLastError();
}

template <typename T, typename TP>
hipError_t norm_backward(const NormPlan& p, const NormGradArgs& a, hipStream_t s) {
    hipError_t e = hipSuccess;
    const bool params = a.dw != nullptr || a.db != nullptr;
    if (a.rows > 0 && p.waves == 0) {
        if (a.dx != nullptr) {
            norm_grad_long_kernel<T, TP><<<p.blocks, 512, 0, s>>>(a);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (params)
            norm_grad_columns_kernel<T, TP><<<dim3((a.n + 255) / 256, p.parts), 256, 0, s>>>(a);
    } else if (a.rows > 0) {
        norm_dispatch<T>(p, [&](auto m, auto c, auto fc) {
            norm_grad_kernel<T, TP, decltype(m)::value, decltype(c)::value, decltype(fc)::value>
                <<<p.blocks, p.threads, p.lds, s>>>(a);
        });
    }
    if ((e = hipGetLastError()) != hipSuccess || !params || p.parts == 1) return e;
    // (without rows there are no parts: 0)
    norm_params_kernel<TP><<<dim3((a.n + 15) / 16, 2), 1024, 0, s>>>(
        a.part, p.parts, a.n, static_cast<TP*>(a.dw), static_cast<TP*>(a.db));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(bool bf16, bool bf16_params, const NormPlan& p, NormArgs a, hipStream_t s) {
    a.shift = p.shift;
    a.waves = p.waves;
    if (!bf16) return norm_forward<float, float>(p, a, s);
    if (bf16_params) return norm_forward<uint16_t, uint16_t>(p, a, s);
    return norm_forward<uint16_t, float>(p, a, s);
}

hipError_t launch_norm_grad(bool bf16, bool bf16_params, const NormPlan& p, NormGradArgs a,
                            hipStream_t s) {
    a.shift = p.shift;
    a.waves = p.waves;
    if (!bf16) return norm_backward<float, float>(p, a, s);
    if (bf16_params) return norm_backward<uint16_t, uint16_t>(p, a, s);
    return norm_backward<uint16_t, float>(p, a, s);
}

}  // namespace kan
