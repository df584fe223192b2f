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
// cancellation, and no rounding of the sum, where the centre is far from 0).  Rows up to one
// 16-byte unit per lane share a wave with others; up to 32 elements per lane one wave
// takes a row; above, four or eight waves take it and join their sums through LDS; above
// kNormRegRow elements a row no longer fits and is read again for each step (from L2).
// The weight gradients are summed in registers over all rows that a workgroup takes (its
// lanes keep their columns from row to row), written once per workgroup and summed in a
// fixed order by a second launch: deterministic, no atomics.
// All sums and statistics are fp32; y, h and dx are rounded once, when stored (y from the
// sum x + r before its rounding to h).
#include "kan_internal.h"
#include "kan_rows.h"

namespace kan {

namespace {

// Sums a and b over the W waves of a workgroup (all waves call; `red` is a buffer that
// no wave still reads: the callers alternate two).
template <int W>
__device__ __forceinline__ void wave_join(float& a, float& b, float (*red)[2], int wave, int lane) {
    if (W == 1) return;
    if (lane == 0) {
        red[wave][0] = a;
        red[wave][1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        a += red[w][0];
        b += red[w][1];
    }
}

// The variance from the mean square q around a rounded mean that is e off: q - e^2, which
// takes away next to nothing (and never all but rounding: e is a rounding of the mean).
__device__ __forceinline__ float spread(float q, float e) {
    return q - __builtin_fminf(e * e, q);
}

// Where a lane works.  W waves take a row (W = 1: each wave of the four its own row, or,
// with one unit per lane, 64 >> shift rows).
template <int W, int C>
struct Place {
    static constexpr bool kSub = W == 1 && C == 1;
    int lane, wave;
    int lanes;   // lanes that share a row, within the wave
    int slot;    // this lane's place among all lanes of the row
    int stride;  // lanes of the row, over all waves
    int rows;    // rows a workgroup takes at a time
    int sub;     // this lane's row among them
    __device__ __forceinline__ explicit Place(int shift) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lanes = kSub ? 1 << shift : 64;
        slot = kSub ? lane & (lanes - 1) : W == 1 ? lane : (int)threadIdx.x;
        stride = kSub ? lanes : 64 * W;
        rows = kSub ? 256 >> shift : W == 1 ? 4 : 1;
        sub = kSub ? (int)threadIdx.x >> shift : W == 1 ? wave : 0;
    }
};

template <int W> constexpr int kThreads = W == 8 ? 512 : 256;

// C units per lane, of which the first FC are full in every lane.
template <typename T, typename TP, int W, int C, int FC>
__global__ void __launch_bounds__(kThreads<W>) norm_kernel(NormArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float red[2][W][2];
    const Place<W, C> p(a.shift);
    const int n = a.n;
    const float inv_n = 1.0f / (float)n;
    float w[C][V], b[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (p.slot + c * p.stride) * V;
        load_params(static_cast<const TP*>(a.w), col, n, 1.0f, w[c]);
        load_params(static_cast<const TP*>(a.b), col, n, 0.0f, b[c]);
    }
    for (int64_t r0 = (int64_t)blockIdx.x * p.rows; r0 < a.rows;
         r0 += (int64_t)gridDim.x * p.rows) {
        const int64_t row = r0 + p.sub;
        if (W == 1 && !Place<W, C>::kSub && row >= a.rows) break;
        // (rows that share a wave: no loads or stores past the last one)
        const bool live = !Place<W, C>::kSub || row < a.rows;
        const int nl = live ? n : 0;
        const int64_t at = live ? row * n : 0;
        float v[C][V];
        StaticFor<0, C>::run([&](auto c) {
            load_unit<(c < FC)>(static_cast<const T*>(a.x) + at,
                                          (p.slot + c * p.stride) * V, nl, 0.0f, v[c]);
        });
        if (a.res != nullptr) {
            StaticFor<0, C>::run([&](auto c) {
                float r[V];
                load_unit<(c < FC)>(static_cast<const T*>(a.res) + at,
                                              (p.slot + c * p.stride) * V, nl, 0.0f, r);
#pragma unroll
                for (int i = 0; i < V; ++i) v[c][i] += r[i];
            });
        }
        if (a.h != nullptr) {
            StaticFor<0, C>::run([&](auto c) {
                store_unit<(c < FC)>(static_cast<T*>(a.h) + at,
                                               (p.slot + c * p.stride) * V, nl, v[c]);
            });
        }
        float s = 0.0f, none = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) s += v[c][i];
        s = group_sum(s, p.lanes);
        wave_join<W>(s, none, red[0], p.wave, p.lane);
        const float mu = s * inv_n;
        float q = 0.0f, e = 0.0f;
        StaticFor<0, C>::run([&](auto c) {
            const int col = (p.slot + c * p.stride) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = (c < FC) || col + i < n ? v[c][i] - mu : 0.0f;
                v[c][i] = d;
                e += d;
                q = __builtin_fmaf(d, d, q);
            }
        });
        q = group_sum(q, p.lanes);
        e = group_sum(e, p.lanes);
        wave_join<W>(q, e, red[1], p.wave, p.lane);
        // what the rounding of the sum left out of the mean
        e *= inv_n;
        const float rstd = 1.0f / __builtin_sqrtf(spread(q * inv_n, e) + a.eps);
        if (a.mean != nullptr && live && p.slot == 0) {
            a.mean[row] = mu + e;
            a.rstd[row] = rstd;
        }
        StaticFor<0, C>::run([&](auto c) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] = __builtin_fmaf((v[c][i] - e) * rstd, w[c][i], b[c][i]);
            store_unit<(c < FC)>(static_cast<T*>(a.y) + at, (p.slot + c * p.stride) * V,
                                           nl, v[c]);
        });
    }
}

// Rows that do not fit in registers: one workgroup per row, read three times.
template <typename T, typename TP>
__global__ void __launch_bounds__(512) norm_long_kernel(NormArgs a) {
    __shared__ float red[2][8][2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * n;
        const T* res = a.res ? static_cast<const T*>(a.res) + row * n : nullptr;
        auto value = [&](int i) {
            return Storage<T>::load(x + i) + (res ? Storage<T>::load(res + i) : 0.0f);
        };
        float s = 0.0f, q = 0.0f, none = 0.0f;
        for (int i = threadIdx.x; i < n; i += 512) s += value(i);
        s = group_sum(s, 64);
        wave_join<8>(s, none, red[0], wave, lane);
        const float mu = s / (float)n;
        float e = 0.0f;
        for (int i = threadIdx.x; i < n; i += 512) {
            const float d = value(i) - mu;
            e += d;
            q = __builtin_fmaf(d, d, q);
        }
        q = group_sum(q, 64);
        e = group_sum(e, 64);
        wave_join<8>(q, e, red[1], wave, lane);
        e /= (float)n;
        const float rstd = 1.0f / __builtin_sqrtf(spread(q / (float)n, e) + a.eps);
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

template <typename T, typename TP, int W, int C, int FC>
__global__ void __launch_bounds__(kThreads<W>) norm_grad_kernel(NormGradArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float red[2][W][2];
    __shared__ float join[W == 1 ? 4 * 64 * C * V : 1];
    const Place<W, C> p(a.shift);
    const int n = a.n;
    const float inv_n = 1.0f / (float)n;
    float w[C][V], dw[C][V], db[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_params(static_cast<const TP*>(a.w), (p.slot + c * p.stride) * V, n, 1.0f, w[c]);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[c][i] = db[c][i] = 0.0f;
    }
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * p.rows; r0 < a.rows;
         r0 += (int64_t)gridDim.x * p.rows, turn ^= 1) {
        const int64_t row = r0 + p.sub;
        if (W == 1 && !Place<W, C>::kSub && row >= a.rows) break;
        const bool live = !Place<W, C>::kSub || row < a.rows;
        const int nl = live ? n : 0;
        const int64_t at = live ? row * n : 0;
        float h[C][V], dy[C][V];
        StaticFor<0, C>::run([&](auto c) {
            const int col = (p.slot + c * p.stride) * V;
            load_unit<(c < FC)>(static_cast<const T*>(a.h) + at, col, nl, 0.0f, h[c]);
            load_unit<(c < FC)>(static_cast<const T*>(a.dy) + at, col, nl, 0.0f, dy[c]);
        });
        const float mu = live ? a.mean[row] : 0.0f, rstd = live ? a.rstd[row] : 0.0f;
        float s1 = 0.0f, s2 = 0.0f;
        // (dy is 0 past the row's end, and so is all that is summed of it, as long as xh is
        // finite there: h takes the row's mean)
        StaticFor<0, C>::run([&](auto c) {
            const int col = (p.slot + c * p.stride) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool in = (c < FC) || col + i < nl;
                const float xh = in ? (h[c][i] - mu) * rstd : 0.0f;
                const float g = dy[c][i] * w[c][i];
                dw[c][i] = __builtin_fmaf(dy[c][i], xh, dw[c][i]);
                db[c][i] += dy[c][i];
                s1 += in ? g : 0.0f;
                s2 = __builtin_fmaf(g, xh, s2);
                h[c][i] = xh;
                dy[c][i] = g;
            }
        });
        if (a.dx == nullptr) continue;
        s1 = group_sum(s1, p.lanes);
        s2 = group_sum(s2, p.lanes);
        wave_join<W>(s1, s2, red[turn], p.wave, p.lane);
        s1 *= inv_n;
        s2 *= inv_n;
        StaticFor<0, C>::run([&](auto c) {
            const int col = (p.slot + c * p.stride) * V;
            float d[V];
            if (a.dh != nullptr)
                load_unit<(c < FC)>(static_cast<const T*>(a.dh) + at, col, nl, 0.0f, d);
            else
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i)
                d[i] = __builtin_fmaf(rstd, dy[c][i] - s1 - h[c][i] * s2, d[i]);
            store_unit<(c < FC)>(static_cast<T*>(a.dx) + at, col, nl, d);
        });
    }
    if (a.part == nullptr) return;
    // this workgroup's sums: [2][workgroups][n]
    float* out = a.part + (int64_t)blockIdx.x * n;
    const int64_t half = (int64_t)gridDim.x * n;
    for (int k = 0; k < 2; ++k) {
        float(&acc)[C][V] = k == 0 ? dw : db;
        if (W > 1) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (p.slot + c * p.stride) * V;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (col + i < n) out[k * half + col + i] = acc[c][i];
            }
            continue;
        }
        if (Place<W, C>::kSub)
            for (int o = p.lanes; o < 64; o *= 2)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[0][i] += __shfl_xor(acc[0][i], o);
        __syncthreads();
        const int span = p.stride * C * V;  // columns of a wave's sums, at least n
        if (p.lane < p.lanes) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    join[p.wave * span + (p.slot + c * p.stride) * V + i] = acc[c][i];
        }
        __syncthreads();
        for (int j = threadIdx.x; j < n; j += 256)
            out[k * half + j] = (join[j] + join[span + j]) + (join[2 * span + j] + join[3 * span + j]);
    }
}

// dx of rows that do not fit in registers: one workgroup per row, read twice.
template <typename T, typename TP>
__global__ void __launch_bounds__(512) norm_grad_long_kernel(NormGradArgs a) {
    __shared__ float red[2][8][2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n;
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
        s1 = group_sum(s1, 64);
        s2 = group_sum(s2, 64);
        wave_join<8>(s1, s2, red[turn], wave, lane);
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
template <typename T>
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
    a.part[(int64_t)blockIdx.y * a.n + col] = dw;
    a.part[((int64_t)gridDim.y + blockIdx.y) * a.n + col] = db;
}

// dw (blockIdx.y 0) and db (1) from the workgroups' sums, in a fixed order: 32 columns
// per workgroup, 32 lanes of each column over the parts.
template <typename TP>
__global__ void __launch_bounds__(1024) norm_params_kernel(const float* part, int parts, int n,
                                                           TP* dw, TP* db) {
    __shared__ float sums[32][33];
    TP* out = blockIdx.y == 0 ? dw : db;
    if (out == nullptr) return;
    const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + c;
    const float* src = part + (int64_t)blockIdx.y * parts * n;
    float s = 0.0f;
    if (col < n)
        for (int k = g; k < parts; k += 32) s += src[(int64_t)k * n + col];
    sums[c][g] = s;
    __syncthreads();
    // (lane g of column c: 32 neighbouring lanes add one column)
    s = group_sum(sums[g][c], 32);
    if (c == 0 && blockIdx.x * 32 + g < n) Storage<TP>::store(out + blockIdx.x * 32 + g, s);
}

constexpr int kLongParts = 64;

}  // namespace

NormPlan norm_plan(int64_t rows, int32_t n, int es, bool grad) {
    NormPlan p;
    const int V = 16 / es;
    p.shift = 6;
    p.waves = 1;
    p.units = 1;
    int64_t per = 4;
    if (n > kNormRegRow) {
        p.waves = 0;
        p.units = 0;
        per = 1;
    } else if (n <= 64 * V) {
        p.shift = 0;
        while (V << p.shift < n) ++p.shift;
        per = 256 >> p.shift;
    } else {
        // 32 elements per lane at most, in steps of 8 (at fewer than two units: 4-byte
        // types only)
        const int e = n <= 512 ? 8 : n <= 1024 ? 16 : n <= 1536 ? 24 : n <= 2048 ? 32
                      : n <= 4096 ? 16 : n <= 6144 ? 24 : n <= 8192 ? 32 : n <= 12288 ? 24 : 32;
        p.waves = n <= 2048 ? 1 : n <= 8192 ? 4 : 8;
        p.units = e / V;
        if (p.waves > 1) per = 1;
    }
    const int64_t need = (rows + per - 1) / per;
    const int64_t most = grad ? (p.waves == 8 ? 256 : 512) : 2048;
    p.blocks = (int)(need < most ? need : most);
    p.parts = p.waves == 0 ? (int)(rows < kLongParts ? rows : kLongParts) : p.blocks;
    return p;
}

namespace {

// f(integral constants W, C, FC) for a plan's kernel.
template <typename T, typename F>
void norm_dispatch(const NormPlan& p, F&& f) {
    constexpr int V = kVec<T>;
    auto at = [&](auto w, auto e) {
        // the units before the last eight elements are full in every lane
        constexpr int C = decltype(e)::value / V;
        f(w, std::integral_constant<int, C>{},
          std::integral_constant<int, C - 8 / V>{});
    };
    using std::integral_constant;
    const int e = p.units * V;
    if (p.units == 1)
        f(integral_constant<int, 1>{}, integral_constant<int, 1>{}, integral_constant<int, 0>{});
    else if (p.waves == 1) {
        if (V == 4 && e == 8) at(integral_constant<int, 1>{}, integral_constant<int, V == 4 ? 8 : 16>{});
        else if (e == 16) at(integral_constant<int, 1>{}, integral_constant<int, 16>{});
        else if (e == 24) at(integral_constant<int, 1>{}, integral_constant<int, 24>{});
        else at(integral_constant<int, 1>{}, integral_constant<int, 32>{});
    } else if (p.waves == 4) {
        if (e == 16) at(integral_constant<int, 4>{}, integral_constant<int, 16>{});
        else if (e == 24) at(integral_constant<int, 4>{}, integral_constant<int, 24>{});
        else at(integral_constant<int, 4>{}, integral_constant<int, 32>{});
    } else {
        if (e == 24) at(integral_constant<int, 8>{}, integral_constant<int, 24>{});
        else at(integral_constant<int, 8>{}, integral_constant<int, 32>{});
    }
}

template <typename T, typename TP>
hipError_t norm_forward(const NormPlan& p, const NormArgs& a, hipStream_t s) {
    if (p.waves == 0) {
        norm_long_kernel<T, TP><<<p.blocks, 512, 0, s>>>(a);
        return hipGetLastError();
    }
    norm_dispatch<T>(p, [&](auto w, auto c, auto fc) {
        constexpr int W = decltype(w)::value;
        norm_kernel<T, TP, W, decltype(c)::value, decltype(fc)::value>
            <<<p.blocks, kThreads<W>, 0, s>>>(a);
    });
    return hipGetLastError();
}

template <typename T, typename TP>
hipError_t norm_backward(const NormPlan& p, const NormGradArgs& a, void* dw, void* db,
                         hipStream_t s) {
    hipError_t e = hipSuccess;
    if (a.rows > 0 && p.waves == 0) {
        if (a.dx != nullptr) {
            norm_grad_long_kernel<T, TP><<<p.blocks, 512, 0, s>>>(a);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (a.part != nullptr)
            norm_grad_columns_kernel<T><<<dim3((a.n + 255) / 256, p.parts), 256, 0, s>>>(a);
    } else if (a.rows > 0) {
        norm_dispatch<T>(p, [&](auto w, auto c, auto fc) {
            constexpr int W = decltype(w)::value;
            norm_grad_kernel<T, TP, W, decltype(c)::value, decltype(fc)::value>
                <<<p.blocks, kThreads<W>, 0, s>>>(a);
        });
    }
    if ((e = hipGetLastError()) != hipSuccess || (dw == nullptr && db == nullptr)) return e;
    norm_params_kernel<TP><<<dim3((a.n + 31) / 32, 2), 1024, 0, s>>>(
        a.part, p.parts, a.n, static_cast<TP*>(dw), static_cast<TP*>(db));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(bool bf16, bool bf16_params, const NormPlan& p, NormArgs a, hipStream_t s) {
    a.shift = p.shift;
    if (!bf16) return norm_forward<float, float>(p, a, s);
    if (bf16_params) return norm_forward<uint16_t, uint16_t>(p, a, s);
    return norm_forward<uint16_t, float>(p, a, s);
}

hipError_t launch_norm_grad(bool bf16, bool bf16_params, const NormPlan& p, NormGradArgs a,
                            void* dw, void* db, hipStream_t s) {
    a.shift = p.shift;
    if (!bf16) return norm_backward<float, float>(p, a, dw, db, s);
    if (bf16_params) return norm_backward<uint16_t, uint16_t>(p, a, dw, db, s);
    return norm_backward<uint16_t, float>(p, a, dw, db, s);
}

}  // namespace kan
