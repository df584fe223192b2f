// kan_clip.hip -- the global 2-norm of many tensors, and scaling them to a bound on it.
//
//   N = sqrt(sum_t sum_i g_t[i]^2),  c = min(1, max_norm / (N + eps)),  out = c g
//
// Bound by HBM: every gradient is read once for the norm and, when it is clipped (or goes to
// other tensors), read again and written.  Squares and their sums are binary64, which costs
// nothing beside the reads and neither overflows nor drops small gradients: every fp32
// gradient's square is exact.  Each workgroup sums its own chunks into one partial, and each
// workgroup of the second launch adds all partials in the same fixed order (at most
// kClipGroups and one per launch: 2 us from the caches, less than a launch between them) before
// it scales, each product rounded to fp32 (and from there to bf16).  It goes through the chunks
// from the last to the first, as the last ones read are still in the Infinity Cache.  In place
// with c = 1 it returns without touching the gradients.
//
// The tensors go by value, as many per launch as a kernel's 4 KB of arguments hold: no table
// is copied to the device or kept.  A tensor is cut into chunks of kClipChunk elements,
// numbered over the launch's tensors; a workgroup takes every gridDim-th chunk and finds its
// tensor by a count over its lanes.
//
// Measured on MI355X: 235 M bf16 gradients in 64 tensors into other tensors 243-251 us (the two
// reads and the write at 5.6-5.8 TB/s) and 254 in place, within the bound 95 us (4.9 TB/s); 64 x
// 2^20 fp32 into other tensors 135 us, in place 160, within the bound 57.
#include "kan_ops.h"
#include "kan_rows.h"

namespace kan {

namespace {

// A chunk's tensor and place in it.
struct Chunk {
    int tensor, n;
    int64_t at;
    bool bf16;
};

// Finds chunks: each lane holds the first chunks of every 64th tensor, so that a search is a
// comparison and a count, without a load.
template <int N>
struct Finder {
    static constexpr int R = (N + 63) / 64;
    int first[R];
    __device__ __forceinline__ explicit Finder(const ClipArgs<N>& a) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int t = r * 64 + lane;
            first[r] = t < a.count ? a.first[t] : 0x7fffffff;
        }
    }
    __device__ __forceinline__ Chunk find(const ClipArgs<N>& a, int chunk) const {
        Chunk c;
        c.tensor = -1;  // (the last tensor whose first chunk is not past it)
#pragma unroll
        for (int r = 0; r < R; ++r) c.tensor += __popcll(__ballot(first[r] <= chunk));
        c.at = (int64_t)(chunk - a.first[c.tensor]) * kClipChunk;
        c.n = chunk + 1 == a.first[c.tensor + 1] ? (a.tail[c.tensor] >> 1) + 1 : kClipChunk;
        c.bf16 = a.tail[c.tensor] & 1;
        return c;
    }
};

// Sum over the workgroup, every lane gets it.
__device__ __forceinline__ double group_total(double v) {
    __shared__ double red[4];
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// f(units of a chunk at p, column of the first, elements left) for the 256 lanes' units, four
// in flight.
template <typename T, typename F>
__device__ __forceinline__ void for_units(const T* p, int n, F&& f) {
    constexpr int V = kVec<T>, U = 4;
    for (int i = threadIdx.x * V; i < n; i += 256 * V * U) {
        u32x4 raw[U];
        issue_units<0, true>(p, i, 256 * V, n, 0u, raw);
        settle_units<0, true, T>(i, 256 * V, n, 0u, raw);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[V];
            widen(raw[u], v);
            f(i + u * 256 * V, v);
        }
    }
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* p, int n) {
    constexpr int V = kVec<T>;
    double s0 = 0.0, s1 = 0.0;
    for_units(p, n, [&](int, const float(&v)[V]) {
#pragma unroll
        for (int k = 0; k < V; k += 2) {
            s0 = __builtin_fma((double)v[k], (double)v[k], s0);
            s1 = __builtin_fma((double)v[k + 1], (double)v[k + 1], s1);
        }
    });
    return s0 + s1;
}

__global__ void __launch_bounds__(256) clip_norm_kernel(ClipArgs<kClipTensors> a, double* part) {
    const Finder<kClipTensors> finder(a);
    double s = 0.0;
    for (int i = blockIdx.x; i < a.chunks; i += gridDim.x) {
        const Chunk c = finder.find(a, i);
        s += c.bf16 ? chunk_squares(static_cast<const uint16_t*>(a.in[c.tensor]) + c.at, c.n)
                    : chunk_squares(static_cast<const float*>(a.in[c.tensor]) + c.at, c.n);
    }
    s = group_total(s);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double* part, int parts) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
    return __builtin_sqrt(group_total(s));
}

__global__ void __launch_bounds__(256) clip_join_kernel(const double* part, int parts,
                                                        float* norm) {
    const double n = norm_of(part, parts);
    if (threadIdx.x == 0) *norm = (float)n;
}

template <bool PAST, typename T>
__device__ __forceinline__ void chunk_scale(const T* p, T* q, int n, double c) {
    constexpr int V = kVec<T>;
    for_units(p, n, [&](int i, float(&v)[V]) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = (float)((double)v[k] * c);
        store_unit<false, PAST>(q, i, n, v);
    });
}

// OUT: the tensors' outputs stand after the N tensors' arguments (else in place).  PAST: they are
// stored past the caches.
template <int N, bool OUT, bool PAST>
__global__ void __launch_bounds__(256) clip_scale_kernel(ClipArgs<N> a, ClipOuts<OUT ? N : 1> o,
                                                         const double* part, int parts,
                                                         ClipBound b) {
    const Finder<N> finder(a);
    const double n = norm_of(part, parts);
    if (blockIdx.x == 0 && threadIdx.x == 0) *b.norm = (float)n;
    // (gradients that are all 0 stay as they are, and all do without a bound, whose ratio to an
    // infinite norm is NaN; a NaN among them reaches all)
    const double bound = b.max_norm, above = n + (double)b.eps;
    const double f = n == 0.0 || bound >= above ? 1.0 : bound / above;
    for (int i = a.chunks - 1 - (int)blockIdx.x; i >= 0; i -= gridDim.x) {
        const Chunk c = finder.find(a, i);
        void* out = OUT ? o.out[c.tensor] : const_cast<void*>(a.in[c.tensor]);
        if (f == 1.0 && a.in[c.tensor] == out) continue;
        if (c.bf16)
            chunk_scale<PAST>(static_cast<const uint16_t*>(a.in[c.tensor]) + c.at,
                        static_cast<uint16_t*>(out) + c.at, c.n, f);
        else
            chunk_scale<PAST>(static_cast<const float*>(a.in[c.tensor]) + c.at,
                        static_cast<float*>(out) + c.at, c.n, f);
    }
}

// The next launch's tensors from *t on (tensors of no elements are left out).
template <int N>
bool next_args(const ClipList& l, int64_t* t, ClipArgs<N>* a, void** out) {
    a->count = 0;
    a->chunks = 0;
    for (; *t < l.count && a->count < N; ++*t) {
        const int64_t n = l.sizes[*t];
        if (n == 0) continue;
        a->in[a->count] = l.in[*t];
        a->first[a->count] = a->chunks;
        a->tail[a->count] = (uint16_t)(((n - 1) % kClipChunk) << 1 | (l.bf16(*t) ? 1 : 0));
        if (out != nullptr) out[a->count] = l.out[*t];
        a->chunks += (int)((n + kClipChunk - 1) / kClipChunk);
        ++a->count;
    }
    a->first[a->count] = a->chunks;
    return a->count > 0;
}

template <int N, bool OUT>
hipError_t scale(const ClipList& l, const double* part, int parts, ClipBound b, bool past,
                 hipStream_t s) {
    ClipArgs<N> a;
    ClipOuts<OUT ? N : 1> o;
    bool first = true;
    for (int64_t t = 0; next_args(l, &t, &a, OUT ? o.out : nullptr) || first; first = false) {
        // (one workgroup at least, for the norm)
        const int groups = a.chunks < 1 ? 1 : a.chunks < kClipGroups ? a.chunks : kClipGroups;
        if (past) clip_scale_kernel<N, OUT, true><<<groups, 256, 0, s>>>(a, o, part, parts, b);
        else clip_scale_kernel<N, OUT, false><<<groups, 256, 0, s>>>(a, o, part, parts, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t clip_launches(int64_t count) { return (count + kClipTensors - 1) / kClipTensors; }

}  // namespace

size_t clip_workspace(int64_t count) {
    return sizeof(double) * (kClipGroups + (size_t)clip_launches(count));
}

hipError_t launch_clip(const ClipList& l, const ClipBound& b, void* ws, hipStream_t s) {
    double* part = static_cast<double*>(ws);
    const int64_t launches = clip_launches(l.count);
    const int most = launches > 0 ? kClipGroups / (int)launches + 1 : 1;
    int parts = 0;
    ClipArgs<kClipTensors> a;
    for (int64_t t = 0; next_args(l, &t, &a, nullptr);) {
        const int groups = a.chunks < most ? a.chunks : most;
        clip_norm_kernel<<<groups, 256, 0, s>>>(a, part + parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        parts += groups;
    }
    if (l.out == nullptr) {
        clip_join_kernel<<<1, 256, 0, s>>>(part, parts, b.norm);
        return hipGetLastError();
    }
    bool in_place = true;
    int64_t bytes = 0;
    for (int64_t t = 0; t < l.count; ++t) {
        in_place &= l.out[t] == l.in[t] || l.sizes[t] == 0;
        bytes += l.sizes[t] * (l.bf16(t) ? 2 : 4);
    }
    const bool past = bytes >= kPastCaches;
    return in_place ? scale<kClipTensors, false>(l, part, parts, b, past, s)
                    : scale<kClipTensorsOut, true>(l, part, parts, b, past, s);
}

}  // namespace kan
