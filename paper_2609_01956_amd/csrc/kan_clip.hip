// kan_clip.hip -- the global 2-norm of many tensors, and scaling them to a bound on it.
//
//   N = sqrt(sum_t sum_i g_t[i]^2),  c = min(1, max_norm / (N + eps)),  out = c g
//
// Bound by HBM: every gradient is read once for the norm and, when it is clipped (or goes to
// other tensors), read again and written.  Squares and their sums are binary64, which costs
// nothing beside the reads and neither overflows nor drops small gradients: every fp32
// gradient's square is exact.  Each workgroup sums its own chunks into one partial; a
// one-workgroup launch adds the partials in a fixed order and leaves N and c; the third
// launch scales, each product rounded once.  In place with c = 1 it returns without touching the gradients.
//
// The tensors go by value, kClipTensors per launch (a kernel's arguments hold 4 KB): no
// table is copied to the device or kept.  A tensor is cut into chunks of kClipChunk
// elements, numbered over the launch's tensors; a workgroup takes every gridDim-th chunk
// and finds its tensor by bisection.
#include "kan_internal.h"
#include "kan_rows.h"

namespace kan {

namespace {

// The chunk's tensor: the last one whose first chunk is not past it.
__device__ __forceinline__ int tensor_of(const ClipArgs& a, int chunk) {
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double sum_of_waves(double v, double* red) {
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < waves; ++w) v += red[w];
    return v;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* p, int n) {
    constexpr int V = kVec<T>;
    double s = 0.0;
    for (int i = threadIdx.x * V; i < n; i += 256 * V) {
        float v[V];
        load_unit(p, i, n, 0u, v);
#pragma unroll
        for (int k = 0; k < V; ++k) s = __builtin_fma((double)v[k], (double)v[k], s);
    }
    return s;
}

__global__ void __launch_bounds__(256) clip_norm_kernel(ClipArgs a, double* part) {
    __shared__ double red[4];
    double s = 0.0;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int t = tensor_of(a, c);
        const int64_t at = (int64_t)(c - a.first[t]) * kClipChunk;
        const int64_t left = (a.size[t] >> 1) - at;
        const int n = (int)(left < kClipChunk ? left : kClipChunk);
        s += (a.size[t] & 1) ? chunk_squares(static_cast<const uint16_t*>(a.in[t]) + at, n)
                             : chunk_squares(static_cast<const float*>(a.in[t]) + at, n);
    }
    s = sum_of_waves(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm, and the factor after it.
__global__ void __launch_bounds__(256) clip_join_kernel(const double* part, int parts,
                                                        float max_norm, float eps, float* norm,
                                                        double* factor) {
    __shared__ double red[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
    s = sum_of_waves(s, red);
    if (threadIdx.x != 0) return;
    const double n = __builtin_sqrt(s);
    *norm = (float)n;
    if (factor != nullptr) {
        // (gradients that are all 0 stay as they are; a NaN among them reaches all)
        const double c = n == 0.0 ? 1.0 : (double)max_norm / (n + (double)eps);
        *factor = c >= 1.0 ? 1.0 : c;
    }
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T* p, T* q, int n, double c) {
    constexpr int V = kVec<T>;
    for (int i = threadIdx.x * V; i < n; i += 256 * V) {
        float v[V];
        load_unit(p, i, n, 0u, v);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = (float)((double)v[k] * c);
        store_unit<false>(q, i, n, v);
    }
}

__global__ void __launch_bounds__(256) clip_scale_kernel(ClipArgs a, ClipOuts o,
                                                         const double* factor) {
    const double f = *factor;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int t = tensor_of(a, c);
        if (f == 1.0 && a.in[t] == o.out[t]) continue;
        const int64_t at = (int64_t)(c - a.first[t]) * kClipChunk;
        const int64_t left = (a.size[t] >> 1) - at;
        const int n = (int)(left < kClipChunk ? left : kClipChunk);
        if (a.size[t] & 1)
            chunk_scale(static_cast<const uint16_t*>(a.in[t]) + at,
                        static_cast<uint16_t*>(o.out[t]) + at, n, f);
        else
            chunk_scale(static_cast<const float*>(a.in[t]) + at,
                        static_cast<float*>(o.out[t]) + at, n, f);
    }
}

constexpr int kClipGroups = 2048;

// The next launch's tensors from *t on.
bool next_args(const ClipList& l, int64_t* t, ClipArgs* a, ClipOuts* o) {
    a->count = 0;
    a->chunks = 0;
    for (; *t < l.count && a->count < kClipTensors; ++*t) {
        const int64_t n = l.sizes[*t], chunks = (n + kClipChunk - 1) / kClipChunk;
        if (n == 0) continue;
        a->in[a->count] = l.in[*t];
        a->size[a->count] = n << 1 | (l.bf16(*t) ? 1 : 0);
        a->first[a->count] = a->chunks;
        if (l.out != nullptr) o->out[a->count] = l.out[*t];
        a->chunks += (int)chunks;
        ++a->count;
    }
    return a->count > 0;
}

int clip_groups(const ClipArgs& a) { return a.chunks < kClipGroups ? a.chunks : kClipGroups; }

}  // namespace

size_t clip_workspace(int64_t count) {
    // (tensors of no elements take no place in a launch: this many launches at most)
    const int64_t launches = (count + kClipTensors - 1) / kClipTensors;
    return 16 + sizeof(double) * kClipGroups * (size_t)launches;
}

hipError_t launch_clip(const ClipList& l, float max_norm, float eps, float* norm, void* ws,
                       hipStream_t s) {
    double* factor = static_cast<double*>(ws);
    double* part = reinterpret_cast<double*>(static_cast<char*>(ws) + 16);
    ClipArgs a;
    ClipOuts o;
    int parts = 0;
    for (int64_t t = 0; next_args(l, &t, &a, &o);) {
        const int groups = clip_groups(a);
        clip_norm_kernel<<<groups, 256, 0, s>>>(a, part + parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        parts += groups;
    }
    clip_join_kernel<<<1, 256, 0, s>>>(part, parts, max_norm, eps, norm,
                                       l.out != nullptr ? factor : nullptr);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || l.out == nullptr) return e;
    for (int64_t t = 0; next_args(l, &t, &a, &o);) {
        clip_scale_kernel<<<clip_groups(a), 256, 0, s>>>(a, o, factor);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace kan
