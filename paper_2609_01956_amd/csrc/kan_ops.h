// kan_ops.h -- host-side launch interface of the operators around the layer, between the C ABI
// layer and the kernel translation units.  Not installed; not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace kan {

// Most workgroups of 256 lanes in a launch: a grid holds fewer than 2^32 work-items.
constexpr int64_t kMaxGroups = (INT64_C(1) << 24) - 1;

// ---------------------------------------------------------------- layer norm

struct NormArgs {
    const void *x, *res, *w, *b;  // res, w, b may be null
    void *h, *y;                  // h may be null
    float *mean, *rstd;           // both null or both not
    int64_t rows;
    int n;
    float eps;
    int shift;  // log2 of the lanes that share a row (one unit per lane)
    int waves;  // waves that share a row
};
struct NormGradArgs {
    const void *h, *w, *dy, *dh;  // w, dh may be null
    const float *mean, *rstd;
    void* dx;     // may be null
    float* part;  // [2][parts][n] partial weight gradients; null: none, or one part:
    void *dw, *db;  // then the gradients themselves; may be null
    int64_t rows;
    int n;
    int shift, waves;
};
// Longest row that stays in registers.
constexpr int kNormRegRow = 16384;
struct NormPlan {
    int waves;    // per row; 0: rows longer than kNormRegRow
    int units;    // 16-byte units per lane
    int shift;    // log2 of the lanes of a row within a wave (one unit per lane)
    int threads;  // of a workgroup
    size_t lds;   // bytes (backward)
    int blocks;   // workgroups
    int parts;    // partial weight gradients (backward)
};
// es: bytes per element of the rows.
NormPlan norm_plan(int64_t rows, int32_t n, int es, bool grad);
hipError_t launch_norm(bool bf16, bool bf16_params, const NormPlan& p, NormArgs a, hipStream_t s);
hipError_t launch_norm_grad(bool bf16, bool bf16_params, const NormPlan& p, NormGradArgs a,
                            hipStream_t s);

// ---------------------------------------------------------------- log probabilities

struct LogprobArgs {
    const void* z;
    const int64_t* targets;
    int64_t rows, stride;  // elements from row to row
    int64_t ignore;
    int classes, k;
    float *logp, *stats, *entropy;  // entropy may be null
    float* top_logp;
    int64_t* top_index;
    int shift;      // short rows: log2 of the lanes of a row
    int parts;      // waves that share a row
    float4* part;   // [rows][parts] sums of the parts
    uint64_t* keys; // [rows][parts][k] their best classes
};
struct LogprobGradArgs {
    const void* z;
    const int64_t* targets;
    const float *stats, *dlogp, *entropy, *dentropy;  // the last two both null or both not
    void* dz;
    int64_t rows, stride, dstride, ignore;
    int classes;
    int shift;       // short rows
    uint32_t items;  // (row, tile)
    uint32_t tiles;  // per row
};
// Workgroups of the tiled forward: four items each at a time, as many turns as it takes.
inline int logprob_groups(int64_t items) {
    const int64_t groups = (items + 3) / 4;
    return (int)(groups < kMaxGroups ? groups : kMaxGroups);
}
// The tiled gradient's rows in pieces of one launch each, four tiles per workgroup: launch(args
// of a piece, its workgroups) until one fails.  es: bytes per logit.
template <typename F>
hipError_t logprob_grad_pieces(LogprobGradArgs a, size_t es, F&& launch) {
    const int64_t all = a.rows, most = 4 * kMaxGroups / a.tiles;
    for (int64_t done = 0; done < all;) {
        a.rows = all - done < most ? all - done : most;
        a.items = (uint32_t)(a.rows * a.tiles);
        const LogprobGradArgs& piece = a;
        const hipError_t e = launch(piece, (int)((a.items + 3) / 4));
        if (e != hipSuccess) return e;
        a.z = static_cast<const char*>(a.z) + a.rows * a.stride * (int64_t)es;
        a.dz = static_cast<char*>(a.dz) + a.rows * a.dstride * (int64_t)es;
        a.targets += a.rows;
        a.stats += 2 * a.rows;
        a.dlogp += a.rows;
        if (a.dentropy != nullptr) {
            a.entropy += a.rows;
            a.dentropy += a.rows;
        }
        done += a.rows;
    }
    return hipSuccess;
}
constexpr int kMaxTop = 64;
struct LogprobPlan {
    int elems;  // of a tile, per lane; 0: rows that share a wave
    int shift, parts;
    size_t bytes;  // workspace
};
LogprobPlan logprob_plan(int64_t rows, int32_t classes, int es, int k);
hipError_t launch_logprob(bool bf16, const LogprobPlan& p, LogprobArgs a, void* ws, hipStream_t s);
hipError_t launch_logprob_grad(bool bf16, LogprobGradArgs a, hipStream_t s);

// ---------------------------------------------------------------- gradient clipping

// Tensors of one launch, by value: 14 bytes each and 8 for an output elsewhere, within the
// 4 KB of a kernel's arguments.
constexpr int kClipTensors = 272, kClipTensorsOut = 176;
constexpr int kClipChunk = 1 << 14;  // elements
constexpr int kClipGroups = 2048;    // workgroups of a launch, and partial sums in all
template <int N>
struct ClipArgs {
    const void* in[N];
    int first[N + 1];  // a tensor's first chunk; after the last tensor: all chunks
    uint16_t tail[N];  // elements of the last chunk less 1, times 2, plus 1 for bf16
    int count, chunks;
};
template <int N>
struct ClipOuts {
    void* out[N];
};
struct ClipBound {
    float max_norm, eps;
    float* norm;
};
static_assert(sizeof(ClipArgs<kClipTensors>) + 64 <= 4096, "kernel arguments");
static_assert(sizeof(ClipArgs<kClipTensorsOut>) + sizeof(ClipOuts<kClipTensorsOut>) + 64 <= 4096,
              "kernel arguments");
struct ClipList {
    int64_t count;
    const void* const* in;
    void* const* out;  // null: the norm alone
    const int64_t* sizes;
    const int32_t* dtypes;  // kan_dtype
    bool bf16(int64_t t) const { return dtypes[t] == 1; }
};
// Most tensors and elements of a call (the check for overlaps numbers tensors in 16 bits, chunks
// are counted in 32 bits).
constexpr int kClipMaxTensors = 1 << 14;
constexpr int64_t kClipMaxElements = INT64_C(1) << 40;
size_t clip_workspace(int64_t count);
hipError_t launch_clip(const ClipList& l, const ClipBound& b, void* ws, hipStream_t s);

}  // namespace kan
