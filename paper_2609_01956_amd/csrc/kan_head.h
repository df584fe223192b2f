// kan_head.h -- host-side launch interface of the token operators (embedding, linear head),
// between the C ABI layer and the kernel translation units.  Not installed; not part of the
// public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace kan {

// ---------------------------------------------------------------- linear head

// Rows x of n elements against classes weights of n elements.
struct HeadShape {
    int64_t rows;
    int32_t classes, n;
    int es;            // bytes per element
    bool xs, ws;       // can x and the weights be read as they stand (16-byte rows)
    int64_t xstride, wstride;
};
struct HeadArgs {
    const void *x, *w;
    const int64_t* targets;
    int64_t ignore;
    float scale;
    float *logp, *stats;
    int64_t* best;  // may be null
};
struct HeadGradArgs {
    const void *x, *w;
    const int64_t* targets;
    int64_t ignore;
    float scale;
    const float *stats, *dlogp;
    void *dx, *dw;  // either may be null
};
size_t head_workspace(const HeadShape& s);
size_t head_grad_workspace(const HeadShape& s, bool dx, bool dw);
hipError_t launch_head(const HeadShape& s, const HeadArgs& a, void* ws, hipStream_t st);
hipError_t launch_head_grad(const HeadShape& s, const HeadGradArgs& a, void* ws, hipStream_t st);

// ---------------------------------------------------------------- embedding

struct EmbedArgs {
    const int64_t* tokens;
    const void* table;
    void* y;
    int64_t rows, tstride;
    int32_t classes, n;
    int64_t ignore;
    float scale;
};
struct EmbedGradArgs {
    const int64_t* tokens;
    const void *dy, *base;  // base may be null, or dtable itself
    void* dtable;
    int64_t rows, dystride;
    int32_t classes, n;
    int64_t ignore;
    float scale;
};
size_t embed_grad_workspace(int64_t rows, int32_t classes, int32_t n);
hipError_t launch_embed(bool bf16, bool bf16_table, const EmbedArgs& a, hipStream_t s);
hipError_t launch_embed_grad(bool bf16, bool bf16_table, const EmbedGradArgs& a, void* ws,
                             hipStream_t s);

}  // namespace kan
