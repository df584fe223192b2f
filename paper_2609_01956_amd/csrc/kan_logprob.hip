// kan_logprob.hip -- log probabilities of given classes (tokens) under a softmax over
// logits, with entropy and the k most probable classes, and their gradient.
//
//   m = max_v z_v,  t_v = z_v - m,  s = sum_v exp(t_v)
//   logp = t_target - log s
//   H    = log s - sum_v exp(t_v) t_v / s
//   top k: by (value, then lowest index)
//   dz_v = d ([v = target] - p_v) - dH p_v (log p_v + H),  p_v = exp(t_v - log s)
//
// The forward reads each logit once: every lane keeps a running maximum, sum and weighted
// sum of its own elements (rescaled when a tile raises the maximum), which are joined once
// per row.  log s and the weighted sum are both at least 0, so H does not cancel; m and
// log s go to the backward apart, so p is good to a rounding however far the logits lie from
// 0.  Everything is fp32; a masked class is -infinity (or so low that its weight is 0).
//
// Rows of at most one 16-byte unit per lane of half a wave share a wave.  Longer rows are
// taken by one wave, or four where rows are long and many, or by several workgroups where
// rows are few (each leaves its sums and its best k in the workspace and a second launch
// joins them).
//
// The best k of a wave stand sorted across its lanes, one 64-bit key per lane (the value's
// bits in order, then the complement of the index, so that keys are distinct and ties go
// to the lowest index).  A tile is looked at again only if some lane's largest value
// reaches the k-th best so far; then only its elements that reach the k-th largest of the
// lanes' own maxima can enter (k lanes hold one at least as large), so that few of a first
// tile's elements are inserted, one after the other.
#include "kan_internal.h"
#include "kan_rows.h"

namespace kan {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(t * kLog2e); }

// Running softmax sums relative to m: s = sum exp(z - m), q = sum exp(z - m) (z - m).
struct Sums {
    float m, s, q;
};

// What a maximum is subtracted as: rows (so far) without any class stay at 0.
__device__ __forceinline__ float anchor(float m) { return m == kNegInf ? 0.0f : m; }

// The sums a relative to m instead (m >= a.m).  The difference is held above -200, where its
// exponential is 0 in fp32: no 0 times infinity.
__device__ __forceinline__ void rescale(Sums& a, float m) {
    const float d = __builtin_fmaxf(a.m - anchor(m), -200.0f);
    const float f = exp_of(d);
    a.q = __builtin_fmaf(a.s, d, a.q) * f;
    a.s *= f;
    a.m = m;
}

// Joined over groups of `lanes` lanes; every lane gets the result.
__device__ __forceinline__ void join_lanes(Sums& a, int lanes) {
    rescale(a, group_max(a.m, lanes));
    a.s = group_sum(a.s, lanes);
    a.q = group_sum(a.q, lanes);
}

// Adds the N values (maximum vm among them) to a lane's sums.
template <bool ENT, int N>
__device__ __forceinline__ void add_values(Sums& a, const float (&v)[N], float vm) {
    rescale(a, __builtin_fmaxf(a.m, vm));
    const float m = anchor(a.m);
    float q = 0.0f, s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = v[i] - m, e = exp_of(t);
        s += e;
        if (ENT) q = __builtin_fmaf(e, __builtin_fmaxf(t, -200.0f), q);
    }
    a.s += s;
    a.q += q;
}

template <int N>
__device__ __forceinline__ float max_of(const float (&v)[N]) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = __builtin_fmaxf(m, v[i]);
    return __builtin_fmaxf(m, kNegInf);  // (of NaN alone: -infinity)
}

// (-infinity for a row without any class)
__device__ __forceinline__ float log_sum(const Sums& a) { return logf(a.s); }

// ------------------------------------------------------------------ best k

// Distinct, ordered by (value, lowest index first); NaN below every number, 0 for none.
__device__ __forceinline__ uint64_t key_of(float v, int index) {
    const uint32_t b = __float_as_uint(v + 0.0f);  // (-0 equals 0)
    const uint32_t o = v != v ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (uint64_t)o << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    if (o == 0) return kNegInf;  // NaN or none: whatever is compared with it enters
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_index(uint64_t key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ uint64_t lane_key(uint64_t key, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)key, lane);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(key >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}

// The best k <= 64 keys of a wave: lane i holds the i-th best.  All lanes call.
struct Best {
    uint64_t mine;  // this lane's key
    uint64_t last;  // the k-th best (0: not full yet)
    int k;

    __device__ __forceinline__ explicit Best(int k_) : mine(0), last(0), k(k_) {}

    // Offers one key per lane (0: none).
    __device__ __forceinline__ void offer(uint64_t key, int lane) {
        uint64_t todo = __ballot(key > last);
        while (todo != 0) {
            const uint64_t one = lane_key(key, __builtin_ctzll(todo));
            const int at = __popcll(__ballot(mine > one));
            const uint32_t lo = dpp<kDppWaveShr1>((uint32_t)mine, (uint32_t)mine);
            const uint32_t hi = dpp<kDppWaveShr1>((uint32_t)(mine >> 32), (uint32_t)(mine >> 32));
            mine = lane < at ? mine : lane == at ? one : (uint64_t)hi << 32 | lo;
            last = lane_key(mine, k - 1);
            todo &= todo - 1;
            todo &= __ballot(key > last);
        }
    }
};

// The k-th largest of the lanes' values (k <= 64).
__device__ __forceinline__ float kth_of_lanes(float v, int k) {
    int above = 0;
    for (int l = 0; l < 64; ++l)
        above += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)) > v;
    // the smallest value with fewer than k above it
    return -group_max(above < k ? -v : kNegInf, 64);
}

// ------------------------------------------------------------------ outputs of a row

// z_target - m - log s of a row: NaN for a target outside the classes, 0 for one that is
// ignored, -infinity where no class is left.
__device__ __forceinline__ float target_logp(const LogprobArgs& a, int64_t target, float z,
                                             const Sums& r, float logs) {
    if (target == a.ignore) return 0.0f;
    if (target < 0 || target >= a.classes) return __builtin_nanf("");
    return r.s == 0.0f ? kNegInf : z - r.m - logs;
}

template <typename T>
__device__ __forceinline__ void store_row(const LogprobArgs& a, int64_t row, const Sums& r) {
    const int64_t target = a.targets[row];
    float z = 0.0f;
    if (target >= 0 && target < a.classes)
        z = Storage<T>::load(static_cast<const T*>(a.z) + row * a.stride + target);
    const float logs = log_sum(r);
    a.logp[row] = target_logp(a, target, z, r, logs);
    a.stats[2 * row] = r.m;
    a.stats[2 * row + 1] = logs;
    if (a.entropy != nullptr) a.entropy[row] = r.s == 0.0f ? 0.0f : logs - r.q / r.s;
}

__device__ __forceinline__ void store_top(const LogprobArgs& a, int64_t at, uint64_t key,
                                          const Sums& r) {
    a.top_logp[at] = r.s == 0.0f ? kNegInf : key_value(key) - r.m - log_sum(r);
    a.top_index[at] = key_index(key);
}

// ------------------------------------------------------------------ short rows

// 1 << shift lanes (at most 32) per row, one unit each.
template <typename T>
__global__ void __launch_bounds__(256) logprob_short_kernel(LogprobArgs a) {
    constexpr int V = kVec<T>;
    const int lanes = 1 << a.shift, lane = threadIdx.x & 63;
    const int slot = lane & (lanes - 1), per = 256 >> a.shift;
    for (int64_t r0 = (int64_t)blockIdx.x * per; r0 < a.rows; r0 += (int64_t)gridDim.x * per) {
        const int64_t row = r0 + (threadIdx.x >> a.shift);
        const bool live = row < a.rows;
        const int n = live ? a.classes : 0;
        float v[V];
        load_unit(static_cast<const T*>(a.z) + (live ? row * a.stride : 0), slot * V, n,
                  kNegInfBits<T>, v);
        Sums r = {kNegInf, 0.0f, 0.0f};
        add_values<true>(r, v, max_of(v));
        join_lanes(r, lanes);
        if (live && slot == 0) store_row<T>(a, row, r);
        if (a.k == 0) continue;
        uint64_t key[V];
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = slot * V + i < n ? key_of(v[i], slot * V + i) : 0;
        for (int j = 0; j < a.k; ++j) {
            uint64_t best = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) best = key[i] > best ? key[i] : best;
            for (int o = 1; o < lanes; o *= 2) {
                const uint64_t other = __shfl_xor((unsigned long long)best, o);
                best = other > best ? other : best;
            }
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (key[i] == best) key[i] = 0;
            if (live && slot == 0) store_top(a, row * a.k + j, best, r);
        }
    }
}

// ------------------------------------------------------------------ long rows

constexpr int kTileElems = 32;  // per lane
constexpr int kTile = 64 * kTileElems;

template <typename T> constexpr int kTileUnits = kTileElems / kVec<T>;

// One tile of a row into registers, 16-byte units interleaved over the lanes.
template <typename T>
__device__ __forceinline__ void load_tile(const T* row, int base, int n, int lane,
                                          u32x4 (&raw)[kTileUnits<T>]) {
    constexpr int V = kVec<T>;
    issue_units<0, false>(row, base + lane * V, 64 * V, n, 0u, raw);
    if (base + kTile > n) settle_units<0, false, T>(base + lane * V, 64 * V, n, kNegInfBits<T>, raw);
}

template <typename T>
__device__ __forceinline__ void widen_tile(const u32x4 (&raw)[kTileUnits<T>],
                                           float (&v)[kTileElems]) {
    constexpr int V = kVec<T>;
#pragma unroll
    for (int u = 0; u < kTileUnits<T>; ++u) {
        float unit[V];
        widen(raw[u], unit);
#pragma unroll
        for (int i = 0; i < V; ++i) v[u * V + i] = unit[i];
    }
}

// Offers a tile's elements that can enter the best k (see the file's comment); `vm` is the
// lane's largest.
template <typename T>
__device__ __forceinline__ void offer_tile(Best& best, const float (&v)[kTileElems], float vm,
                                           int base, int n, int lane) {
    constexpr int V = kVec<T>;
    float floor = key_value(best.last);
    const int lanes = __popcll(__ballot(vm >= floor));
    if (lanes == 0) return;
    if (lanes > best.k) floor = __builtin_fmaxf(floor, kth_of_lanes(vm, best.k));
    StaticFor<0, kTileElems>::run([&](auto e) {
        const int index = base + ((e / V) * 64 + lane) * V + e % V;
        const bool in = index < n && !(v[e] < floor);
        best.offer(in ? key_of(v[e], index) : 0, lane);
    });
}

// W waves per (row, part): W = 1, four of them per workgroup, or W = 4.
template <typename T, int W, bool ENT, bool TOP>
__global__ void __launch_bounds__(256) logprob_kernel(LogprobArgs a) {
    __shared__ Sums part[W];
    __shared__ uint64_t keys[W][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t items = a.rows * a.parts;
    for (int64_t i0 = (int64_t)blockIdx.x * (4 / W); i0 < items;
         i0 += (int64_t)gridDim.x * (4 / W)) {
        const int64_t item = i0 + (W == 1 ? wave : 0);
        if (item >= items) break;  // (W = 1)
        const int64_t row = a.parts == 1 ? item : item / a.parts;
        const int p = (int)(item - row * a.parts);
        const T* z = static_cast<const T*>(a.z) + row * a.stride;
        Sums r = {kNegInf, 0.0f, 0.0f};
        Best best(TOP ? a.k : 1);
        const int tiles = (a.classes + kTile - 1) / kTile;
        for (int t = p * W + (W == 1 ? 0 : wave); t < tiles; t += a.parts * W) {
            u32x4 raw[kTileUnits<T>];
            load_tile(z, t * kTile, a.classes, lane, raw);
            float v[kTileElems];
            widen_tile<T>(raw, v);
            const float vm = max_of(v);
            add_values<ENT>(r, v, vm);
            if (TOP) offer_tile<T>(best, v, vm, t * kTile, a.classes, lane);
        }
        join_lanes(r, 64);
        if (W > 1) {
            if (lane == 0) part[wave] = r;
            if (TOP) keys[wave][lane] = lane < a.k ? best.mine : 0;
            __syncthreads();
            if (wave == 0) {
                r = lane < W ? part[lane] : Sums{kNegInf, 0.0f, 0.0f};
                join_lanes(r, 64);
                if (TOP)
                    for (int w = 1; w < W; ++w) best.offer(keys[w][lane], lane);
            }
            __syncthreads();
            if (wave != 0) continue;
        }
        if (a.parts > 1) {
            if (lane == 0) a.part[item] = make_float4(r.m, r.s, r.q, 0.0f);
            if (TOP && lane < a.k) a.keys[item * a.k + lane] = best.mine;
        } else {
            if (lane == 0) store_row<T>(a, row, r);
            if (TOP && lane < a.k) store_top(a, row * a.k + lane, best.mine, r);
        }
    }
}

// Joins the parts (at most 64) of each row: one wave per row.
template <typename T>
__global__ void __launch_bounds__(256) logprob_join_kernel(LogprobArgs a) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = (int64_t)blockIdx.x * 4 + wave;
    if (row >= a.rows) return;
    Sums r = {kNegInf, 0.0f, 0.0f};
    if (lane < a.parts) {
        const float4 f = a.part[row * a.parts + lane];
        r = {f.x, f.y, f.z};
    }
    join_lanes(r, 64);
    if (lane == 0) store_row<T>(a, row, r);
    if (a.k == 0) return;
    // (each part's keys are sorted: the lanes offer theirs rank by rank)
    Best best(a.k);
    const uint64_t* keys = a.keys + (row * a.parts + lane) * a.k;
    for (int j = 0; j < a.k; ++j) best.offer(lane < a.parts ? keys[j] : 0, lane);
    if (lane < a.k) store_top(a, row * a.k + lane, best.mine, r);
}

// ------------------------------------------------------------------ gradient

// What a row's gradient is made of.
struct RowGrad {
    float m, logs, d, dh, h;
    int target;  // -1: none
    bool empty;
};

__device__ __forceinline__ RowGrad row_grad(const LogprobGradArgs& a, int64_t row) {
    RowGrad g;
    const int64_t target = a.targets[row];
    const bool in = target >= 0 && target < a.classes;
    g.m = a.stats[2 * row];
    g.logs = a.stats[2 * row + 1];
    g.empty = g.m == kNegInf;  // no class left: no gradient
    g.target = target != a.ignore && in && !g.empty ? (int)target : -1;
    g.d = target == a.ignore ? 0.0f : in ? a.dlogp[row] : __builtin_nanf("");
    g.dh = a.dentropy != nullptr ? a.dentropy[row] : 0.0f;
    g.h = a.dentropy != nullptr ? a.entropy[row] : 0.0f;
    return g;
}

// In place: the logits to their gradients, for the classes from col on.
template <int V>
__device__ __forceinline__ void unit_grad(const RowGrad& g, int col, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float lp = v[i] - g.m - g.logs;
        const float p = g.empty ? 0.0f : exp_of(lp);
        // (below -1e4 the weight is 0, and the entropy's term with it)
        const float slope = __builtin_fmaf(g.dh, __builtin_fmaxf(lp, -1e4f) + g.h, g.d);
        v[i] = (g.target == col + i ? g.d : 0.0f) - (g.empty ? 0.0f : p * slope);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) logprob_grad_short_kernel(LogprobGradArgs a) {
    constexpr int V = kVec<T>;
    const int lanes = 1 << a.shift;
    const int slot = threadIdx.x & (lanes - 1), per = 256 >> a.shift;
    for (int64_t row = (int64_t)blockIdx.x * per + (threadIdx.x >> a.shift); row < a.rows;
         row += (int64_t)gridDim.x * per) {
        if (slot * V >= a.classes) continue;
        const RowGrad g = row_grad(a, row);
        float v[V];
        load_unit(static_cast<const T*>(a.z) + row * a.stride, slot * V, a.classes, 0u, v);
        unit_grad(g, slot * V, v);
        store_unit<false>(static_cast<T*>(a.dz) + row * a.dstride, slot * V, a.classes, v);
    }
}

constexpr int kGradUnits = 4;  // per lane

template <typename T>
__global__ void __launch_bounds__(256) logprob_grad_kernel(LogprobGradArgs a) {
    constexpr int V = kVec<T>;
    const int64_t items = a.rows * a.segments;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = item / a.segments;
        const int base = (int)(item - row * a.segments) * (256 * kGradUnits * V);
        const RowGrad g = row_grad(a, row);
        const T* z = static_cast<const T*>(a.z) + row * a.stride;
        T* dz = static_cast<T*>(a.dz) + row * a.dstride;
        const int first = base + (int)threadIdx.x * V;
        u32x4 raw[kGradUnits];
        issue_units<0, false>(z, first, 256 * V, a.classes, 0u, raw);
        if (base + 256 * kGradUnits * V > a.classes)
            settle_units<0, false, T>(first, 256 * V, a.classes, 0u, raw);
#pragma unroll
        for (int u = 0; u < kGradUnits; ++u) {
            float v[V];
            widen(raw[u], v);
            unit_grad(g, first + u * 256 * V, v);
            store_unit<false>(dz, first + u * 256 * V, a.classes, v);
        }
    }
}

int grid_of(int64_t n, int64_t most) { return (int)(n < most ? n : most); }

}  // namespace

LogprobPlan logprob_plan(int64_t rows, int32_t classes, int es, int k) {
    LogprobPlan p = {0, 0, 1, 0};
    const int V = 16 / es;
    if (classes <= 32 * V) {
        while (V << p.shift < classes) ++p.shift;
        return p;
    }
    const int64_t tiles = (classes + kTile - 1) / kTile;
    // four waves a row where rows alone fill the GPU with such workgroups and are long
    // enough that each wave gets a tile; below that, parts of rows to 16 waves per CU
    p.waves = rows >= 1024 && tiles >= 4 ? 4 : 1;
    if (p.waves == 1 && rows < 4096) {
        int64_t parts = rows > 0 ? (4096 + rows - 1) / rows : 1;
        if (parts > 64) parts = 64;
        if (parts > tiles) parts = tiles;
        p.parts = (int)parts;
    }
    if (p.parts > 1) p.bytes = (size_t)rows * p.parts * (16 + 8 * (size_t)k);
    return p;
}

namespace {

template <typename T>
hipError_t run_logprob(const LogprobPlan& p, const LogprobArgs& a, hipStream_t s) {
    if (p.waves == 0) {
        const int64_t per = 256 >> p.shift;
        logprob_short_kernel<T><<<grid_of((a.rows + per - 1) / per, 8192), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    const int64_t items = a.rows * p.parts, per = 4 / p.waves;
    const int grid = grid_of((items + per - 1) / per, 1 << 30);
    const bool ent = a.entropy != nullptr, top = a.k > 0;
    auto go = [&](auto w, auto e, auto t) {
        logprob_kernel<T, decltype(w)::value, decltype(e)::value, decltype(t)::value>
            <<<grid, 256, 0, s>>>(a);
    };
    auto pick = [&](auto w) {
        if (ent && top) go(w, std::true_type{}, std::true_type{});
        else if (ent) go(w, std::true_type{}, std::false_type{});
        else if (top) go(w, std::false_type{}, std::true_type{});
        else go(w, std::false_type{}, std::false_type{});
    };
    if (p.waves == 4) pick(std::integral_constant<int, 4>{});
    else pick(std::integral_constant<int, 1>{});
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    logprob_join_kernel<T><<<(int)((a.rows + 3) / 4), 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t run_logprob_grad(LogprobGradArgs a, hipStream_t s) {
    constexpr int V = kVec<T>;
    if (a.classes <= 64 * V) {
        a.shift = 0;
        while (V << a.shift < a.classes) ++a.shift;
        const int64_t per = 256 >> a.shift;
        logprob_grad_short_kernel<T><<<grid_of((a.rows + per - 1) / per, 8192), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    a.segments = (a.classes + 256 * kGradUnits * V - 1) / (256 * kGradUnits * V);
    logprob_grad_kernel<T><<<grid_of(a.rows * a.segments, 1 << 30), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_logprob(bool bf16, const LogprobPlan& p, LogprobArgs a, void* ws,
                          hipStream_t s) {
    a.shift = p.shift;
    a.parts = p.parts;
    a.part = static_cast<float4*>(ws);
    a.keys = p.parts > 1 ? reinterpret_cast<uint64_t*>(a.part + a.rows * p.parts) : nullptr;
    return bf16 ? run_logprob<uint16_t>(p, a, s) : run_logprob<float>(p, a, s);
}

hipError_t launch_logprob_grad(bool bf16, LogprobGradArgs a, hipStream_t s) {
    return bf16 ? run_logprob_grad<uint16_t>(a, s) : run_logprob_grad<float>(a, s);
}

}  // namespace kan
