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
// log s go to the backward apart, so p loses nothing where the logits lie far from 0 (what it
// keeps is the rounding of z - m - log s).  Everything is fp32; a masked class is -infinity (or
// so low that its weight is 0).
//
// Rows of at most one 16-byte unit per lane of half a wave share a wave.  Longer rows are
// taken in tiles of up to 32 elements per lane, the next tile's loads in flight, by a wave
// each, or by several where rows are few (each leaves its sums and its best k in the
// workspace and a second launch joins them).
//
// The best k of a wave stand sorted across its lanes, one 64-bit key per lane (the value's
// bits in order, then the complement of the index, so that keys are distinct and ties go
// to the lowest index).  A tile is looked at again only if some lane's largest value
// reaches the k-th best so far.  Then every such lane offers its largest: many at once (the
// first tile) are sorted across the lanes and merged, few are inserted one after the
// other; those lanes' next largest are compared again, until none reaches the k-th best.
//
// Measured on MI355X: 2001 x 50001 bf16 with entropy 37-39 us (5.1-5.4 TB/s), with 5 alternatives
// 51-54 us (bound by the vector ALUs: 10.5 operations per element counting the exponential
// as four, and the lists); 4096 x 131072 bf16 190 us (5.7 TB/s); 1 x 131072 bf16 with 20
// alternatives 7.3 us and 4 us for the join; gradient of 4096 x 131072 bf16 361 us (5.9 TB/s).
// fp32: 2001 x 50001 with entropy 70 us (5.8 TB/s), with 5 alternatives 73; rows that share a wave,
// 65536 x 10 with 3 or 10 alternatives 14 us (12 without; host bound), 65536 x 100 bf16 with 20
// 61 us, a search over the row's lanes for each.
#include "kan_ops.h"
#include "kan_rows.h"

namespace kan {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f, kLn2Low = -1.904654299957768e-9f;  // their sum
constexpr float kNegInf = -__builtin_huge_valf();

// The forward's.  The roundings of t log2 e and of the constant stay, so a term is off by at most
// 1e-7 + 7.3e-8 |t| of itself (3.8e-6 at t = -50).  In s terms weigh by their size: the constant's
// share, which has one sign, adds at most 1.3e-8 of the entropy (1.6e-7 in log s over 131072
// classes), the products' roundings have either.  The exact form takes 10-20% more where the
// vector ALUs bound (2001 x 50001 bf16 37.6 -> 44.6 us, with 5 alternatives 53 -> 64; 65536 x 1000
// bf16 37 -> 43.5).
__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(t * kLog2e); }

// The gradient's, whose every p is an output: to 2^-22 of the value (t above -1e5).  What the
// rounding of t log2 e and of the constant left out, t - h ln 2, is taken back as a factor; mostly
// hidden behind the memory (against the short form, bf16: 4096 x 131072 361 us both, 20000 x 4000
// 60.0 -> 60.8, and where the gradient stays in the caches 65536 x 1000 49.2 -> 50.3).
__device__ __forceinline__ float exp_exact(float t) {
    const float h = t * kLog2e, e = __builtin_amdgcn_exp2f(h);
    return __builtin_fmaf(e, __builtin_fmaf(-h, kLn2Low, __builtin_fmaf(-h, kLn2, t)), e);
}

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

// Joined over the wave.
__device__ __forceinline__ void join_wave(Sums& a) {
    rescale(a, wave_max(a.m));
    a.s = wave_sum(a.s);
    a.q = wave_sum(a.q);
}

// Adds the N values (vm = max_of(v)) to a lane's sums.
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

// The largest of the values that are numbers (NaN if none is).
template <int N>
__device__ __forceinline__ float max_of(const float (&v)[N]) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = __builtin_fmaxf(m, v[i]);
    return m;
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

// The key of lane `lane` ^ S.
template <int S>
__device__ __forceinline__ uint64_t key_xor(uint64_t key) {
    const uint32_t lo = (uint32_t)key, hi = (uint32_t)(key >> 32);
    if constexpr (S == 1) return (uint64_t)dpp<kDppXor1>(hi) << 32 | dpp<kDppXor1>(lo);
    if constexpr (S == 2) return (uint64_t)dpp<kDppXor2>(hi) << 32 | dpp<kDppXor2>(lo);
    if constexpr (S == 4) {
        const uint32_t l = dpp<kDppHalfMirror>(lo), h = dpp<kDppHalfMirror>(hi);
        return (uint64_t)dpp<kDppFlip4>(h) << 32 | dpp<kDppFlip4>(l);
    }
    if constexpr (S == 8) return (uint64_t)dpp<kDppRor8>(hi) << 32 | dpp<kDppRor8>(lo);
    if constexpr (S >= 16) return __shfl_xor((unsigned long long)key, S);
}

// Lanes that keep the larger key in a step of a bitonic sort (largest first) of groups of
// `size`: those whose bit `step` agrees with the order of their group.
constexpr uint64_t keep_larger(int size, int step) {
    uint64_t m = 0;
    for (int l = 0; l < 64; ++l)
        if (((l & step) == 0) == ((l & size) == 0)) m |= UINT64_C(1) << l;
    return m;
}
template <int SIZE, int STEP>
__device__ __forceinline__ uint64_t sort_step(uint64_t key) {
    const uint64_t other = key_xor<STEP>(key);
    const bool larger = __builtin_amdgcn_inverse_ballot_w64(keep_larger(SIZE, STEP));
    return (other > key) == larger ? other : key;
}
// Steps STEP, STEP / 2 .. 1.
template <int SIZE, int STEP>
__device__ __forceinline__ uint64_t sort_steps(uint64_t key) {
    key = sort_step<SIZE, STEP>(key);
    if constexpr (STEP > 1) key = sort_steps<SIZE, STEP / 2>(key);
    return key;
}
// The keys of a wave in falling order over its lanes.
__device__ __forceinline__ uint64_t sort_keys(uint64_t key) {
    key = sort_steps<2, 1>(key);
    key = sort_steps<4, 2>(key);
    key = sort_steps<8, 4>(key);
    key = sort_steps<16, 8>(key);
    key = sort_steps<32, 16>(key);
    return sort_steps<64, 32>(key);
}

// The best k <= 64 keys of a wave: lane i holds the i-th best.  All lanes call.
struct Best {
    uint64_t mine;  // this lane's key
    uint64_t bar;   // what a key has to pass: the k-th best (0: not full yet)
    int k;

    __device__ __forceinline__ explicit Best(int k_) : mine(0), bar(0), k(k_) {}

    __device__ __forceinline__ void raise(uint64_t b) { bar = b > bar ? b : bar; }

    // Merges 64 keys in falling order.
    __device__ __forceinline__ void merge(uint64_t sorted, int lane) {
        if (lane_key(mine, 0) == 0) {
            mine = sorted;
        } else {
            const uint64_t other = __shfl((unsigned long long)sorted, 63 - lane);
            mine = sort_steps<64, 32>(other > mine ? other : mine);
        }
        raise(lane_key(mine, k - 1));
    }

    // Offers one key per lane (0: none).
    __device__ __forceinline__ void offer(uint64_t key, int lane) {
        uint64_t todo = __ballot(key > bar);
        // (an insertion takes about a seventh of sorting and merging)
        if (__popcll(todo) > 7) {
            merge(sort_keys(key > bar ? key : 0), lane);
            return;
        }
        while (todo != 0) {
            const uint64_t one = lane_key(key, __builtin_ctzll(todo));
            const int at = __popcll(__ballot(mine > one));
            const uint32_t lo = dpp_shr((uint32_t)mine), hi = dpp_shr((uint32_t)(mine >> 32));
            mine = lane < at ? mine : lane == at ? one : (uint64_t)hi << 32 | lo;
            raise(lane_key(mine, k - 1));
            todo &= todo - 1;
            todo &= __ballot(key > bar);
        }
    }
};

// ------------------------------------------------------------------ outputs of a row

// A row's target and its logit, read ahead of the sums.
struct Target {
    int64_t index;
    float z;
};
template <typename T>
__device__ __forceinline__ Target target_of(const LogprobArgs& a, int64_t row) {
    Target t;
    t.index = a.targets[row];
    const bool in = t.index >= 0 && t.index < a.classes;
    t.z = Storage<T>::load(static_cast<const T*>(a.z) + row * a.stride + (in ? t.index : 0));
    return t;
}

__device__ __forceinline__ void store_row(const LogprobArgs& a, int64_t row, const Target& t,
                                          const Sums& r) {
    const float logs = log_sum(r);
    const bool in = t.index >= 0 && t.index < a.classes;
    a.logp[row] = t.index == a.ignore ? 0.0f
                  : !in               ? __builtin_nanf("")
                  : r.s == 0.0f       ? kNegInf
                                      : t.z - r.m - logs;
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
        if (live && slot == 0) store_row(a, row, target_of<T>(a, row), r);
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

// One tile of a row, E elements per lane, in 16-byte units interleaved over the lanes.
template <typename T, int E>
struct Tile {
    static constexpr int V = kVec<T>, U = E / V, kElems = 64 * E;
    u32x4 raw[U];
    __device__ __forceinline__ void issue(const T* row, int base, int n, int lane) {
        issue_units<0, false>(row, base + lane * V, 64 * V, n, 0u, raw);
    }
    __device__ __forceinline__ void values(int base, int n, int lane, float (&v)[E]) {
        if (base + kElems > n)
            settle_units<0, false, T>(base + lane * V, 64 * V, n, kNegInfBits<T>, raw);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float unit[V];
            widen(raw[u], unit);
#pragma unroll
            for (int i = 0; i < V; ++i) v[u * V + i] = unit[i];
        }
    }
    // The class of a lane's element e.
    static __device__ __forceinline__ int index(int base, int lane, int e) {
        return base + ((e / V) * 64 + lane) * V + e % V;
    }
};

// Offers a tile's elements to the best k (see the file's comment; vm = max_of(v)).  The
// elements are used up: an offered one becomes NaN.
template <typename T, int E>
__device__ __forceinline__ void offer_tile(Best& best, float (&v)[E], float vm, int base, int n,
                                           int lane) {
    while (true) {
        const bool reach = vm >= key_value(best.bar);
        if (__ballot(reach) == 0) return;
        int at = 0;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) at = v[e] == vm ? e : at;
        const int index = Tile<T, E>::index(base, lane, at);
        const uint64_t key = reach && index < n ? key_of(vm, index) : 0;
        const bool use = key > best.bar;
        // (only ties are left, of a higher index: the first of a lane's equal elements is its
        // lowest)
        if (__ballot(use) == 0) return;
        best.offer(key, lane);
        vm = __builtin_nanf("");
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = use && at == e ? __builtin_nanf("") : v[e];
            vm = __builtin_fmaxf(vm, v[e]);
        }
    }
}

// Where a row has fewer than k classes that are numbers: its NaN classes, lowest index
// first.
template <typename T>
__device__ __forceinline__ void offer_nan(Best& best, const T* z, int n, int lane) {
    for (int base = 0; base < n; base += 64) {
        const float v = base + lane < n ? Storage<T>::load(z + base + lane) : 0.0f;
        best.offer(v != v ? key_of(v, base + lane) : 0, lane);
    }
}

// A wave per (row, part), four per workgroup.
template <typename T, int E, bool ENT, bool TOP>
__global__ void __launch_bounds__(256) logprob_kernel(LogprobArgs a) {
    constexpr int kTile = Tile<T, E>::kElems;
    const int lane = threadIdx.x & 63, n = a.classes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t items = a.rows * a.parts;
    for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < items;
         item += (int64_t)gridDim.x * 4) {
        const int64_t row = a.parts == 1 ? item : item / a.parts;
        const T* z = static_cast<const T*>(a.z) + row * a.stride;
        Sums r = {kNegInf, 0.0f, 0.0f};
        Best best(TOP ? a.k : 1);
        int base = (int)(item - row * a.parts) * kTile;
        const int step = a.parts * kTile;
        Tile<T, E> next;
        next.issue(z, base, n, lane);
        const Target target = target_of<T>(a, row);
        // (classes and a step stay below 2^31)
        for (; base < n; base += step) {
            Tile<T, E> tile = next;
            if (base + step < n) next.issue(z, base + step, n, lane);
            float v[E];
            tile.values(base, n, lane, v);
            const float vm = max_of(v);
            add_values<ENT>(r, v, vm);
            if (TOP) offer_tile<T>(best, v, vm, base, n, lane);
        }
        join_wave(r);
        if (a.parts > 1) {
            if (lane == 0) a.part[item] = make_float4(r.m, r.s, r.q, 0.0f);
            if (TOP && lane < a.k) a.keys[item * a.k + lane] = best.mine;
            continue;
        }
        if (lane == 0) store_row(a, row, target, r);
        if (!TOP) continue;
        if (r.s != r.s && best.bar == 0) offer_nan(best, z, n, lane);
        if (lane < a.k) store_top(a, row * a.k + lane, best.mine, r);
    }
}

// Joins the parts (at most 64) of each row: one wave per row.
template <typename T>
__global__ void __launch_bounds__(64) logprob_join_kernel(LogprobArgs a) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const bool on = lane < a.parts;
    Sums r = {kNegInf, 0.0f, 0.0f};
    if (on) {
        const float4 f = a.part[row * a.parts + lane];
        r = {f.x, f.y, f.z};
    }
    // (each part's keys are sorted: the lanes offer theirs rank by rank, the next one
    // loaded ahead, until none passes)
    const uint64_t* keys = a.keys + (row * a.parts + lane) * a.k;
    uint64_t next = on && a.k > 0 ? keys[0] : 0;
    const Target target = target_of<T>(a, row);
    join_wave(r);
    if (lane == 0) store_row(a, row, target, r);
    if (a.k == 0) return;
    Best best(a.k);
    for (int j = 0; j < a.k; ++j) {
        const uint64_t key = next;
        next = on && j + 1 < a.k ? keys[j + 1] : 0;
        if (__ballot(key > best.bar) == 0) break;
        best.offer(key, lane);
    }
    const T* z = static_cast<const T*>(a.z) + row * a.stride;
    if (r.s != r.s && best.bar == 0) offer_nan(best, z, a.classes, lane);
    if (lane < a.k) store_top(a, row * a.k + lane, best.mine, r);
}

// ------------------------------------------------------------------ gradient

// What a row's gradient is made of.
struct RowGrad {
    float m, logs, d, dh, h;
    int target;  // -1: none
};

__device__ __forceinline__ RowGrad row_grad(const LogprobGradArgs& a, int64_t row) {
    const int64_t target = a.targets[row];
    const bool in = target >= 0 && target < a.classes, ignored = target == a.ignore;
    RowGrad g;
    g.m = a.stats[2 * row];
    g.logs = a.stats[2 * row + 1];
    // No class left (log s is -infinity too: the maximum passes over NaN, which log s shows): no
    // gradient, but for an invalid target, whose NaN shows in any row.  Its logits are -infinity,
    // so p and all it is multiplied by are 0.
    if (g.m == kNegInf && g.logs == kNegInf && (in || ignored)) return {0, 0, 0, 0, 0, -1};
    g.target = in && !ignored ? (int)target : -1;
    g.d = ignored ? 0.0f : in ? a.dlogp[row] : __builtin_nanf("");
    g.dh = a.dentropy != nullptr ? a.dentropy[row] : 0.0f;
    g.h = a.dentropy != nullptr ? a.entropy[row] : 0.0f;
    return g;
}

// In place: the logits to their gradients, for the classes from col on.
template <int V>
__device__ __forceinline__ void unit_grad(const RowGrad& g, int col, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float at = v[i] - g.m - g.logs;
        // (below -1e4 the weight is 0, and the entropy's term with it; NaN stays)
        const float lp = at < -1e4f ? -1e4f : at;
        const float slope = __builtin_fmaf(g.dh, lp + g.h, g.d);
        v[i] = (g.target == col + i ? g.d : 0.0f) - exp_exact(lp) * slope;
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

// One wave per (row, tile).  PAST: the gradient is stored past the caches.
template <typename T, int E, bool PAST>
__global__ void __launch_bounds__(256) logprob_grad_kernel(LogprobGradArgs a) {
    constexpr int V = kVec<T>;
    const int lane = threadIdx.x & 63, n = a.classes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t item = blockIdx.x * 4 + wave;
    if (item >= a.items) return;
    const uint32_t row = a.tiles == 1 ? item : item / a.tiles;
    const int base = (int)(item - row * a.tiles) * Tile<T, E>::kElems;
    Tile<T, E> tile;
    tile.issue(static_cast<const T*>(a.z) + row * a.stride, base, n, lane);
    const RowGrad g = row_grad(a, row);
    float v[E];
    tile.values(base, n, lane, v);
    T* dz = static_cast<T*>(a.dz) + row * a.dstride;
#pragma unroll
    for (int u = 0; u < E / V; ++u) {
        const int col = base + (u * 64 + lane) * V;
        float d[V];
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = v[u * V + i];
        unit_grad(g, col, d);
        if (base + Tile<T, E>::kElems <= n) store_unit<true, PAST>(dz, col, n, d);
        else store_unit<false, PAST>(dz, col, n, d);
    }
}

// Elements per lane of a tile: a row of one tile leaves few lanes idle.
int tile_elems(int32_t classes) { return classes <= 512 ? 8 : classes <= 1024 ? 16 : 32; }

int grid_of(int64_t n, int64_t most) { return (int)(n < most ? n : most); }

}  // namespace

LogprobPlan logprob_plan(int64_t rows, int32_t classes, int es, int k) {
    LogprobPlan p = {0, 0, 1, 0};
    const int V = 16 / es;
    if (classes <= 32 * V) {
        while (V << p.shift < classes) ++p.shift;
        return p;
    }
    p.elems = tile_elems(classes);
    const int64_t tiles = (classes + 64 * p.elems - 1) / (64 * p.elems);
    // a wave a row where rows alone give every SIMD one, else parts of rows to four (1000 x
    // 131072 bf16: 52 us in 5 parts; 2001 x 50001 39 us whole, 45 in 3 parts; four waves a row
    // take 41, and with 5 alternatives 20000 x 9000 172 us against 105, since each wave
    // begins a list of its own)
    if (rows < 1024) {
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
    if (p.elems == 0) {
        const int64_t per = 256 >> p.shift;
        logprob_short_kernel<T><<<grid_of((a.rows + per - 1) / per, 8192), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    const int grid = logprob_groups(a.rows * p.parts);
    const bool ent = a.entropy != nullptr, top = a.k > 0;
    using std::false_type;
    using std::integral_constant;
    using std::true_type;
    auto go = [&](auto e, auto ent_, auto top_) {
        logprob_kernel<T, decltype(e)::value, decltype(ent_)::value, decltype(top_)::value>
            <<<grid, 256, 0, s>>>(a);
    };
    auto pick = [&](auto e) {
        if (ent && top) go(e, true_type{}, true_type{});
        else if (ent) go(e, true_type{}, false_type{});
        else if (top) go(e, false_type{}, true_type{});
        else go(e, false_type{}, false_type{});
    };
    if (p.elems == 8) pick(integral_constant<int, 8>{});
    else if (p.elems == 16) pick(integral_constant<int, 16>{});
    else pick(integral_constant<int, 32>{});
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    logprob_join_kernel<T><<<(int)a.rows, 64, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t run_logprob_grad(LogprobGradArgs a, hipStream_t s) {
    constexpr int V = kVec<T>;
    if (a.classes <= 32 * V) {
        a.shift = 0;
        while (V << a.shift < a.classes) ++a.shift;
        const int64_t per = 256 >> a.shift;
        logprob_grad_short_kernel<T><<<grid_of((a.rows + per - 1) / per, 8192), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    const int elems = tile_elems(a.classes);
    const bool past = a.rows * a.classes * (int64_t)sizeof(T) >= kPastCaches;
    a.tiles = (a.classes + 64 * elems - 1) / (64 * elems);
    return logprob_grad_pieces(a, sizeof(T), [&](const LogprobGradArgs& piece, int grid) {
        auto go = [&](auto e) {
            constexpr int E = decltype(e)::value;
            if (past) logprob_grad_kernel<T, E, true><<<grid, 256, 0, s>>>(piece);
            else logprob_grad_kernel<T, E, false><<<grid, 256, 0, s>>>(piece);
        };
        if (elems == 8) go(std::integral_constant<int, 8>{});
        else if (elems == 16) go(std::integral_constant<int, 16>{});
        else go(std::integral_constant<int, 32>{});
        return hipGetLastError();
    });
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
