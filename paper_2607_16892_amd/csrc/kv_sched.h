// How the attention's work is cut into workgroups, found by every workgroup itself.
//
// Request r has n new tokens, so n G rows a key head (G query heads each), in tiles of
// `rows` rows; an item is a tile of a key head.
//
// Few rows a request: a step is 32 keys of an item, and the steps of all items in order
// are dealt to `groups` workgroups in equal runs, so requests of any lengths load them
// alike (few rows are bound by what they read, whoever reads it).  A run that holds a whole item writes its rows; a run that begins or ends within
// an item leaves a partial result, at most two a workgroup, for the join.
#pragma once

#include <type_traits>

#include "kv.h"
#include "kv_types.h"
#include "wave.h"

namespace dro {

constexpr int kInlineRequests = 64;  // up to a wave of requests every workgroup scans them

struct KvShare {  // of one request
    int n, ctx;   // rows' tokens, and keys in the cache
    int tiles;
    int span;     // keys that a tile can see, at most (0: none)
};

struct KvItem {
    int r, n, ctx, first_token;
    int tile, head;
    int step, steps;  // the item's step asked for, and how many it has
};

// Many rows a request: the tiles of all requests are listed first (their steps differ, as a
// tile's keys end where its last row's do), a request's last tile, the longest, first.  A
// workgroup takes a tile and the hardware deals them, longest first, since beginning a tile
// takes as long as several steps and workgroups do not run at one speed.  A tile is cut into
// as many chunks as it has equal shares of all steps, a quarter aside: so one of less than 1.75
// shares stays whole and no part of it is written or joined.  (Equal runs of steps, as above,
// against this, side by side when it was chosen: a prompt of 8192 tokens, 64 heads on 8, 1546 against
// 1160 us; four prompts of 2000 tokens, 32 heads on 8, 256 against 168; four chunks of 512 tokens over
// 4000 to 8192, 281 against 244, and 320 with every tile of more than one share cut.)

// Requests of up to `few` tokens belong to the one kernel, others to the other.
struct KvCut {
    int rows = 1;  // of a tile (where the kernel is not launched, any)
    int groups;    // workgroups
    int few;       // tokens
    bool below;    // the kernel of the requests of up to `few` tokens
};

constexpr int kStepKeys = 32;

template <class A> constexpr bool kShared = __is_same(A, KvSharedArgs);
template <class A> constexpr bool kJoined = __is_same(A, KvJoinedArgs);

// The requests, or the sources of keys: the groups' prefixes, then the requests' own tokens.
template <class A> __device__ __forceinline__ int kv_requests(const A &a)
{
    if constexpr (kShared<A>) return a.groups + a.R;
    else return a.R;
}
template <class A> __device__ __forceinline__ bool kv_is_prefix(const A &a, int r)
{
    if constexpr (kShared<A>) return r < a.groups;
    else return false;
}
template <class A> __device__ __forceinline__ int kv_own(const A &a, int r)  // the request's number
{
    if constexpr (kShared<A>) return r - a.groups;
    else return r;
}
template <class A> __device__ __forceinline__ int kv_first_token(const A &a, int r)
{
    if constexpr (kShared<A>)
        if (r < a.groups) return a.p_start[r];
    return min(max(a.start[kv_own(a, r)], 0), a.T);
}
template <class A> __device__ __forceinline__ int kv_end_token(const A &a, int r)
{
    if constexpr (kShared<A>)
        if (r < a.groups) return a.p_start[r + 1];
    return min(max(a.start[kv_own(a, r) + 1], 0), a.T);
}
template <class A> __device__ __forceinline__ int kv_context(const A &a, int r)
{
    if constexpr (kShared<A>)
        if (r < a.groups) return (int)min((long long)max(a.p_context[r], 0), (long long)a.p_W << a.shift);
    return (int)min((long long)max(a.context[kv_own(a, r)], 0), (long long)a.W << a.shift);
}
template <class A> __device__ __forceinline__ const int32_t *kv_table(const A &a, int r)
{
    if constexpr (kShared<A>)
        if (r < a.groups) return a.p_table + (int64_t)r * a.p_stride;
    return a.table + (int64_t)kv_own(a, r) * a.table_stride;
}
template <class A> __device__ __forceinline__ int kv_prefix_of(const A &a, int r)  // keys that all rows see
{
    return a.prefix && !kv_is_prefix(a, r) ? a.prefix[kv_own(a, r)] : 0;
}

template <class A> __device__ __forceinline__ int kv_few(const A &a, const KvCut &c, int r)
{
    if constexpr (kShared<A>)
        if (r < a.groups) return a.p_few;
    return c.few;
}

template <class A> __device__ __forceinline__ KvShare kv_share(const A &a, const KvCut &c, int r)
{
    KvShare s{0, 0, 0, 0};
    if (r >= kv_requests(a)) return s;
    const int n = max(kv_end_token(a, r) - kv_first_token(a, r), 0);
    if (n == 0 || (n <= kv_few(a, c, r)) != c.below) return s;
    s.n = n;
    s.ctx = kv_context(a, r);
    s.tiles = (int)(((long long)n * a.G + c.rows - 1) / c.rows);
    s.span = s.ctx;
    if (kv_is_prefix(a, r)) {
        if constexpr (kShared<A>)
            if (a.ends) s.span = s.ctx - (a.ends[r].x & ~(kStepKeys - 1));
    } else if (a.window && !a.prefix) {  // a tile's rows lie within rows / G + 2 tokens
        s.span = (int)min((long long)s.ctx,
                          (long long)a.window + min(c.rows / a.G + 2, n) + kStepKeys);
    }
    return s;
}

__device__ __forceinline__ uint32_t kv_steps(const KvShare &s)
{
    return s.tiles ? (uint32_t)max((s.span + kStepKeys - 1) / kStepKeys, 1) : 0;
}
__device__ __forceinline__ uint64_t kv_units(const KvAttnArgs &a, const KvShare &s)
{
    return (uint64_t)((uint32_t)s.tiles * (uint32_t)a.H) * kv_steps(s);
}

// steps a workgroup, for `all` steps, the longest of the wave's items having `longest`.  An
// item of many steps alone would be cut so fine that the join takes longer than the steps (one
// request of 131,000 keys, 8 heads on one: 81 us with runs of one step, 34 with eight; of
// 16,000: 27 with one, 19 with two).
__device__ __forceinline__ uint64_t kv_run_of(const KvCut &c, uint64_t all, uint64_t least)
{
    if (all < 0xffff0000u) return max((uint64_t)(((uint32_t)all + (uint32_t)c.groups - 1) / (uint32_t)c.groups), least);
    return (all + c.groups - 1) / (uint32_t)c.groups;
}
__device__ __forceinline__ uint64_t kv_run(const KvCut &c, uint64_t all, uint32_t longest)
{
    return kv_run_of(c, all, __any(longest >= 2048) ? 8 : __any(longest >= 512) ? 4 : __any(longest >= 128) ? 2 : 1);
}

// First index of the ascending x[0 .. n) whose next entry exceeds v (the n-th counts as
// larger): 64 probes a step, by the whole wave.
template <class U> __device__ __forceinline__ int kv_find(const U *x, int n, U v)
{
    int lo = 0, hi = n;  // x[lo] <= v < x[hi]
    const int lane = threadIdx.x & 63;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step;
        const uint64_t above = __ballot(at >= hi || x[at] > v);
        const int k = __builtin_ctzll(above);  // lane 63 probes hi or beyond
        hi = min(lo + (k + 1) * step, hi);
        lo += k * step;
    }
    return lo;
}

// The requests' shares and sums of steps where a workgroup scans them itself.
struct KvLds {
    uint64_t upto[kInlineRequests];  // inclusive
    KvShare share[kInlineRequests];
};
// Requests that read their prefixes themselves: a request's keys are on one axis, its prefix's `keys`
// from 0 on and its own from `own` on, the next multiple of a step.
struct KvPrefix {
    int group, keys, own;
};
struct KvJoinedLds : KvLds {
    KvPrefix prefix[kInlineRequests];
    int32_t first[kInlineRequests + 1];
};
template <class A> using KvLdsOf = std::conditional_t<kJoined<A>, KvJoinedLds, KvLds>;

// The items by their steps: from the workgroup's own scan in LDS, or, beyond
// kInlineRequests and behind shared prefixes, from the exclusive sums [n + 2] of a launch before
// (the last: steps a workgroup).
template <class A> struct KvSched {
    uint64_t all, run;  // all steps, and those of a workgroup

    static __device__ __forceinline__ bool scanned(const A &a) { return !kShared<A> && a.R <= kInlineRequests; }

    // (all waves; the results are in LDS after it)
    __device__ __forceinline__ void init(const A &a, const KvCut &c, const uint64_t *sums, KvLdsOf<A> &lds)
    {
        if (scanned(a)) {
            const int lane = threadIdx.x & 63;
            KvShare s = kv_share(a, c, lane);
            if constexpr (kJoined<A>) {  // (a wave; up to 64 groups)
                for (int g = lane; g <= a.groups; g += 64) lds.first[g] = a.first[g];
                __syncthreads();
                int g = 0;
                for (int hi = a.groups; hi - g > 1;) {
                    const int m = (g + hi) >> 1;
                    if (lds.first[m] <= lane) g = m;
                    else hi = m;
                }
                KvPrefix p{g, 0, 0};
                if (lds.first[g] <= lane && lane < lds.first[g + 1])
                    p.keys = (int)min((long long)max(a.p_context[g], 0), (long long)a.p_W << a.shift);
                p.own = (p.keys + kStepKeys - 1) & ~(kStepKeys - 1);
                lds.prefix[lane] = p;
                s.span += p.own;
            }
            const uint64_t upto = scan_wave(kv_units(a, s));
            all = lane_value(upto, 63);
            if (threadIdx.x < 64) {
                lds.upto[lane] = upto;
                lds.share[lane] = s;
            }
            __syncthreads();
            run = kv_run(c, all, kv_steps(s));
        } else {
            all = sums[kv_requests(a)];
            run = kShared<A> ? sums[kv_requests(a) + 1] : kv_run(c, all, 1);
        }
    }

    // The item that step u (< all, uniform) belongs to.
    __device__ __forceinline__ KvItem item(const A &a, const KvCut &c, const uint64_t *sums,
                                           const KvLdsOf<A> &lds, uint64_t u) const
    {
        KvItem w;
        KvShare s;
        uint64_t first;
        if (scanned(a)) {
            w.r = __builtin_ctzll(__ballot(lds.upto[threadIdx.x & 63] > u));
            first = w.r ? lds.upto[w.r - 1] : 0;
            s = lds.share[w.r];
        } else {
            w.r = __builtin_amdgcn_readfirstlane(kv_find(sums, kv_requests(a), u));
            first = sums[w.r];
            s = kv_share(a, c, w.r);
        }
        auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
        w.n = uniform(s.n);
        w.ctx = uniform(s.ctx);
        w.steps = uniform((int)kv_steps(s));
        w.first_token = uniform(kv_first_token(a, w.r));
        const uint64_t local = u - first;
        uint32_t item;
        if (local < 0xffffffffu) item = (uint32_t)local / (uint32_t)w.steps;
        else item = (uint32_t)(local / (uint32_t)w.steps);
        item = uniform(item);
        w.step = uniform((int)(local - (uint64_t)item * (uint32_t)w.steps));
        const uint32_t tiles = uniform(s.tiles);
        w.head = uniform(item / tiles);
        w.tile = uniform(item - (uint32_t)w.head * tiles);
        return w;
    }
};

// An item in parts, for the join.
struct KvJoin {
    int parts;  // 0: nothing to join here
    int first_token, row0, rows, head;
    int first, next, stride;  // places of part 0, of part 1, and from there on
};

// Place of a run's partial result: the run that an item begins in, or a later one.
__device__ __forceinline__ int kv_part(uint32_t group, bool begins) { return 2 * (int)group + begins; }

// The keys of a tile and of its rows: row `i` (of n G) sees [lo, hi).
struct KvRange {
    int lo, hi;
};
__device__ __forceinline__ KvRange kv_row_range(const KvAttnArgs &a, int ctx, int n, int token, int prefix)
{
    const int p = ctx - n + token;  // negative where the cache holds fewer tokens than there are rows
    KvRange v;
    v.hi = min(max(p + 1, prefix), ctx);
    v.lo = a.window ? max(p - a.window + 1, 0) : 0;
    return v;
}
// The same of a row of request or group r; it is row t of the call's.  A shared prefix is seen by
// all rows of its group, but for a window by their places.
template <class A>
__device__ __forceinline__ KvRange kv_see(const A &a, int r, int ctx, int n, int token, int prefix, int t)
{
    if (!kv_is_prefix(a, r)) return kv_row_range(a, ctx, n, token, prefix);
    KvRange v{0, ctx};
    if constexpr (kShared<A>)
        if (a.ends) v.lo = (int)min(max((long long)ctx + a.row_pos[t] - a.p_window + 1, 0LL), (long long)ctx);
    return v;
}
// The same of the first and of the last of some rows: up to where none of them sees keys, and from
// where on all do.
template <class A>
__device__ __forceinline__ KvRange kv_first_range(const A &a, int r, int ctx, int n, int token, int prefix)
{
    if (!kv_is_prefix(a, r)) return kv_row_range(a, ctx, n, token, prefix);
    KvRange v{0, ctx};
    if constexpr (kShared<A>)
        if (a.ends) v.lo = a.ends[r].x;
    return v;
}
template <class A>
__device__ __forceinline__ KvRange kv_last_range(const A &a, int r, int ctx, int n, int token, int prefix)
{
    if (!kv_is_prefix(a, r)) return kv_row_range(a, ctx, n, token, prefix);
    KvRange v{0, ctx};
    if constexpr (kShared<A>)
        if (a.ends) v.lo = a.ends[r].y;
    return v;
}
// A row's place, counted from its source's first key, for a bias by distance.
template <class A> __device__ __forceinline__ int kv_row_place(const A &a, int r, int ctx, int n, int token, int t)
{
    if constexpr (kShared<A>)
        if (r < a.groups) return ctx + a.row_pos[t];
    return ctx - n + token;
}
// Where a finished row of sums goes that is joined with its other source's.
template <class A> struct KvRaw {
    float *o;
    float2 *ml;
};
template <class A> __device__ __forceinline__ KvRaw<A> kv_raw(const A &a, int r)
{
    if constexpr (kShared<A>) return {a.raw_o[r >= a.groups], a.raw_ml[r >= a.groups]};
    else return {nullptr, nullptr};
}

// ---- many rows a request ------------------------------------------------------------

constexpr int kDies = 8;  // workgroups go to the dies (an L2 each) in turn

struct KvTile {
    int r, tile;
    int n, ctx, first_token;  // of the request
    int steps;
    int part;    // place of its first partial result, of head 0
    int chunks;  // 1: whole
    uint32_t before;  // chunks of the tiles before it
};
struct KvTileList {  // (one load)
    int count;  // tiles
    int parts;  // partial results of a head
    uint32_t all;  // chunks of a head (fewer than 2^26 over all heads)
};
struct KvTiles {
    const uint32_t *sums;  // [count + 1] exclusive sums of the tiles' chunks
    const KvTile *tiles;   // [count]
    const KvTileList *list;
};

// Steps of `keys` keys of a tile.
template <class A>
__device__ __forceinline__ uint32_t kv_tile_steps(const A &a, const KvShare &s, int r, int tile, int rows, int keys)
{
    const int prefix = kv_prefix_of(a, r), row0 = tile * rows;
    const int last = min(s.n - 1, (row0 + rows - 1) / a.G);
    const int lo = kv_first_range(a, r, s.ctx, s.n, row0 / a.G, prefix).lo & ~31;
    const int hi = kv_last_range(a, r, s.ctx, s.n, last, prefix).hi;
    return (uint32_t)max((hi - lo + keys - 1) / keys, 1);
}

// An equal share of `all` steps, not below four: a part of a tile costs about as much as two
// steps to write and join (64 tokens of 8 heads over 8000 keys: 37 us, and 60 with shares down
// to one step).
__device__ __forceinline__ uint64_t kv_tile_share(const KvCut &c, uint64_t all)
{
    return max((all + (uint32_t)c.groups - 1) / (uint32_t)c.groups, (uint64_t)4);
}

// What a kernel over a cache of type C takes, of arguments A (KvMxArgs, KvSharedArgs or KvJoinedArgs).
template <class A, class C> using KvKernelArgs = std::conditional_t<kShared<A> || kJoined<A> || kMx<C>, A, KvAttnArgs>;

// The kernels of few and of many rows a request; they zero the rows of no request as well
// if `pad`.
template <class T, class A>
void launch_kv_decode(const A &a, const KvCut &c, const uint64_t *sums, int cache_dtype, int DP,
                      bool pad, float *o, float2 *ml, KvJoin *joins, hipStream_t st);
// its waves a SIMD
int kv_decode_waves(int cache_dtype, int DP);

template <class T, class A>
void launch_kv_prefill(const A &a, const KvCut &c, const KvTiles &t, unsigned grid, int cache_dtype, int DP, bool pad,
                       float *o, float2 *ml, KvJoin *joins, hipStream_t st);
// its workgroups a compute unit, rows of a tile, and keys a step
int kv_prefill_groups(int DP);
int kv_prefill_rows(int DP);
int kv_prefill_keys(int DP);

}  // namespace dro
