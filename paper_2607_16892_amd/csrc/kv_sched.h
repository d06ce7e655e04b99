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

#include "kv.h"
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
    int rows;      // of a tile
    int groups;    // workgroups
    int few;       // tokens
    bool below;    // the kernel of the requests of up to `few` tokens
};

constexpr int kStepKeys = 32;

__device__ __forceinline__ KvShare kv_share(const KvAttnArgs &a, const KvCut &c, int r)
{
    KvShare s{0, 0, 0, 0};
    if (r >= a.R) return s;
    const int t0 = min(max(a.start[r], 0), a.T), t1 = min(max(a.start[r + 1], 0), a.T);
    const int n = max(t1 - t0, 0);
    if (n == 0 || (n <= c.few) != c.below) return s;
    s.n = n;
    s.ctx = (int)min((long long)max(a.context[r], 0), (long long)a.W << a.shift);
    s.tiles = (int)(((long long)n * a.G + c.rows - 1) / c.rows);
    s.span = s.ctx;
    if (a.window && !a.prefix)  // a tile's rows lie within rows / G + 2 tokens
        s.span = (int)min((long long)s.ctx,
                          (long long)a.window + min(c.rows / a.G + 2, n) + kStepKeys);
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
__device__ __forceinline__ uint64_t kv_run(const KvCut &c, uint64_t all, uint32_t longest)
{
    const uint64_t least = __any(longest >= 2048) ? 8 : __any(longest >= 512) ? 4 : __any(longest >= 128) ? 2 : 1;
    if (all < 0xffff0000u) return max((uint64_t)(((uint32_t)all + (uint32_t)c.groups - 1) / (uint32_t)c.groups), least);
    return (all + c.groups - 1) / (uint32_t)c.groups;
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

// The items by their steps: from the workgroup's own scan in LDS, or, beyond
// kInlineRequests, from the exclusive sums [R + 1] of kv_plan_kernel.
struct KvSched {
    uint64_t all, run;  // all steps, and those of a workgroup

    // (all waves; the results are in LDS after it)
    __device__ __forceinline__ void init(const KvAttnArgs &a, const KvCut &c, const uint64_t *sums, KvLds &lds)
    {
        if (a.R <= kInlineRequests) {
            const int lane = threadIdx.x & 63;
            const KvShare s = kv_share(a, c, lane);
            const uint64_t upto = scan_wave(kv_units(a, s));
            all = lane_value(upto, 63);
            if (threadIdx.x < 64) {
                lds.upto[lane] = upto;
                lds.share[lane] = s;
            }
            __syncthreads();
            run = kv_run(c, all, kv_steps(s));
        } else {
            all = sums[a.R];
            run = kv_run(c, all, 1);
        }
    }

    // The item that step u (< all, uniform) belongs to.
    __device__ __forceinline__ KvItem item(const KvAttnArgs &a, const KvCut &c, const uint64_t *sums,
                                           const KvLds &lds, uint64_t u) const
    {
        KvItem w;
        KvShare s;
        uint64_t first;
        if (a.R <= kInlineRequests) {
            w.r = __builtin_ctzll(__ballot(lds.upto[threadIdx.x & 63] > u));
            first = w.r ? lds.upto[w.r - 1] : 0;
            s = lds.share[w.r];
        } else {
            w.r = __builtin_amdgcn_readfirstlane(kv_find(sums, a.R, u));
            first = sums[w.r];
            s = kv_share(a, c, w.r);
        }
        auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
        w.n = uniform(s.n);
        w.ctx = uniform(s.ctx);
        w.steps = uniform((int)kv_steps(s));
        w.first_token = uniform(min(max(a.start[w.r], 0), a.T));
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
__device__ __forceinline__ uint32_t kv_tile_steps(const KvAttnArgs &a, const KvShare &s, int r, int tile, int rows,
                                                  int keys)
{
    const int prefix = a.prefix ? a.prefix[r] : 0, row0 = tile * rows;
    const int last = min(s.n - 1, (row0 + rows - 1) / a.G);
    const int lo = kv_row_range(a, s.ctx, s.n, row0 / a.G, prefix).lo & ~31;
    const int hi = kv_row_range(a, s.ctx, s.n, last, prefix).hi;
    return (uint32_t)max((hi - lo + keys - 1) / keys, 1);
}

// An equal share of `all` steps, not below four: a part of a tile costs about as much as two
// steps to write and join (64 tokens of 8 heads over 8000 keys: 37 us, and 60 with shares down
// to one step).
__device__ __forceinline__ uint64_t kv_tile_share(const KvCut &c, uint64_t all)
{
    return max((all + (uint32_t)c.groups - 1) / (uint32_t)c.groups, (uint64_t)4);
}

// The kernels of few and of many rows a request; they zero the rows of no request as well
// if `pad`.
template <class T>
void launch_kv_decode(const KvAttnArgs &a, const KvCut &c, const uint64_t *sums, int cache_dtype, int DP,
                      bool pad, float *o, float2 *ml, KvJoin *joins, hipStream_t st);
// its waves a SIMD
int kv_decode_waves(int cache_dtype, int DP);

template <class T>
void launch_kv_prefill(const KvAttnArgs &a, const KvCut &c, const KvTiles &t, unsigned grid, int cache_dtype, int DP, bool pad,
                       float *o, float2 *ml, KvJoin *joins, hipStream_t st);
// its workgroups a compute unit, rows of a tile, and keys a step
int kv_prefill_groups(int DP);
int kv_prefill_rows(int DP);
int kv_prefill_keys(int DP);

}  // namespace dro
