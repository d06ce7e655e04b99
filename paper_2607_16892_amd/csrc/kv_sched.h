// How the attention's work is cut into workgroups, found by every workgroup itself.
//
// Request r has n new tokens, so n G rows a key head (G query heads each), in tiles of
// `rows` rows, and spans the keys that its rows can see.  Its tiles' keys are cut into
// chunks of C keys, where C spreads the keys of all tiles over about 2^target_log2
// workgroups: one long request beside short ones is split, and many requests of about
// one length are not.  A request of one chunk writes its rows; the chunks of others
// leave partial results, fewer than 2^(target_log2 + 1) of them since a request that is
// cut has more than C keys a tile.
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
    int r, n, ctx, first_token, tiles, tile, head, chunk, chunks;
    int C;        // keys a chunk
    int partial;  // place of the chunk's partial result (chunks > 1)
};

// Requests of up to `few` tokens belong to the one kernel, others to the other.
struct KvCut {
    int rows;         // of a tile
    int align;        // keys a chunk is a multiple of
    int target_log2;
    int few;          // tokens
    bool below;       // the kernel of the requests of up to `few` tokens
};

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
                          (long long)a.window + min(c.rows / a.G + 2, n) + c.align);
    return s;
}

// Keys a chunk, from the keys of all tiles.
__device__ __forceinline__ int kv_chunk(const KvCut &c, uint64_t keys)
{
    const uint64_t x = ((keys >> c.target_log2) + c.align) / c.align * c.align;
    return (int)min(x, (uint64_t)0x7fffff00);
}

__device__ __forceinline__ int kv_chunks(const KvShare &s, int C)
{
    return s.tiles ? max((s.span + C - 1) / C, 1) : 0;
}

// The scan's results for R > kInlineRequests, from kv_plan_kernel.
struct KvPlan {
    const uint32_t *items;     // [R + 1] exclusive sums of the requests' items
    const uint32_t *partials;  // [R + 1] and of their partial results
    const int *C;
};

// First index of the ascending x[0 .. n] whose next entry exceeds v (x[n] > v): 64 probes a step.
__device__ __forceinline__ int kv_find(const uint32_t *x, int n, uint32_t v)
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

// The work of workgroup b (uniform); false: none.  Workgroups b, b + 8, .. run on one
// die, which gets consecutive items: the tiles of a request's head share their keys in
// its L2.
__device__ __forceinline__ bool kv_item(const KvAttnArgs &a, const KvCut &c, const KvPlan &p, uint32_t b,
                                        KvItem &w)
{
    const int lane = threadIdx.x & 63;
    uint32_t all, local;
    KvShare s;
    auto place = [&](uint32_t &i) {
        const uint32_t each = (all + 7) / 8;
        i = (b & 7) * each + (b >> 3);
        return (b >> 3) < each && i < all;
    };
    if (a.R <= kInlineRequests) {
        s = kv_share(a, c, lane);
        const uint64_t keys = scan_wave((uint64_t)s.tiles * (uint64_t)s.span * (uint64_t)a.H);
        w.C = kv_chunk(c, lane_value(keys, 63));
        const int chunks = kv_chunks(s, w.C);
        const uint32_t items = (uint32_t)s.tiles * (uint32_t)chunks * (uint32_t)a.H;
        const uint32_t part = chunks > 1 ? items : 0;
        const uint32_t upto = scan_wave(items), pupto = scan_wave(part);
        all = lane_value(upto, 63);
        uint32_t i;
        if (!place(i)) return false;
        w.r = __builtin_ctzll(__ballot(upto > i));
        local = i - lane_value(upto - items, w.r);
        w.partial = (int)lane_value(pupto - part, w.r);
        w.n = (int)lane_value((uint32_t)s.n, w.r);
        w.ctx = (int)lane_value((uint32_t)s.ctx, w.r);
        w.tiles = (int)lane_value((uint32_t)s.tiles, w.r);
        w.chunks = (int)lane_value((uint32_t)chunks, w.r);
    } else {
        all = p.items[a.R];
        uint32_t i;
        if (!place(i)) return false;
        w.r = __builtin_amdgcn_readfirstlane(kv_find(p.items, a.R, i));
        w.C = p.C[0];
        s = kv_share(a, c, w.r);
        local = i - p.items[w.r];
        w.partial = (int)p.partials[w.r];
        w.n = s.n;
        w.ctx = s.ctx;
        w.tiles = s.tiles;
        w.chunks = kv_chunks(s, w.C);
    }
    w.first_token = min(max(a.start[w.r], 0), a.T);
    w.partial += (int)local;
    // tiles within chunks within heads
    const uint32_t per_head = (uint32_t)w.tiles * (uint32_t)w.chunks;
    w.head = (int)(local / per_head);
    local -= (uint32_t)w.head * per_head;
    w.chunk = (int)(local / (uint32_t)w.tiles);
    w.tile = (int)(local - (uint32_t)w.chunk * (uint32_t)w.tiles);
    return true;
}

// The partial results of a row: one of its request's per chunk.
struct KvParts {
    int chunks;      // <= 1: none, the row is written already
    int64_t first;   // of chunk 0, in rows
    int64_t stride;  // from chunk to chunk, in rows
};
__device__ __forceinline__ KvParts kv_row_parts(const KvAttnArgs &a, const KvCut &c, const KvPlan &p, int t,
                                                int hq)
{
    const int lane = threadIdx.x & 63;
    KvShare s;
    int r, chunks, part0;
    if (a.R <= kInlineRequests) {
        s = kv_share(a, c, lane);
        const uint64_t keys = scan_wave((uint64_t)s.tiles * (uint64_t)s.span * (uint64_t)a.H);
        const int C = kv_chunk(c, lane_value(keys, 63));
        chunks = kv_chunks(s, C);
        const uint32_t part = chunks > 1 ? (uint32_t)s.tiles * (uint32_t)chunks * (uint32_t)a.H : 0;
        const uint32_t pupto = scan_wave(part);
        const uint64_t mine = __ballot(lane < a.R && s.tiles && a.start[min(lane, a.R)] <= t &&
                                       t < a.start[min(lane, a.R - 1) + 1]);
        if (!mine) return KvParts{0, 0, 0};
        r = __builtin_ctzll(mine);
        part0 = (int)lane_value(pupto - part, r);
        s.tiles = (int)lane_value((uint32_t)s.tiles, r);
        chunks = (int)lane_value((uint32_t)chunks, r);
    } else {
        if (t < a.start[0] || t >= a.start[a.R]) return KvParts{0, 0, 0};
        r = __builtin_amdgcn_readfirstlane(kv_find((const uint32_t *)a.start, a.R, (uint32_t)t));
        s = kv_share(a, c, r);
        chunks = kv_chunks(s, p.C[0]);
        part0 = (int)p.partials[r];
    }
    if (chunks <= 1) return KvParts{0, 0, 0};
    const int h = hq / a.G, row = (t - a.start[r]) * a.G + hq - h * a.G, tile = row / c.rows;
    if (tile >= s.tiles) return KvParts{0, 0, 0};
    KvParts x;
    x.chunks = chunks;
    x.stride = (int64_t)s.tiles * c.rows;
    x.first = ((int64_t)part0 + (int64_t)h * chunks * s.tiles + tile) * c.rows + row - tile * c.rows;
    return x;
}

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

// Workgroups [first, first + n) of the kernel of few rows a request; `pad`: they zero the
// rows of no request as well.
template <class T>
void launch_kv_decode(const KvAttnArgs &a, const KvCut &c, const KvPlan &p, int cache_dtype, int DP,
                      uint32_t first, uint32_t n, bool pad, float *o, float2 *ml, hipStream_t st);

}  // namespace dro
