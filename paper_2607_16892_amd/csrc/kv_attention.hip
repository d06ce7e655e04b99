// Attention over the paged cache: the plan of many requests, the join of partial
// results, and the choice of kernels.
#include <algorithm>
#include <type_traits>

#include "kv_math.h"
#include "kv_sched.h"

namespace dro {

// ---- plan -----------------------------------------------------------------------
//
// Sums over more requests than a wave scans (kInlineRequests): one workgroup.

constexpr int kPlanThreads = 1024;

static __device__ uint64_t plan_scan(uint64_t x, uint64_t *part, uint64_t &total)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    x = scan_wave(x);
    if (lane == 63) part[wave] = x;
    __syncthreads();
    static_assert(kPlanThreads / 64 == 16, "a row of lanes");
    const uint64_t waves = scan_row16(lane < 16 ? part[lane] : 0);  // the waves' sums, one a lane
    total = lane_value(waves, 15);
    if (wave) x += lane_value(waves, __builtin_amdgcn_readfirstlane(wave) - 1);
    __syncthreads();
    return x;
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(const KvAttnArgs a, const KvCut cut, uint64_t *sums)
{
    __shared__ uint64_t part[kPlanThreads / 64];
    const int per = (a.R + kPlanThreads - 1) / kPlanThreads;
    const int r0 = min((int)threadIdx.x * per, a.R), r1 = min(r0 + per, a.R);
    uint64_t units = 0, total;
    for (int r = r0; r < r1; ++r) units += kv_units(a, kv_share(a, cut, r));
    uint64_t at = plan_scan(units, part, total) - units;
    for (int r = r0; r < r1; ++r) {
        sums[r] = at;
        at += kv_units(a, kv_share(a, cut, r));
    }
    if (threadIdx.x == 0) sums[a.R] = total;
}

// The tiles of the requests of many rows and the sums of their chunks: first the tiles before
// each request, then the list and its steps, then the chunks, 1024 tiles at a time.
__global__ __launch_bounds__(kPlanThreads) void kv_tiles_kernel(const KvAttnArgs a, const KvCut cut, int keys, int most,
                                                                uint64_t *before, uint32_t *sums, KvTile *tiles,
                                                                KvTileList *list)
{
    __shared__ uint64_t part[kPlanThreads / 64];
    __shared__ uint32_t steps_at[kPlanThreads];
    __shared__ uint32_t before_lds[kPlanThreads];  // up to a request a thread: a search in LDS
    __shared__ KvShare share_lds[kPlanThreads];
    const bool lds = a.R <= kPlanThreads;
    const int per = (a.R + kPlanThreads - 1) / kPlanThreads;
    const int r0 = min((int)threadIdx.x * per, a.R), r1 = min(r0 + per, a.R);
    uint64_t own = 0, total;
    KvShare s0{};
    for (int r = r0; r < r1; ++r) {
        s0 = kv_share(a, cut, r);
        own += s0.tiles;
    }
    uint64_t at = plan_scan(own, part, total) - own;
    if (lds) {
        before_lds[threadIdx.x] = (uint32_t)min(at, (uint64_t)0xffffffff);
        share_lds[threadIdx.x] = s0;
    } else {
        for (int r = r0; r < r1; ++r) {
            before[r] = at;
            at += kv_share(a, cut, r).tiles;
        }
    }
    __syncthreads();  // (makes `before` visible to the workgroup)
    const int n = (int)min(total, (uint64_t)most);
    uint64_t steps_all = 0;
    KvTile mine{};
    for (int e0 = 0; e0 < n; e0 += kPlanThreads) {
        const int e = e0 + threadIdx.x;
        uint32_t steps = 0;
        if (e < n) {
            int lo = 0, hi = a.R;  // the last request with before[r] <= e: it has tiles
            while (hi - lo > 1) {
                const int m = (lo + hi) >> 1;
                if ((lds ? before_lds[m] : before[m]) <= (uint64_t)e) lo = m;
                else hi = m;
            }
            const KvShare s = lds ? share_lds[lo] : kv_share(a, cut, lo);
            const int tile = max(s.tiles - 1 - (e - (int)(lds ? before_lds[lo] : before[lo])), 0);
            steps = kv_tile_steps(a, s, lo, tile, cut.rows, keys);
            mine = KvTile{lo, tile, s.n, s.ctx, min(max(a.start[lo], 0), a.T), (int)steps, 0, 1, 0};
            tiles[e] = mine;
        }
        plan_scan(steps, part, total);
        steps_all += total;
    }
    const uint64_t share = kv_tile_share(cut, steps_all * a.H);
    // Where not all tiles run at once and one pass holds them, they go by quarters of a share, the
    // longest first, so that none of them is waited for alone (128 requests of 500 to 4000 keys, three
    // tokens of 8 heads to each of 8: 206 us as they come, so 180; six prompts of 300 to 2000 tokens, 12
    // heads of 64 components: 48 and 45; 31 single tokens beside 9 chunks: 59 and 60).
    const bool sort = n <= kPlanThreads &&
                      (__syncthreads_or(mine.steps + share / 4 >= 2 * share) || n * a.H > cut.groups);
    if (sort) {
        const bool is = (int)threadIdx.x < n;
        const int shift = (int)(3 - min((uint64_t)mine.steps * 4 / share, (uint64_t)3)) * 16;
        const uint64_t one = is ? 1ull << shift : 0, upto = plan_scan(one, part, total) - one;
        uint32_t to = (uint32_t)(upto >> shift) & 0xffff;
        for (int s = 0; s < shift; s += 16) to += (uint32_t)(total >> s) & 0xffff;
        if (is) {
            tiles[to] = mine;
            steps_at[to] = mine.steps;
        }
        __syncthreads();
    }
    // Chunks: of the tiles that are cut, with 1.75 shares or more, a tile has at most 8/7 as many
    // as shares, so there are fewer than 2 `groups` of them over all heads.
    uint32_t all = 0, parts = 0;
    for (int e0 = 0; e0 < n; e0 += kPlanThreads) {
        const int e = e0 + threadIdx.x;
        const uint32_t steps = e >= n ? 0 : sort ? steps_at[e] : tiles[e].steps;  // (tiles: this thread's)
        const uint64_t chunks = e < n ? max((steps + share / 4) / share, (uint64_t)1) : 0;
        const uint64_t count = chunks > 1 ? chunks | chunks << 32 : chunks;
        const uint64_t upto = plan_scan(count, part, total) - count;
        if (e < n) {
            sums[e] = tiles[e].before = all + (uint32_t)upto;
            tiles[e].part = (int)(parts + (uint32_t)(upto >> 32));
            tiles[e].chunks = (int)chunks;
        }
        all += (uint32_t)total;
        parts += (uint32_t)(total >> 32);
    }
    if (threadIdx.x == 0) {
        sums[n] = all;
        *list = KvTileList{n, (int)parts, all};
    }
}

// ---- join -------------------------------------------------------------------------
//
// Workgroup (b, y): for each of the PER entries from b PER on that has parts, rows of the item
// from its partial results.  The kernel before left the entries.  Up to kFewParts parts
// a wave joins as many rows as its lanes reach with 16 bytes each; more (a long request alone)
// the waves share, a workgroup to a row (with 16 in its place 64 tokens of 8 heads over 8000 keys
// take 67 us, so 37).  Bound by latency (the parts come from other dies' caches), so a wave asks
// for several parts at once.

// The running join of a row's parts, V components a lane.
template <int V> struct RowSum {
    float m, l, o[V];
    __device__ __forceinline__ void clear()
    {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = 0.0f;
    }
    __device__ __forceinline__ void add(float2 x, const float *z)
    {
        if (x.y == 0.0f) return;  // no key that the row sees
        float f;
        const float by = join_scales(m, l, x, f);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = o[j] * by + f * z[j];
    }
    // parts c, c + by, .. of row y, AHEAD at once, components from d on
    template <int DP, int AHEAD>
    __device__ __forceinline__ void sum(const KvJoin &it, int tile_rows, const float *part_o, const float2 *part_ml,
                                        int y, int d, int c, int by)
    {
        for (; c < it.parts; c += by * AHEAD) {
            float2 x[AHEAD];
            Vec<float, V> z[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int n = min(c + i * by, it.parts - 1);
                const int64_t at = (int64_t)(n == 0 ? it.first : it.next + (n - 1) * it.stride) * tile_rows + y;
                x[i] = part_ml[at];
                z[i] = *(const Vec<float, V> *)(part_o + at * DP + d);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (c + i * by < it.parts) {
                    float w[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) w[j] = z[i][j];
                    add(x[i], w);
                }
        }
    }
    template <class T, int DP>
    __device__ __forceinline__ void write(const KvAttnArgs &a, const KvJoin &it, int y, int d)
    {
        const int row = it.row0 + y, token = row / a.G, hq = it.head * a.G + row - token * a.G;
        const int64_t t = it.first_token + token, row_at = t * a.Hq + hq;
        if (a.with_ml) {  // behind a shared prefix
            const float2 x = a.with_ml[row_at];
            if (x.y != 0.0f) {
                const Vec<float, V> z = *(const Vec<float, V> *)(a.with_o + row_at * DP + d);
                float w[V];
#pragma unroll
                for (int j = 0; j < V; ++j) w[j] = ((const float *)&z)[j];
                add(x, w);
            }
        }
        if (a.raw_ml) {  // over one
            Vec<float, V> z;
#pragma unroll
            for (int j = 0; j < V; ++j) ((float *)&z)[j] = o[j];
            *(Vec<float, V> *)(a.raw_o + row_at * DP + d) = z;
            if (d == 0) a.raw_ml[row_at] = make_float2(m, l);
            return;
        }
        const float inv = l == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[it.head] : 1.0f) / l;
        T *out = (T *)a.out + t * a.out_token + hq * a.out_head + d;
        if constexpr (V == 4) {  // (the dimension is a multiple of 8)
            if (d < a.D)
                *(uint2 *)out = l == 0.0f ? make_uint2(0, 0) : make_uint2(pack2<T>(o[0] * inv, o[1] * inv),
                                                                          pack2<T>(o[2] * inv, o[3] * inv));
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (d + j < a.D) out[j] = (T)(l == 0.0f ? 0.0f : o[j] * inv);
        }
        if (a.lse && d == 0) a.lse[row_at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
};

template <class T, int DP, int WAVES, int PER>
__global__ __launch_bounds__(WAVES * 64) void kv_join_kernel(const KvAttnArgs a, int tile_rows, int entries,
                                                             const float *part_o, const float2 *part_ml,
                                                             const KvJoin *joins)
{
    constexpr int V = DP / 64, Lanes = DP / 4, Rows = 64 / Lanes;
    constexpr int kFewParts = 64;
    __shared__ float2 red[WAVES];
    __shared__ float acc[WAVES][DP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t one = 0, many = 0;  // entries whose rows a wave joins, and the others
    {
        const int e = blockIdx.x * PER + lane;
        static_assert(PER <= 64, "a lane per entry");
        const int parts = lane < PER && e < entries ? joins[e].parts : 0;
        one = __ballot(parts > 0 && parts <= kFewParts);
        many = __ballot(parts > kFewParts);
    }
    // with several entries the waves take them in turn, with one its rows
    const int d = lane % Lanes * 4, mine = PER > 1 ? wave : 0, y_waves = PER > 1 ? 1 : WAVES;
    const int y0 = (blockIdx.y * y_waves + (PER > 1 ? 0 : wave)) * Rows + lane / Lanes;
    for (int nth = 0; one; one &= one - 1, ++nth) {
        if (PER > 1 && nth % WAVES != mine) continue;
        const KvJoin it = joins[blockIdx.x * PER + __builtin_ctzll(one)];
        for (int y = y0; y < it.rows; y += gridDim.y * y_waves * Rows) {
            RowSum<4> s;
            s.clear();
            if (it.parts <= 2) s.sum<DP, 2>(it, tile_rows, part_o, part_ml, y, d, 0, 1);
            else s.sum<DP, 8>(it, tile_rows, part_o, part_ml, y, d, 0, 1);
            s.template write<T, DP>(a, it, y, d);
        }
    }
    for (; many; many &= many - 1) {
        const KvJoin it = joins[blockIdx.x * PER + __builtin_ctzll(many)];
        for (int y = blockIdx.y; y < it.rows; y += gridDim.y) {
            RowSum<V> s;
            s.clear();
            s.template sum<DP, 8>(it, tile_rows, part_o, part_ml, y, lane * V, wave, WAVES);
            if (lane == 0) red[wave] = make_float2(s.m, s.l);
            for (int j = 0; j < V; ++j) acc[wave][lane * V + j] = s.o[j];
            __syncthreads();
            if (wave == 0) {
                for (int w = 1; w < WAVES; ++w) s.add(red[w], &acc[w][lane * V]);
                s.template write<T, DP>(a, it, y, lane * V);
            }
            __syncthreads();
        }
    }
}

// ---- launches -----------------------------------------------------------------------

static int padded_dim(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// Requests of up to this many rows a key head are the kernel's for few rows, others the other's:
// one of its tiles.  Where the calls are small, two, as they have no list of tiles to wait for.
// (128 requests of 500 to 4000 keys, 24 rows a key head: one tile 180 us, two 314; 32 of 1000 to
// 8000, 32 rows: 58 and 75; one of 1000, 32 rows: 20 and 15.)
static int few_rows(const KvAttnArgs &a) { return (int64_t)a.R * a.H < 16 ? 32 : 16; }

constexpr int kFewRequests = 64;

struct KvPlans {
    KvCut few, many;       // groups == 0: not launched
    int most_tiles;        // of the requests of many rows
    unsigned grid;
};

static KvPlans plans(const KvAttnArgs &a, int cache_dtype)
{
    const int DP = padded_dim(a.D), few = std::max(few_rows(a) / a.G, 1);
    const bool all_few = a.max_new <= few;
    // The one kernel takes all with so many rows that each request has more than few (by max_new,
    // so that a bound that does not hold loses no request), and where there are few requests: the
    // other's two launches and its reading beside no products cost more than it mostly saves (31 single
    // tokens beside 9 chunks of 33 to 300, 8 heads on 4 of 256 components: 78 us by both, so 60; 58
    // beside two of 512 over 500 to 8000 keys, 32 heads on 8: 220 and 187; 30 beside 30: 812 and 786;
    // 30 beside two of 100 to 300: 139 and 124).  It loses where a long chunk's tiles fill the compute
    // units and a single token's tile waits for them: one beside a chunk of 500 over 60,000 keys, 546 us
    // by both, so 722.  The contexts that tell the two apart are on the device.
    const bool all_many = !all_few && (a.R <= kFewRequests || a.T > (int64_t)(a.R - 1) * a.max_new + few);
    KvPlans p{};
    if (!all_many) {
        p.few.rows = 16;
        p.few.groups = a.num_cu * 4 * kv_decode_waves(cache_dtype, DP);
        p.few.few = all_few ? 0x7fffffff : few;
        p.few.below = true;
    }
    if (!all_few) {
        p.many.rows = kv_prefill_rows(DP);
        p.many.groups = a.num_cu * kv_prefill_groups(DP) / kDies * kDies;
        p.many.few = all_many ? 0 : few;
        p.many.below = false;
        p.most_tiles = (int)((int64_t)a.T * a.G / p.many.rows + std::min(a.R, all_many ? a.T : a.T / (few + 1) + 1));
        const int64_t items = (int64_t)p.most_tiles * a.H;
        // a workgroup to a chunk (2^23 of 256 threads are a grid's limit at half)
        p.grid = (unsigned)std::min<int64_t>((items + 2 * p.many.groups + kDies) / kDies * kDies, 1 << 23);
    }
    return p;
}

struct KvWork {
    float *o;
    float2 *ml;
    KvJoin *joins;
    uint64_t *sums;    // few rows: [R + 1]
    uint64_t *before;
    uint32_t *tile_sums;
    KvTile *tiles;
    KvTileList *list;
    size_t bytes;
};

static KvWork work_of(const KvAttnArgs &a, const KvPlans &p, void *ws)
{
    KvWork w{};
    char *at = (char *)ws;
    auto take = [&](size_t bytes) {
        char *q = at;
        at += (bytes + 255) & ~size_t(255);
        return q;
    };
    // the kernels run one after the other: their partial results share one place
    const size_t rows = (size_t)2 * std::max((size_t)p.few.groups * p.few.rows, (size_t)p.many.groups * p.many.rows);
    w.o = (float *)take(rows * padded_dim(a.D) * 4);
    w.ml = (float2 *)take(rows * 8);
    w.joins = (KvJoin *)take(std::max(p.few.groups, 2 * p.many.groups) * sizeof(KvJoin));
    w.sums = (uint64_t *)take(((size_t)a.R + 1) * 8);
    if (p.many.groups) {
        w.before = (uint64_t *)take((size_t)a.R * 8);
        w.tile_sums = (uint32_t *)take(((size_t)p.most_tiles + 1) * 4);
        w.tiles = (KvTile *)take((size_t)p.most_tiles * sizeof(KvTile));
        w.list = (KvTileList *)take(sizeof(KvTileList));
    }
    w.bytes = at - (char *)ws;
    return w;
}

size_t kv_attention_bytes(const KvAttnArgs &a, int cache_dtype)
{
    return work_of(a, plans(a, cache_dtype), nullptr).bytes;
}

template <class T> static void launch_join(const KvAttnArgs &a, const KvCut &c, int entries, int most_tiles, const KvWork &w, int DP,
                        hipStream_t st)
{
    // Items so few that each may have more than 64 parts are few among the entries too: eight waves
    // to a row, 32 entries a workgroup.  Else a workgroup to an entry or four and as many rows as
    // it joins at once.  (The call with sixteen waves 32 us, with eight 24,
    // for 32 requests of 1000 to 8000 keys, two tokens of eight heads to one key head of 64
    // components each.)
    const unsigned most = (unsigned)std::max<int64_t>(1, std::min<int64_t>((int64_t)a.max_new * a.G, c.rows));
    const int64_t items = (c.rows == 16 ? (int64_t)a.R : (int64_t)most_tiles) * a.H;
    const bool few = items * 64 <= c.groups;
    const unsigned at_once = 4 * (256 / DP);  // rows of four waves
    const unsigned rows = (most + at_once - 1) / at_once;
    auto pick = [&](auto waves, auto per, unsigned y) {
        constexpr int W = decltype(waves)::value, P = decltype(per)::value;
        auto kernel = DP == 64 ? kv_join_kernel<T, 64, W, P> : DP == 128 ? kv_join_kernel<T, 128, W, P>
                                                                         : kv_join_kernel<T, 256, W, P>;
        kernel<<<dim3((entries + P - 1) / P, y), W * 64, 0, st>>>(a, c.rows, entries, w.o, w.ml, w.joins);
    };
    if (few) pick(std::integral_constant<int, 8>{}, std::integral_constant<int, 32>{}, most);
    else if (c.rows == 16) pick(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{}, rows);
    else pick(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{}, 2 * rows);
}

template <class T>
static void run_attention(const KvAttnArgs &a, const KvPlans &p, const KvWork &w, int cache_dtype, bool pad, hipStream_t st)
{
    const int DP = padded_dim(a.D);
    if (p.many.groups) {
        kv_tiles_kernel<<<1, kPlanThreads, 0, st>>>(a, p.many, kv_prefill_keys(DP), p.most_tiles,
                                                    w.before, w.tile_sums, w.tiles, w.list);
        const KvTiles t{w.tile_sums, w.tiles, w.list};
        launch_kv_prefill<T>(a, p.many, t, p.grid, cache_dtype, DP, pad, w.o, w.ml, w.joins, st);
        launch_join<T>(a, p.many, 2 * p.many.groups, p.most_tiles, w, DP, st);
    }
    if (!p.few.groups) return;
    if (a.R > kInlineRequests) kv_plan_kernel<<<1, kPlanThreads, 0, st>>>(a, p.few, w.sums);
    launch_kv_decode<T>(a, p.few, w.sums, cache_dtype, DP, pad && !p.many.groups, w.o, w.ml, w.joins, st);
    launch_join<T>(a, p.few, p.few.groups, 0, w, DP, st);
}

static hipError_t attend(const KvAttnArgs &a, int dtype, int cache_dtype, bool pad, void *ws, hipStream_t st)
{
    const KvPlans p = plans(a, cache_dtype);
    const KvWork w = work_of(a, p, ws);
    if (dtype == DRO_BF16) run_attention<bf16>(a, p, w, cache_dtype, pad, st);
    else run_attention<f16>(a, p, w, cache_dtype, pad, st);
    return hipGetLastError();
}

hipError_t launch_kv_attention(const KvAttnArgs &a, int dtype, int cache_dtype, void *ws, hipStream_t st)
{
    return attend(a, dtype, cache_dtype, true, ws, st);
}

// ---- shared prefixes --------------------------------------------------------------------
//
// The softmax over a row's keys is that over the prefix joined with that over its own, by their
// maxima and sums.  All rows of a group see the same keys of the prefix, so first the groups are
// attended like requests whose rows these are (a row of any of them is as good as another in a tile),
// and the prefix is read once a tile instead of once a request; the sums stay as they are, in 32
// bits.  Then each request's own keys are, and whoever finishes a row joins it with its sums.

constexpr int kSharedThreads = 256;

// The groups' rows, each row's place among its request's own tokens, sums of nothing for all rows,
// and, below a window, where a group's rows begin to see its prefix.
__global__ __launch_bounds__(kSharedThreads) void kv_shared_rows_kernel(const KvAttnArgs a, const KvSharedArgs s,
                                                                        int32_t *start, int32_t *row_pos, int2 *ends,
                                                                        float2 *ml)
{
    const uint32_t me = blockIdx.x * kSharedThreads + threadIdx.x, all = gridDim.x * kSharedThreads;
    const int64_t rows = (int64_t)a.T * a.Hq;
    for (int64_t i = me; i < rows; i += all) ml[i] = make_float2(-INFINITY, 0.0f);
    auto at = [&](int r) { return min(max(a.start[r], 0), a.T); };
    auto context = [&](int r) { return (int)min((long long)max(a.context[r], 0), (long long)a.W << a.shift); };
    for (uint32_t t = me; t < (uint32_t)a.T; t += all) {
        int lo = 0, hi = a.R;  // the last request that begins at t or before
        while (hi - lo > 1) {
            const int m = (lo + hi) >> 1;
            if (at(m) <= (int)t) lo = m;
            else hi = m;
        }
        row_pos[t] = a.R ? context(lo) - at(lo + 1) + (int)t : 0;
    }
    auto request = [&](int g) { return min(max(s.first[g], 0), a.R); };
    for (uint32_t g = me; g <= (uint32_t)s.groups; g += all) start[g] = at(request(g));
    if (!ends) return;
    const int lane = threadIdx.x & 63;
    for (uint32_t g = me >> 6; g < (uint32_t)s.groups; g += all >> 6) {  // a wave to a group
        const int S = (int)min((long long)max(s.context[g], 0), (long long)s.W << a.shift), r1 = request(g + 1);
        int lo = S, hi = 0;
        for (int r = request(g) + lane; r < r1; r += 64) {
            const int ctx = context(r), n = at(r + 1) - at(r);
            if (n <= 0) continue;
            const long long from = (long long)S + ctx - s.window;  // of its last row
            lo = min(lo, (int)max(from - n + 1, 0LL));
            hi = max(hi, (int)min(max(from, 0LL), (long long)S));
        }
        for (int d = 32; d; d >>= 1) {
            lo = min(lo, __shfl_xor(lo, d));
            hi = max(hi, __shfl_xor(hi, d));
        }
        if (lane == 0) ends[g] = make_int2(lo, max(lo, hi));
    }
}

struct KvSharedWork {
    float *o;
    float2 *ml;
    int32_t *row_pos, *start;
    int2 *ends;
    void *rest;
    size_t bytes;  // without the rest
};

static KvSharedWork shared_work(const KvAttnArgs &a, const KvSharedArgs &s, void *ws)
{
    KvSharedWork w{};
    char *at = (char *)ws;
    auto take = [&](size_t bytes) {
        char *q = at;
        at += (bytes + 255) & ~size_t(255);
        return q;
    };
    const size_t rows = (size_t)a.T * a.Hq;
    w.o = (float *)take(rows * padded_dim(a.D) * 4);
    w.ml = (float2 *)take(rows * 8);
    w.row_pos = (int32_t *)take((size_t)a.T * 4);
    w.start = (int32_t *)take(((size_t)s.groups + 1) * 4);
    w.ends = (int2 *)take((size_t)s.groups * 8);
    w.rest = at;
    w.bytes = at - (char *)ws;
    return w;
}

static KvAttnArgs over_prefixes(const KvAttnArgs &a, const KvSharedArgs &s, const KvSharedWork &w)
{
    KvAttnArgs p = a;
    p.R = s.groups;
    p.W = s.W;
    p.max_new = s.max_new;
    p.start = w.start;
    p.context = s.context;
    p.table = s.table;
    p.table_stride = s.table_stride;
    p.window = 0;
    p.prefix = nullptr;
    p.raw_ml = w.ml;
    p.raw_o = w.o;
    p.row_pos = w.row_pos;
    p.ends = s.window ? w.ends : nullptr;
    p.prefix_window = s.window;
    return p;
}

size_t kv_shared_bytes(const KvAttnArgs &a, const KvSharedArgs &s, int cache_dtype)
{
    const KvSharedWork w = shared_work(a, s, nullptr);
    return w.bytes + std::max(kv_attention_bytes(over_prefixes(a, s, w), cache_dtype), kv_attention_bytes(a, cache_dtype));
}

hipError_t launch_kv_shared(const KvAttnArgs &a, const KvSharedArgs &s, int dtype, int cache_dtype, void *ws,
                            hipStream_t st)
{
    const KvSharedWork w = shared_work(a, s, ws);
    const KvAttnArgs p = over_prefixes(a, s, w);
    const int64_t items = std::max((int64_t)a.T * std::max(a.Hq / 4, 1), (int64_t)s.groups * 64);
    const unsigned blocks = (unsigned)std::min<int64_t>((items + kSharedThreads) / kSharedThreads, 4 * a.num_cu);
    kv_shared_rows_kernel<<<blocks, kSharedThreads, 0, st>>>(a, s, w.start, w.row_pos, s.window ? w.ends : nullptr, w.ml);
    if (hipError_t e = attend(p, dtype, cache_dtype, false, w.rest, st)) return e;
    KvAttnArgs own = a;
    own.with_ml = w.ml;
    own.with_o = w.o;
    return attend(own, dtype, cache_dtype, true, w.rest, st);
}

}  // namespace dro
