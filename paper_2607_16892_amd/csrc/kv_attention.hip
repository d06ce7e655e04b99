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

// The sums [n + 1] of the requests' steps; behind shared prefixes, where they are of all sources of
// keys, the steps of a workgroup after them.
template <class A> static __device__ __forceinline__ void plan_sums(const A &a, const KvCut &cut, uint64_t *sums, uint64_t *part)
{
    const int n = kv_requests(a), per = (n + kPlanThreads - 1) / kPlanThreads;
    const int r0 = min((int)threadIdx.x * per, n), r1 = min(r0 + per, n);
    uint64_t units = 0, total;
    uint32_t longest = 0;
    for (int r = r0; r < r1; ++r) {
        const KvShare s = kv_share(a, cut, r);
        units += kv_units(a, s);
        longest = max(longest, kv_steps(s));
    }
    uint64_t at = plan_scan(units, part, total) - units;
    for (int r = r0; r < r1; ++r) {
        sums[r] = at;
        at += kv_units(a, kv_share(a, cut, r));
    }
    if constexpr (kShared<A>) {
        const uint64_t least = __syncthreads_or(longest >= 2048) ? 8 : __syncthreads_or(longest >= 512) ? 4
                             : __syncthreads_or(longest >= 128) ? 2 : 1;
        if (threadIdx.x == 0) sums[n + 1] = kv_run_of(cut, total, least);
    }
    if (threadIdx.x == 0) sums[n] = total;
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(const KvAttnArgs a, const KvCut cut, uint64_t *sums)
{
    __shared__ uint64_t part[kPlanThreads / 64];
    plan_sums(a, cut, sums, part);
}

// The tiles of the requests of many rows and the sums of their chunks: first the tiles before
// each request, then the list and its steps, then the chunks, 1024 tiles at a time.
struct KvTileLds {
    uint64_t part[kPlanThreads / 64];
    uint32_t steps_at[kPlanThreads];
    uint32_t before[kPlanThreads];  // up to a request a thread: a search in LDS
    uint32_t nth_at[kPlanThreads];  // behind shared prefixes
    KvShare share[kPlanThreads];
};

// (behind shared prefixes also `where`: of each tile, as they are listed before they are sorted, its
// first partial result, of head 0, and its chunks)
template <class A>
static __device__ __forceinline__ void plan_tiles(const A &a, const KvCut &cut, int keys, int most, uint64_t *before,
                                                  uint32_t *sums, KvTile *tiles, KvTileList *list, int2 *where, KvTileLds &l)
{
    uint64_t *part = l.part;
    const int requests = kv_requests(a);
    const bool lds = requests <= kPlanThreads;
    const int per = (requests + kPlanThreads - 1) / kPlanThreads;
    const int r0 = min((int)threadIdx.x * per, requests), r1 = min(r0 + per, requests);
    uint64_t own = 0, total;
    KvShare s0{};
    for (int r = r0; r < r1; ++r) {
        s0 = kv_share(a, cut, r);
        own += s0.tiles;
    }
    uint64_t at = plan_scan(own, part, total) - own;
    if (lds) {
        l.before[threadIdx.x] = (uint32_t)min(at, (uint64_t)0xffffffff);
        l.share[threadIdx.x] = s0;
    }
    if (!lds || kShared<A>) {
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
            int lo = 0, hi = requests;  // the last request with before[r] <= e: it has tiles
            while (hi - lo > 1) {
                const int m = (lo + hi) >> 1;
                if ((lds ? l.before[m] : before[m]) <= (uint64_t)e) lo = m;
                else hi = m;
            }
            const KvShare s = lds ? l.share[lo] : kv_share(a, cut, lo);
            const int tile = max(s.tiles - 1 - (e - (int)(lds ? l.before[lo] : before[lo])), 0);
            steps = kv_tile_steps(a, s, lo, tile, cut.rows, keys);
            mine = KvTile{lo, tile, s.n, s.ctx, kv_first_token(a, lo), (int)steps, 0, 1, 0};
            tiles[e] = mine;
        }
        plan_scan(steps, part, total);
        steps_all += total;
    }
    uint64_t share = kv_tile_share(cut, steps_all * a.H);
    // Prefixes' tiles have many rows to write and join for few steps: eight steps where every compute
    // unit gets a part all the same (64 requests behind 8192 tokens, 32 heads on 8: 92 us, so 83).
    if constexpr (kShared<A>) share = max(share, min((uint64_t)8, steps_all * a.H / (uint32_t)(cut.groups / 2)));
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
            l.steps_at[to] = mine.steps;
            if constexpr (kShared<A>) l.nth_at[to] = threadIdx.x;
        }
        __syncthreads();
    }
    // Chunks: of the tiles that are cut, with 1.75 shares or more, a tile has at most 8/7 as many
    // as shares, so there are fewer than 2 `groups` of them over all heads.
    uint32_t all = 0, parts = 0;
    for (int e0 = 0; e0 < n; e0 += kPlanThreads) {
        const int e = e0 + threadIdx.x;
        const uint32_t steps = e >= n ? 0 : sort ? l.steps_at[e] : tiles[e].steps;  // (tiles: this thread's)
        const uint64_t chunks = e < n ? max((steps + share / 4) / share, (uint64_t)1) : 0;
        const uint64_t count = chunks > 1 ? chunks | chunks << 32 : chunks;
        const uint64_t upto = plan_scan(count, part, total) - count;
        if (e < n) {
            sums[e] = tiles[e].before = all + (uint32_t)upto;
            tiles[e].part = (int)(parts + (uint32_t)(upto >> 32));
            tiles[e].chunks = (int)chunks;
            if constexpr (kShared<A>)
                where[sort ? l.nth_at[e] : e] = make_int2((int)(parts + (uint32_t)(upto >> 32)), (int)chunks);
        }
        all += (uint32_t)total;
        parts += (uint32_t)(total >> 32);
    }
    if (threadIdx.x == 0) {
        sums[n] = all;
        *list = KvTileList{n, (int)parts, all};
    }
}

__global__ __launch_bounds__(kPlanThreads) void kv_tiles_kernel(const KvAttnArgs a, const KvCut cut, int keys, int most,
                                                                uint64_t *before, uint32_t *sums, KvTile *tiles,
                                                                KvTileList *list)
{
    __shared__ KvTileLds lds;
    plan_tiles(a, cut, keys, most, before, sums, tiles, list, nullptr, lds);
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
        const float to = fmaxf(m, x.x), by = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
        const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(x.x - to);
        m = to;
        l = l * by + f * x.y;
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
    template <class T>
    __device__ __forceinline__ void write(const KvAttnArgs &a, const KvJoin &it, int y, int d) const
    {
        const int row = it.row0 + y, token = row / a.G, hq = it.head * a.G + row - token * a.G;
        write_row<T>(a, it.first_token + token, it.head, hq, d);
    }
    template <class T>
    __device__ __forceinline__ void write_row(const KvAttnArgs &a, int64_t t, int head, int hq, int d) const
    {
        const float inv = l == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[head] : 1.0f) / l;
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
        if (a.lse && d == 0) a.lse[t * a.Hq + hq] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
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
            s.write<T>(a, it, y, d);
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
                s.template write<T>(a, it, y, lane * V);
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

// Cuts a workspace up; from a null one, sizes.
struct KvTake {
    char *at;
    template <class U> void operator()(U *&p, size_t count)
    {
        p = (U *)at;
        at += (count * sizeof(U) + 255) & ~size_t(255);
    }
};

static KvWork work_of(const KvAttnArgs &a, const KvPlans &p, void *ws)
{
    KvWork w{};
    KvTake take{(char *)ws};
    // the kernels run one after the other: their partial results share one place
    const size_t rows = (size_t)2 * std::max((size_t)p.few.groups * p.few.rows, (size_t)p.many.groups * p.many.rows);
    take(w.o, rows * padded_dim(a.D));
    take(w.ml, rows);
    take(w.joins, std::max(p.few.groups, 2 * p.many.groups));
    take(w.sums, (size_t)a.R + 1);
    if (p.many.groups) {
        take(w.before, a.R);
        take(w.tile_sums, (size_t)p.most_tiles + 1);
        take(w.tiles, p.most_tiles);
        take(w.list, 1);
    }
    w.bytes = take.at - (char *)ws;
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
static void run_attention(const KvMxArgs &a, const KvPlans &p, const KvWork &w, int cache_dtype, hipStream_t st)
{
    const int DP = padded_dim(a.D);
    if (p.many.groups) {
        kv_tiles_kernel<<<1, kPlanThreads, 0, st>>>(a, p.many, kv_prefill_keys(DP), p.most_tiles,
                                                    w.before, w.tile_sums, w.tiles, w.list);
        const KvTiles t{w.tile_sums, w.tiles, w.list};
        launch_kv_prefill<T>(a, p.many, t, p.grid, cache_dtype, DP, true, w.o, w.ml, w.joins, st);
        launch_join<T>(a, p.many, 2 * p.many.groups, p.most_tiles, w, DP, st);
    }
    if (!p.few.groups) return;
    if (a.R > kInlineRequests) kv_plan_kernel<<<1, kPlanThreads, 0, st>>>(a, p.few, w.sums);
    launch_kv_decode<T>(a, p.few, w.sums, cache_dtype, DP, !p.many.groups, w.o, w.ml, w.joins, st);
    launch_join<T>(a, p.few, p.few.groups, 0, w, DP, st);
}

hipError_t launch_kv_attention(const KvMxArgs &a, int dtype, int cache_dtype, void *ws, hipStream_t st)
{
    const KvPlans p = plans(a, cache_dtype);
    const KvWork w = work_of(a, p, ws);
    if (dtype == DRO_BF16) run_attention<bf16>(a, p, w, cache_dtype, st);
    else run_attention<f16>(a, p, w, cache_dtype, st);
    return hipGetLastError();
}

// ---- shared prefixes --------------------------------------------------------------------
//
// The softmax over a row's keys is that over its group's prefix joined with that over its own tokens,
// by their maxima and sums.  All rows of a group see the same keys of its prefix, so it is attended
// like one request whose rows these are: a tile takes rows of several requests, and reads the
// prefix once for them.  One launch of a workgroup plans both (the same lists, over the groups
// and then the requests), the kernels of few and of many rows leave sums, and one launch joins
// each row's, up to the order of the sources and of their keys.

static __device__ __forceinline__ int group_request(const KvSharedArgs &a, int g) { return min(max(a.first[g], 0), a.R); }

// The last index of the ascending x[0 .. n) whose entry is at most v (0: or none is).
template <class U> static __device__ __forceinline__ int last_upto(const U *x, int n, int v)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (x[m] <= v) lo = m;
        else hi = m;
    }
    return lo;
}

// The plan, by parts: workgroup 0 sums the steps of the sources of few rows, workgroup 1 lists the
// tiles of the others (both find the groups' rows, and below a window where a group's rows begin to
// see its prefix), and the others give each row its request and group, 1024 rows at a time.  (One
// workgroup for all took 12 us, and a join whose rows search for themselves 2 us more; now plan and join
// take 8.4 and 11.1, of 64 requests behind one prefix of 8192 tokens, 32 heads on 8.)
constexpr int kSearched = 2048;

static __device__ __forceinline__ void plan_rows(const KvSharedArgs &a, int32_t *start_lds, int32_t *first_lds)
{
    const bool near = a.R < kSearched && a.groups < kSearched;
    if (near) {
        for (int i = threadIdx.x; i <= a.R; i += kPlanThreads) start_lds[i] = a.start[i];
        for (int i = threadIdx.x; i <= a.groups; i += kPlanThreads) first_lds[i] = a.first[i];
        __syncthreads();
    }
    auto start = [&](int r) { return min(max(near ? start_lds[r] : a.start[r], 0), a.T); };
    auto first = [&](int g) { return min(max(near ? first_lds[g] : a.first[g], 0), a.R); };
    for (int64_t t0 = (int64_t)(blockIdx.x - 2) * kPlanThreads; t0 < a.T; t0 += (int64_t)(gridDim.x - 2) * kPlanThreads) {
        const int t = (int)t0 + threadIdx.x;
        if (t >= a.T) continue;
        const int r = near ? last_upto(start_lds, a.R, t) : last_upto(a.start, a.R, t);
        const bool own = start(r) <= t && t < start(r + 1);
        const int g = near ? last_upto(first_lds, a.groups, r) : last_upto(a.first, a.groups, r);
        const bool behind = own && first(g) <= r && r < first(g + 1) && start(first(g)) <= t && t < start(first(g + 1));
        a.row_of[t] = make_int2(own ? r : -1, behind ? g : -1);
        if (a.row_pos) a.row_pos[t] = kv_context(a, a.groups + r) - start(r + 1) + t;
    }
}

__global__ __launch_bounds__(kPlanThreads) void kv_shared_plan_kernel(const KvSharedArgs a, const KvCut few, const KvCut many,
                                                                      int keys, int most, uint64_t *sums, uint64_t *before,
                                                                      uint32_t *tile_sums, KvTile *tiles, KvTileList *list,
                                                                      int2 *where)
{
    __shared__ KvTileLds lds;
    if (blockIdx.x >= 2) {
        static_assert(sizeof(KvTileLds) >= 8 * kSearched, "starts and first requests");
        plan_rows(a, (int32_t *)&lds, (int32_t *)&lds + kSearched);
        return;
    }
    if (!(blockIdx.x ? many.groups : few.groups)) return;
    for (int g = threadIdx.x; g <= a.groups; g += kPlanThreads)  // (both workgroups write the same)
        a.p_start[g] = min(max(a.start[group_request(a, g)], 0), a.T);
    if (a.ends) {
        const int lane = threadIdx.x & 63;
        for (int g = threadIdx.x >> 6; g < a.groups; g += kPlanThreads / 64) {  // a wave to a group
            const int S = kv_context(a, g), r1 = group_request(a, g + 1);
            int lo = S, hi = 0;
            for (int r = group_request(a, g) + lane; r < r1; r += 64) {
                const int n = kv_end_token(a, a.groups + r) - kv_first_token(a, a.groups + r);
                if (n <= 0) continue;
                const long long from = (long long)S + kv_context(a, a.groups + r) - a.p_window;  // of its last row
                lo = min(lo, (int)max(from - n + 1, 0LL));
                hi = max(hi, (int)min(max(from, 0LL), (long long)S));
            }
            for (int d = 32; d; d >>= 1) {
                lo = min(lo, __shfl_xor(lo, d));
                hi = max(hi, __shfl_xor(hi, d));
            }
            if (lane == 0) a.ends[g] = make_int2(lo, max(lo, hi));
        }
    }
    __syncthreads();  // (both are there for the workgroup)
    if (blockIdx.x == 0) plan_sums(a, few, sums, lds.part);
    else plan_tiles(a, many, keys, most, before, tile_sums, tiles, list, where, lds);
}

struct KvSharedWork {
    float *o[2];       // partial results of the kernels of few and of many rows
    float2 *ml[2];
    uint64_t *sums, *before;
    uint32_t *tile_sums;
    KvTile *tiles;
    KvTileList *list;
    int2 *where;
    size_t bytes;
};

// Where the sums of a row over one of its sources are: `parts` rows, of which part 0 is row `first`
// and part c row next + (c - 1) stride.
struct KvSums32 {
    const float *o;
    const float2 *ml;
    int parts;
    int64_t first, next;
    int stride;
};

// A wave to as many of a token's rows as its lanes reach with 16 bytes each: first a row's prefix, then
// its own keys, each in the order of the keys.  Bound by latency, so what says where both are is asked
// for at once (whichever kernel's it is), and then several parts of both, up to eight (16: more registers,
// and 3 % more of the call, 128 requests behind 12 prefixes in 4 bits).
constexpr int kRowsWaves = 4;
template <class T, int DP>
__global__ __launch_bounds__(kRowsWaves * 64) void kv_shared_join_kernel(const KvSharedArgs a, const KvCut few, const KvCut many,
                                                                         const KvSharedWork w, uint32_t units, uint32_t per)
{
    constexpr int Lanes = DP / 4, Rows = 64 / Lanes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = lane % Lanes * 4;
    KvTileList list{0, 0, 0};
    if (many.groups) list = *w.list;
    const uint64_t run = few.groups ? w.sums[a.groups + a.R + 1] : 1;
    for (uint32_t unit = blockIdx.x * kRowsWaves + wave; unit < units; unit += gridDim.x * kRowsWaves) {
        const int t = unit / per, hq = (int)(unit - (uint32_t)t * per) * Rows + lane / Lanes;
        const int2 of = a.row_of[t];
        if (hq >= a.Hq) continue;
        const int h = hq / a.G, j = hq - h * a.G;
        const int64_t row_at = (int64_t)t * a.Hq + hq;
        auto find = [&](int i, int source, bool is) {
            KvSums32 x{a.raw_o[source], a.raw_ml[source], 1, row_at, 0, 0};
            const int first = kv_first_token(a, i), n = kv_end_token(a, i) - first, row = (t - first) * a.G + j;
            const KvShare s = kv_share(a, few, i);
            const uint64_t sum = few.groups ? w.sums[i] : 0, listed = many.groups ? w.before[i] : 0;
            if (few.groups && n <= kv_few(a, few, i)) {
                const int tile = row / few.rows, y = row - tile * few.rows;
                const uint64_t u0 = sum + ((uint64_t)h * s.tiles + tile) * kv_steps(s), u1 = u0 + kv_steps(s) - 1;
                const bool small = u1 < 0xffffffffu;  // (then the run is)
                const uint32_t b0 = small ? (uint32_t)u0 / (uint32_t)run : (uint32_t)(u0 / run);
                const uint32_t b1 = small ? (uint32_t)u1 / (uint32_t)run : (uint32_t)(u1 / run);
                if (b0 < b1)
                    x = KvSums32{w.o[0], w.ml[0], (int)(b1 - b0) + 1, (int64_t)kv_part(b0, true) * few.rows + y,
                                 (int64_t)kv_part(b0 + 1, false) * few.rows + y, 2 * few.rows};
            } else {
                const int tile = row / many.rows, y = row - tile * many.rows;
                const int tiles = (int)(((long long)n * a.G + many.rows - 1) / many.rows);
                const uint64_t nth = listed + (tiles - 1 - tile);  // (listed last tile first)
                is &= nth < (uint64_t)list.count;                  // (starts that are not ascending)
                const int2 at = is ? w.where[nth] : make_int2(0, 1);
                const int64_t place = at.x + list.parts * h;
                if (at.y > 1)
                    x = KvSums32{w.o[1], w.ml[1], at.y, place * many.rows + y, (place + 1) * many.rows + y, many.rows};
            }
            if (!is) x.parts = 0;
            return x;
        };
        const KvSums32 prefix = find(max(of.y, 0), 0, of.y >= 0), own = find(a.groups + max(of.x, 0), 1, of.x >= 0);
        const int all = prefix.parts + own.parts;
        RowSum<4> s;
        s.clear();
        auto sum = [&](auto ahead) {
            constexpr int N = decltype(ahead)::value;
            for (int c = 0; c < all; c += N) {
                float2 x[N];
                Vec<float, 4> z[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int n = min(c + i, all - 1), k = n < prefix.parts ? n : n - prefix.parts;
                    const KvSums32 &from = n < prefix.parts ? prefix : own;
                    const int64_t at = k == 0 ? from.first : from.next + (int64_t)(k - 1) * from.stride;
                    x[i] = from.ml[at];
                    z[i] = *(const Vec<float, 4> *)(from.o + at * DP + d);
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (c + i < all) {
                        const float y[4] = {z[i][0], z[i][1], z[i][2], z[i][3]};
                        s.add(x[i], y);
                    }
            }
        };
        if (all <= 4) sum(std::integral_constant<int, 4>{});
        else sum(std::integral_constant<int, 8>{});
        s.template write_row<T>(a, t, h, hq, d);
    }
}

// Tokens up to which a group's prefix is the kernel's for few rows: one of its tiles, and four where
// the prefixes are small (by their table), since the other kernel takes 10 us to begin.  (Calls of single
// tokens whose requests do not read their prefixes themselves.  Eight requests behind 1000 tokens, 8 heads
// on one, below a window of 900: 24 us by four tiles, 38 by the other; 16 behind 500, 8 on two, below 400:
// 22 and 38; eight behind 900 beside 64 without a prefix, 8 on one: 23 and 33.  16 behind 4000, 32 on 8, below
// a window of 4000: 43 either way; 64 behind 16 prefixes of 1000 to 4000, 64 on 8, two tiles a group: 95 and
// 68.)
static int shared_few(const KvSharedArgs &a)
{
    const int64_t keys = (int64_t)a.groups * a.H * a.p_W << a.shift;
    return std::max((keys <= 8192 ? 64 : 16) / a.G, 1);
}

static KvPlans shared_plans(const KvSharedArgs &a, int cache_dtype)
{
    const int DP = padded_dim(a.D), requests = a.groups + a.R;
    const int few = std::max(((int64_t)requests * a.H < 16 ? 32 : 16) / a.G, 1), p_few = shared_few(a);
    // As without prefixes, but single tokens keep their kernel beside groups of many rows, whose
    // tiles are few and long.  One kernel takes all sources of up to kFewRequests requests with chunks here
    // as well: both have their rows planned and joined by the same launches, but run one after the other.
    // (7 chunks of 33 to 300 beside 13 single tokens, 12 heads of 64 components, behind two prefixes of 1801
    // to 3500: 51 us by one, 64 by both, below a window and a cap 74 and 77; 8 of 33 to 256 beside 16, 32
    // heads on 8, MXFP4: 131 and 141; 4 of 512 beside 56 over 600 to 4000: 324 and 370; one of 500 beside 7
    // over 600 to 30,000: 382 and 390.)
    const bool all_few = a.max_new <= few && a.p_max_new <= p_few;
    const bool all_many = a.max_new > few && (a.R <= kFewRequests || a.T > (int64_t)(a.R - 1) * a.max_new + few);
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
        // sources that have tiles
        const int64_t longer = all_many ? a.T : a.T / (few + 1) + 1, wider = all_many ? a.T : a.T / (p_few + 1) + 1;
        p.most_tiles = (int)(2 * ((int64_t)a.T * a.G / p.many.rows) + std::min<int64_t>(a.groups, wider) +
                             std::min<int64_t>(a.R, longer));
        const int64_t items = (int64_t)p.most_tiles * a.H;
        p.grid = (unsigned)std::min<int64_t>((items + 2 * p.many.groups + kDies) / kDies * kDies, 1 << 23);
    }
    return p;
}

// Also sets the scratch of the arguments.
static KvSharedWork shared_work(KvSharedArgs &a, const KvPlans &p, void *ws)
{
    KvSharedWork w{};
    KvTake take{(char *)ws};
    const int DP = padded_dim(a.D);
    const size_t rows = (size_t)a.T * a.Hq, requests = (size_t)a.groups + a.R;
    for (int i = 0; i < 2; ++i) {
        take(a.raw_o[i], rows * DP);
        take(a.raw_ml[i], rows);
        const KvCut &c = i ? p.many : p.few;
        take(w.o[i], (size_t)2 * c.groups * c.rows * DP);
        take(w.ml[i], (size_t)2 * c.groups * c.rows);
    }
    take(a.p_start, (size_t)a.groups + 1);
    take(a.ends, a.groups);
    take(a.row_pos, a.T);
    take(a.row_of, a.T);
    take(w.sums, requests + 2);
    take(w.before, requests);
    take(w.tile_sums, (size_t)p.most_tiles + 1);
    take(w.tiles, p.most_tiles);
    take(w.where, p.most_tiles);
    take(w.list, 1);
    if (!a.p_window) a.ends = nullptr;
    if (!a.p_window && !a.slopes) a.row_pos = nullptr;
    a.p_few = !p.many.groups ? 0x7fffffff : !p.few.groups ? 0 : shared_few(a);
    w.bytes = take.at - (char *)ws;
    return w;
}

// Whether each request reads its prefix itself, the same bytes from the caches mostly, which takes two
// launches instead of three or four: where single tokens read at most 300 MB of the prefixes in all (by
// their table).  (32 heads on 8 of 128 components, 16 bits, one prefix unless said: 16 requests
// behind 256 tokens 17 us and by groups 22; 16 behind four of 2000, 131 MB, 30 and 47; 64 behind 992, 260
// MB, 35 and 42; 32 behind two of 4000, 524 MB, 77 and 40; 64 behind 8192, 287 and 83.  The lengths
// are on the device, so a table wider than its prefixes counts as it is: 48 behind six of 300 in a table
// for 2512 tokens, 39 us by groups where their own reading takes 22.)
constexpr double kReadItself = 300e6;
static bool reads_itself(const KvSharedArgs &a, int cache_dtype)
{
    if (a.p_window || a.R > kInlineRequests || a.groups > kInlineRequests || a.max_new > std::max(few_rows(a) / a.G, 1))
        return false;
    const int bits = cache_dtype == DRO_MXFP4 ? 4 : cache_dtype == DRO_MXFP8 || cache_dtype == DRO_FP8_E4M3 ? 8 : 16;
    return (double)a.R * a.H * a.D * bits / 4 * ((int64_t)a.p_W << a.shift) <= kReadItself;
}

static KvJoinedArgs joined_args(const KvSharedArgs &a)
{
    KvJoinedArgs j{a, a.groups, a.p_W, a.first, a.p_context, a.p_table, a.p_stride};
    j.window = 0;
    return j;
}

size_t kv_shared_bytes(const KvSharedArgs &a, int cache_dtype)
{
    if (reads_itself(a, cache_dtype)) return kv_attention_bytes(joined_args(a), cache_dtype);
    KvSharedArgs b = a;
    return shared_work(b, shared_plans(a, cache_dtype), nullptr).bytes;
}

template <class T> static void run_shared(const KvSharedArgs &a, const KvPlans &p, const KvSharedWork &w, int cache_dtype, hipStream_t st)
{
    const int DP = padded_dim(a.D);
    const unsigned row_groups = (unsigned)std::min((a.T + kPlanThreads - 1) / kPlanThreads, a.num_cu);
    kv_shared_plan_kernel<<<2 + row_groups, kPlanThreads, 0, st>>>(a, p.few, p.many, kv_prefill_keys(DP), p.most_tiles, w.sums,
                                                                  w.before, w.tile_sums, w.tiles, w.list, w.where);
    if (p.many.groups) {
        const KvTiles t{w.tile_sums, w.tiles, w.list};
        launch_kv_prefill<T>(a, p.many, t, p.grid, cache_dtype, DP, false, w.o[1], w.ml[1], nullptr, st);
    }
    if (p.few.groups) launch_kv_decode<T>(a, p.few, w.sums, cache_dtype, DP, false, w.o[0], w.ml[0], nullptr, st);
    const int rows = 64 / (DP / 4);  // of a wave
    const uint32_t per = (uint32_t)(a.Hq + rows - 1) / rows, units = (uint32_t)a.T * per;
    const unsigned blocks = std::min((units + kRowsWaves - 1) / kRowsWaves, 1u << 20);
    auto kernel = DP == 64 ? kv_shared_join_kernel<T, 64> : DP == 128 ? kv_shared_join_kernel<T, 128> : kv_shared_join_kernel<T, 256>;
    kernel<<<blocks, kRowsWaves * 64, 0, st>>>(a, p.few, p.many, w, units, per);
}

template <class T> static void run_joined(const KvJoinedArgs &a, const KvPlans &p, const KvWork &w, int cache_dtype, hipStream_t st)
{
    const int DP = padded_dim(a.D);
    launch_kv_decode<T>(a, p.few, nullptr, cache_dtype, DP, true, w.o, w.ml, w.joins, st);
    launch_join<T>(a, p.few, p.few.groups, 0, w, DP, st);
}

hipError_t launch_kv_shared(KvSharedArgs a, int dtype, int cache_dtype, void *ws, hipStream_t st)
{
    if (reads_itself(a, cache_dtype)) {
        const KvJoinedArgs j = joined_args(a);
        const KvPlans p = plans(j, cache_dtype);
        const KvWork w = work_of(j, p, ws);
        if (dtype == DRO_BF16) run_joined<bf16>(j, p, w, cache_dtype, st);
        else run_joined<f16>(j, p, w, cache_dtype, st);
        return hipGetLastError();
    }
    const KvPlans p = shared_plans(a, cache_dtype);
    const KvSharedWork w = shared_work(a, p, ws);
    if (dtype == DRO_BF16) run_shared<bf16>(a, p, w, cache_dtype, st);
    else run_shared<f16>(a, p, w, cache_dtype, st);
    return hipGetLastError();
}

}  // namespace dro
