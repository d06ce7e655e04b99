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
    uint64_t before = 0;
    total = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) before += part[w];
        total += part[w];
    }
    __syncthreads();
    return before + x;
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

// ---- join -------------------------------------------------------------------------
//
// Workgroup (b, y): if an item begins in run b and ends in a later one, rows of it from the
// partial results of the runs that it reaches over.  The run left what there is to do.  Up
// to kFewParts parts a wave joins a row; more (a long request alone) the waves share, a
// workgroup to a row.  Bound by latency (the parts come from other dies' caches), so a wave
// asks for kAhead parts at once.

constexpr int kFewParts = 16;
constexpr int kAhead = 8;

template <class T, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void kv_join_kernel(const KvAttnArgs a, int tile_rows, const float *part_o,
                                                                  const float2 *part_ml, const KvJoin *joins)
{
    constexpr int V = DP / 64;
    __shared__ float2 red[WAVES];
    __shared__ float acc[WAVES][DP];
    const KvJoin it = joins[blockIdx.x];
    if (it.parts == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float scale = a.v_scale ? a.v_scale[it.head] : 1.0f;
    float m, l, o[V];
    auto join = [&](float2 x, const float *z) {
        if (x.y == 0.0f) return;  // no key that the row sees
        const float to = fmaxf(m, x.x), by = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
        const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(x.x - to);
        m = to;
        l = l * by + f * x.y;
        for (int j = 0; j < V; ++j) o[j] = o[j] * by + f * z[j];
    };
    auto clear = [&]() {
        m = -INFINITY;
        l = 0.0f;
        for (int j = 0; j < V; ++j) o[j] = 0.0f;
    };
    // parts c, c + by, .. of row y
    auto sum = [&](int y, int c, int by) {
        clear();
        for (; c < it.parts; c += by * kAhead) {
            float2 x[kAhead];
            Vec<float, V> z[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int n = min(c + i * by, it.parts - 1);
                const int64_t at = kv_part(blockIdx.x + n, n == 0) * tile_rows + y;
                x[i] = part_ml[at];
                z[i] = *(const Vec<float, V> *)(part_o + at * DP + lane * V);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (c + i * by < it.parts) {
                    float w[V];
                    for (int j = 0; j < V; ++j) w[j] = z[i][j];
                    join(x[i], w);
                }
        }
    };
    auto write = [&](int y) {
        const int row = it.row0 + y, token = row / a.G, hq = it.head * a.G + row - token * a.G;
        const int64_t t = it.first_token + token;
        const float inv = l == 0.0f ? 0.0f : scale / l;
        T *out = (T *)a.out + t * a.out_token + hq * a.out_head + lane * V;
        for (int j = 0; j < V; ++j)
            if (lane * V + j < a.D) out[j] = (T)(l == 0.0f ? 0.0f : o[j] * inv);
        if (a.lse && lane == 0)
            a.lse[t * a.Hq + hq] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    };
    if (it.parts <= kFewParts) {
        for (int y = blockIdx.y * WAVES + wave; y < it.rows; y += gridDim.y * WAVES) {
            sum(y, 0, 1);
            write(y);
        }
        return;
    }
    for (int y = blockIdx.y; y < it.rows; y += gridDim.y) {
        sum(y, wave, WAVES);
        if (lane == 0) red[wave] = make_float2(m, l);
        for (int j = 0; j < V; ++j) acc[wave][lane * V + j] = o[j];
        __syncthreads();
        if (wave == 0) {
            for (int w = 1; w < WAVES; ++w) join(red[w], &acc[w][lane * V]);
            write(y);
        }
        __syncthreads();
    }
}

// ---- launches -----------------------------------------------------------------------

static int padded_dim(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

static KvCut decode_cut(const KvAttnArgs &a, int cache_dtype)
{
    KvCut c;
    c.rows = 16;
    c.groups = a.num_cu * 4 * kv_decode_waves(cache_dtype, padded_dim(a.D));
    c.few = 0x7fffffff;
    c.below = true;
    return c;
}

size_t kv_attention_bytes(const KvAttnArgs &a, int cache_dtype)
{
    const KvCut c = decode_cut(a, cache_dtype);
    const size_t rows = (size_t)2 * c.groups * c.rows;
    return kv_rup(rows * padded_dim(a.D) * 4) + kv_rup(rows * 8) + kv_rup(((size_t)a.R + 1) * 8) +
           kv_rup(c.groups * sizeof(KvJoin));
}

hipError_t launch_kv_attention(const KvAttnArgs &a, int dtype, int cache_dtype, void *ws, hipStream_t st)
{
    const KvCut c = decode_cut(a, cache_dtype);
    const int DP = padded_dim(a.D);
    const size_t rows = (size_t)2 * c.groups * c.rows;
    char *p = (char *)ws;
    auto take = [&](size_t bytes) {
        char *q = p;
        p += kv_rup(bytes);
        return q;
    };
    float *o = (float *)take(rows * DP * 4);
    float2 *ml = (float2 *)take(rows * 8);
    uint64_t *sums = (uint64_t *)take(((size_t)a.R + 1) * 8);
    KvJoin *joins = (KvJoin *)take(c.groups * sizeof(KvJoin));
    if (a.R > kInlineRequests) kv_plan_kernel<<<1, kPlanThreads, 0, st>>>(a, c, sums);
    if (dtype == DRO_BF16) launch_kv_decode<bf16>(a, c, sums, cache_dtype, DP, true, o, ml, joins, st);
    else launch_kv_decode<f16>(a, c, sums, cache_dtype, DP, true, o, ml, joins, st);
    // few items may have many parts: sixteen waves to a row; else four rows a workgroup
    const unsigned most = (unsigned)std::max<int64_t>(1, std::min<int64_t>((int64_t)a.max_new * a.G, c.rows));
    const bool few = a.R * (int64_t)a.H <= 64;
    const dim3 grid(c.groups, few ? most : (most + 3) / 4);
    auto join = [&](auto kernel) { kernel<<<grid, few ? 1024 : 256, 0, st>>>(a, c.rows, o, ml, joins); };
    auto pick = [&](auto t, auto w) {
        using T = decltype(t);
        constexpr int W = decltype(w)::value;
        join(DP == 64 ? kv_join_kernel<T, 64, W> : DP == 128 ? kv_join_kernel<T, 128, W> : kv_join_kernel<T, 256, W>);
    };
    auto waves = [&](auto t) {
        if (few) pick(t, std::integral_constant<int, 16>{});
        else pick(t, std::integral_constant<int, 4>{});
    };
    if (dtype == DRO_BF16) waves(bf16{});
    else waves(f16{});
    return hipGetLastError();
}

}  // namespace dro
