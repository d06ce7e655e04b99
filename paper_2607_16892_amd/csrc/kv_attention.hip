// Attention over the paged cache: the plan of many requests, the join of partial
// results, and the choice of kernels.
#include <algorithm>

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

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(const KvAttnArgs a, const KvCut cut,
                                                               uint32_t *items, uint32_t *partials, int *C)
{
    __shared__ uint64_t part[kPlanThreads / 64];
    const int per = (a.R + kPlanThreads - 1) / kPlanThreads;
    const int r0 = min((int)threadIdx.x * per, a.R), r1 = min(r0 + per, a.R);
    uint64_t keys = 0, total;
    for (int r = r0; r < r1; ++r) {
        const KvShare s = kv_share(a, cut, r);
        keys += (uint64_t)s.tiles * (uint64_t)s.span * (uint64_t)a.H;
    }
    plan_scan(keys, part, total);
    const int c = kv_chunk(cut, total);
    uint64_t mine = 0;  // items in the low, partial results in the high half
    for (int pass = 0; pass < 2; ++pass) {
        uint64_t at = pass ? plan_scan(mine, part, total) - mine : 0;
        for (int r = r0; r < r1; ++r) {
            const KvShare s = kv_share(a, cut, r);
            const int chunks = kv_chunks(s, c);
            const uint64_t n = (uint64_t)s.tiles * (uint64_t)chunks * (uint64_t)a.H;
            if (pass) {
                items[r] = (uint32_t)at;
                partials[r] = (uint32_t)(at >> 32);
                at += chunks > 1 ? n | n << 32 : n;
            } else {
                mine += chunks > 1 ? n | n << 32 : n;
            }
        }
    }
    if (threadIdx.x == 0) {
        items[a.R] = (uint32_t)total;
        partials[a.R] = (uint32_t)(total >> 32);
        C[0] = c;
    }
}

// ---- join -------------------------------------------------------------------------
//
// A workgroup per row (token, query head) whose keys were cut into chunks: the largest
// maximum of its partial results, then their sums.  Bound by latency, so the waves take
// chunks in turn.

template <class T, int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void kv_join_kernel(const KvAttnArgs a, const KvCut cut, const KvPlan plan,
                                                             long long first, const float *part_o,
                                                             const float2 *part_ml)
{
    constexpr int V = DP / 64;
    __shared__ float red[WAVES][2];
    __shared__ float acc[WAVES][DP];
    const long long row = first + blockIdx.x;
    const int t = (int)(row / a.Hq), hq = (int)(row - (long long)t * a.Hq), h = hq / a.G;
    const KvParts p = kv_row_parts(a, cut, plan, t, hq);
    if (p.chunks <= 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float m = -INFINITY;
    for (int c = threadIdx.x; c < p.chunks; c += WAVES * 64) m = fmaxf(m, part_ml[p.first + c * p.stride].x);
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (lane == 0) red[wave][0] = m;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, red[w][0]);
    float l = 0.0f, o[V];
    for (int j = 0; j < V; ++j) o[j] = 0.0f;
#pragma unroll 4
    for (int c = wave; c < p.chunks; c += WAVES) {
        const int64_t at = p.first + c * p.stride;
        const float2 x = part_ml[at];
        // a chunk without a key counts for nothing
        const float f = x.y == 0.0f ? 0.0f : m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(x.x - m);
        const Vec<float, V> y = *(const Vec<float, V> *)(part_o + at * DP + lane * V);
        l += f * x.y;
        for (int j = 0; j < V; ++j) o[j] += f == 0.0f ? 0.0f : f * y[j];
    }
    if (lane == 0) red[wave][1] = l;
    for (int j = 0; j < V; ++j) acc[wave][lane * V + j] = o[j];
    __syncthreads();
    if (wave) return;
    l = 0.0f;
    for (int j = 0; j < V; ++j) o[j] = 0.0f;
    for (int w = 0; w < WAVES; ++w) {
        l += red[w][1];
        for (int j = 0; j < V; ++j) o[j] += acc[w][lane * V + j];
    }
    const float inv = l == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[h] : 1.0f) / l;
    T *out = (T *)a.out + t * a.out_token + hq * a.out_head + lane * V;
    for (int j = 0; j < V; ++j)
        if (lane * V + j < a.D) out[j] = (T)(l == 0.0f ? 0.0f : o[j] * inv);
    if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- launches -----------------------------------------------------------------------

constexpr uint32_t kMaxGrid = 1u << 22;  // workgroups a launch: grids stay below 2^32 work-items

int padded_dim(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

KvCut decode_cut(const KvAttnArgs &a)
{
    KvCut c;
    c.rows = 16;
    c.align = 128;  // four waves of 32 keys
    c.target_log2 = 9;
    c.few = 0x7fffffff;
    c.below = true;
    return c;
}

size_t kv_attention_bytes(const KvAttnArgs &a)
{
    const KvCut c = decode_cut(a);
    const size_t parts = (size_t)2 << c.target_log2;
    return kv_rup(parts * c.rows * padded_dim(a.D) * 4) + kv_rup(parts * c.rows * 8) +
           2 * kv_rup(((size_t)a.R + 1) * 4) + kv_rup(4);
}

template <class T, int DP>
static void run_join(const KvAttnArgs &a, const KvCut &c, const KvPlan &p, const float *o, const float2 *ml,
                     hipStream_t st)
{
    const long long rows = (long long)a.T * a.Hq;
    for (long long f = 0; f < rows; f += kMaxGrid) {
        const uint32_t n = (uint32_t)std::min<long long>(rows - f, kMaxGrid);
        if (rows <= 1024) kv_join_kernel<T, DP, 16><<<n, 1024, 0, st>>>(a, c, p, f, o, ml);
        else kv_join_kernel<T, DP, 4><<<n, 256, 0, st>>>(a, c, p, f, o, ml);
    }
}

hipError_t launch_kv_attention(const KvAttnArgs &a, int dtype, int cache_dtype, void *ws, hipStream_t st)
{
    const KvCut c = decode_cut(a);
    const int DP = padded_dim(a.D);
    const size_t parts = (size_t)2 << c.target_log2;
    char *p = (char *)ws;
    auto take = [&](size_t bytes) {
        char *q = p;
        p += kv_rup(bytes);
        return q;
    };
    float *o = (float *)take(parts * c.rows * DP * 4);
    float2 *ml = (float2 *)take(parts * c.rows * 8);
    uint32_t *items = (uint32_t *)take(((size_t)a.R + 1) * 4);
    uint32_t *partials = (uint32_t *)take(((size_t)a.R + 1) * 4);
    int *C = (int *)take(4);
    const KvPlan plan{items, partials, C};
    if (a.R > kInlineRequests) kv_plan_kernel<<<1, kPlanThreads, 0, st>>>(a, c, items, partials, C);
    const uint64_t tiles = (uint64_t)a.T * a.G / c.rows + std::min(a.R, a.T);
    const uint64_t grid = ((uint64_t)1 << c.target_log2) + tiles * a.H + 8;
    for (uint64_t f = 0; f < grid; f += kMaxGrid) {
        const uint32_t n = (uint32_t)std::min<uint64_t>(grid - f, kMaxGrid);
        if (dtype == DRO_BF16) launch_kv_decode<bf16>(a, c, plan, cache_dtype, DP, (uint32_t)f, n, f == 0, o, ml, st);
        else launch_kv_decode<f16>(a, c, plan, cache_dtype, DP, (uint32_t)f, n, f == 0, o, ml, st);
    }
    if (dtype == DRO_BF16) {
        if (DP == 64) run_join<bf16, 64>(a, c, plan, o, ml, st);
        else if (DP == 128) run_join<bf16, 128>(a, c, plan, o, ml, st);
        else run_join<bf16, 256>(a, c, plan, o, ml, st);
    } else {
        if (DP == 64) run_join<f16, 64>(a, c, plan, o, ml, st);
        else if (DP == 128) run_join<f16, 128>(a, c, plan, o, ml, st);
        else run_join<f16, 256>(a, c, plan, o, ml, st);
    }
    return hipGetLastError();
}

}  // namespace dro
