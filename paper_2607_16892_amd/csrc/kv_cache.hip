// Block tables and slots of a serving step, and the store into the paged cache.
#include <algorithm>

#include "kv.h"
#include "kv_sched.h"
#include "kv_types.h"
#include "wave.h"

namespace dro {

// ---- block tables -----------------------------------------------------------
//
// One workgroup takes the sums over the requests (what each gives back, what it
// grows by, where its tokens start) and leaves a record per request; the table
// entries, the free stack and the tokens' slots are written from the records, by the
// same workgroup if there is little to write, else by a second launch.  Nothing written
// there is read there: a block that is handed out comes from the part of the stack that
// was there before, or straight from the table row of the request that gave it back.
// Bound by latency: requests are loaded at once, and searches take 64 probes a step.  64 requests
// take 5.3 us; 4096 with 65,536 new tokens 11.4 and, for the second launch, 9.0.

struct KvRequest {
    long long n, after;
    int held, blocks, back, grow;
    bool live;
};

static __device__ __forceinline__ KvRequest kv_request(const KvTablesArgs &a, int add, int length, int held, int reserve)
{
    KvRequest q;
    const long long len = max(length, 0);
    q.held = min(max(held, 0), a.W);
    q.n = max(add, 0);
    q.after = len + q.n;
    const long long most = max(q.after, (long long)reserve);
    const long long blocks = (most + (1 << a.shift) - 1) >> a.shift;
    q.live = add >= 0 && blocks <= a.W;
    q.blocks = (int)min(blocks, (long long)a.W);
    q.back = add < 0 ? q.held : 0;
    q.grow = q.live ? max(q.blocks - q.held, 0) : 0;
    return q;
}

// Inclusive sums over the workgroup's threads; `total` holds the last one's.  (Blocks: the tables
// have fewer than 2^31 entries.)
struct KvSums {
    uint64_t n;
    uint32_t back, grow;
};
template <int THREADS> static __device__ KvSums scan_threads(KvSums x, KvSums *part, KvSums &total)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    x.n = scan_wave(x.n);
    x.back = scan_wave(x.back);
    x.grow = scan_wave(x.grow);
    if (lane == 63) part[wave] = x;
    __syncthreads();
    // the waves' sums, one a lane
    static_assert(THREADS / 64 <= 16, "a row of lanes");
    KvSums p{0, 0, 0};
    if (lane < THREADS / 64) p = part[lane];
    const uint64_t n = scan_row16(p.n);
    const uint32_t back = scan_row16(p.back), grow = scan_row16(p.grow);
    total = KvSums{lane_value(n, 15), lane_value(back, 15), lane_value(grow, 15)};
    if (wave) {
        const int w = __builtin_amdgcn_readfirstlane(wave) - 1;
        x.n += lane_value(n, w);
        x.back += lane_value(back, w);
        x.grow += lane_value(grow, w);
    }
    return x;
}

// The last index i < n with x[i] <= v, for each lane that asks (x ascending, x[0] <= v).  The
// lanes ask for places near one another: the first and the last of them are found together
// and what lies between is searched in registers.
static __device__ int find_lanes(const uint32_t *x, int n, uint32_t v, bool asks)
{
    const uint64_t who = __ballot(asks);
    if (!who) return 0;
    const uint32_t u = lane_value(v, __builtin_ctzll(who)), w = lane_value(v, 63 - __builtin_clzll(who));
    const int lo = kv_find(x, n, min(u, w)), hi = kv_find(x, n, max(u, w));
    if (lo == hi) return lo;
    int at = lo;
    if (hi - lo < 64) {
        const uint32_t mine = x[min(lo + (int)(threadIdx.x & 63), hi)];
        for (int step = 32; step; step >>= 1) {
            const uint32_t y = __shfl(mine, min(at - lo + step, 63));
            if (at + step <= hi && y <= v) at += step;
        }
        return at;
    }
    int up = hi + 1;
    while (up - at > 1) {
        const int m = (at + up) >> 1;
        if (x[m] <= v) at = m;
        else up = m;
    }
    return at;
}

// The blocks at places `p` of the stack (lanes that ask): below `free` the free list's, above
// it one of the blocks just given back, in its request's row.
static __device__ int kv_stack_block(const KvTablesArgs &a, int p, int free, bool asks)
{
    const bool given = asks && p >= free;
    int block = asks && p >= 0 && !given ? a.free_list[p] : -1;
    if (__any(given)) {
        const int r = find_lanes(a.backs, a.R, (uint32_t)(p - free), given);
        if (given) block = a.table[r * a.table_stride + min(p - free - (int)a.backs[r], a.W - 1)];
    }
    return block;
}

// Table row or free blocks of request r, by a wave.
static __device__ void kv_write_row(const KvTablesArgs &a, int r, int free, int top)
{
    const int lane = threadIdx.x & 63;
    const int4 q = a.rows[r];
    int32_t *row = a.table + r * a.table_stride;
    if (q.w) {  // ended
        // (rows that claim more blocks than the pool has may go beyond 2^31)
        const int64_t at = (int64_t)free + a.backs[r];
        const int n = (int)min((int64_t)q.x, max(top - at, (int64_t)0));
        for (int i = lane; i < n; i += 64) a.free_list[at + i] = row[i];
    } else {
        for (int i0 = q.x; i0 < q.y; i0 += 64) {
            const int i = i0 + lane;
            const int block = kv_stack_block(a, q.z - (i - q.x), free, i < q.y);
            if (i < q.y) row[i] = block;
        }
    }
}

// Slots of tokens t (a wave's, next to one another; t >= T: none).
static __device__ void kv_write_slot(const KvTablesArgs &a, int t, int tokens, int free)
{
    const bool some = t < a.T && t < tokens;
    const int r = find_lanes((const uint32_t *)a.start, a.R, (uint32_t)t, some);
    int64_t slot = -1;
    int pos = -1, p = 0, block = -1;
    bool grown = false;
    if (some && a.granted[r]) {
        const int4 q = a.rows[r];
        pos = max(a.len[r], 0) + t - a.start[r];
        const int b = pos >> a.shift;
        grown = b >= q.x;
        p = q.z - (b - q.x);
        if (!grown) block = a.table[r * a.table_stride + b];
    }
    const int taken = kv_stack_block(a, p, free, grown);
    if (grown) block = taken;
    if (pos >= 0) slot = ((int64_t)block << a.shift) + (pos & ((1 << a.shift) - 1));
    if (t < a.T) {
        a.slot[t] = slot;
        a.pos[t] = pos;
    }
}

// Each thread sums consecutive requests (PER of them, 0: any number, loaded again for the
// second walk) and walks them again with the sums before its own.
// rows[r] = {held, blocks after the step, stack place of the first block taken, ended}.
template <int THREADS, int PER, bool ALL>
__global__ __launch_bounds__(THREADS) void kv_scan_kernel(const KvTablesArgs a)
{
    __shared__ KvSums part[THREADS / 64];
    __shared__ long long most[THREADS / 64];
    const int per = PER ? PER : (a.R + THREADS - 1) / THREADS;
    const int r0 = min((int)threadIdx.x * per, a.R), r1 = min(r0 + per, a.R);
    int add[PER ? PER : 1], len[PER ? PER : 1], held[PER ? PER : 1], res[PER ? PER : 1];
    if constexpr (PER > 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = min(r0 + i, a.R - 1);
            add[i] = a.add[r];
            len[i] = a.len[r];
            held[i] = a.held[r];
            res[i] = a.reserve ? a.reserve[r] : 0;
        }
    }
    auto request = [&](int i) {
        if constexpr (PER > 0) return kv_request(a, add[i], len[i], held[i], res[i]);
        const int r = r0 + i;
        return kv_request(a, a.add[r], a.len[r], a.held[r], a.reserve ? a.reserve[r] : 0);
    };
    const long long free = min(max(a.free_count[0], 0), a.num_blocks);
    KvSums own{0, 0, 0}, all;
    for (int i = 0; i < (PER ? PER : r1 - r0); ++i) {
        if (r0 + i >= r1) break;
        const KvRequest q = request(i);
        own.n += q.n;
        own.back += q.back;
        own.grow += q.grow;
    }
    KvSums at = scan_threads<THREADS>(own, part, all);
    at.n -= own.n;
    at.back -= own.back;
    at.grow -= own.grow;
    // no more blocks than the pool has can be free, whatever the rows claim to hold
    const long long top = min(free + (long long)all.back, (long long)a.num_blocks);
    const long long kTop = 0x7fffffff;
    long long taken = 0;
    for (int i = 0; i < (PER ? PER : r1 - r0); ++i) {
        if (r0 + i >= r1) break;
        const int r = r0 + i;
        const KvRequest q = request(i);
        const long long end = (long long)at.grow + q.grow;
        const bool ok = q.live && (q.grow == 0 || end <= top);
        const bool ended = (PER ? add[PER ? i : 0] : a.add[r]) < 0;
        a.rows[r] = make_int4(q.held, ok ? max(q.held, q.blocks) : q.held,
                              (int)max(top - 1 - (long long)at.grow, -1LL), ended);
        a.backs[r] = (uint32_t)at.back;
        a.start[r] = (int)min((long long)at.n, kTop);
        a.context[r] = ok ? (int)min(q.after, kTop) : 0;
        a.granted[r] = ok;
        a.held_out[r] = ended ? 0 : ok ? max(q.held, q.blocks) : q.held;
        if (ok && q.grow) taken = max(taken, end);
        at.n += q.n;
        at.back += q.back;
        at.grow += q.grow;
    }
    // the largest sum that was granted is what leaves the stack
    for (int d = 32; d; d >>= 1) taken = max(taken, __shfl_xor(taken, d));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = taken;
    __syncthreads();  // (and the records are there for the workgroup)
    const int tokens = (int)min((long long)all.n, kTop);
    if (threadIdx.x == 0) {
        for (int w = 0; w < THREADS / 64; ++w) taken = max(taken, most[w]);
        a.start[a.R] = tokens;
        a.tops[0] = (int)free;
        a.tops[1] = (int)top;
        a.free_out[0] = (int)(top - taken);
    }
    if constexpr (ALL) {
        for (int r = threadIdx.x >> 6; r < a.R; r += THREADS / 64) kv_write_row(a, r, (int)free, (int)top);
        for (int t = threadIdx.x; t < (a.T + 63) / 64 * 64; t += THREADS) kv_write_slot(a, t, tokens, (int)free);
    }
}

constexpr int kExpandThreads = 256;

__global__ __launch_bounds__(kExpandThreads) void kv_expand_kernel(const KvTablesArgs a, int row_blocks)
{
    const int free = a.tops[0], top = a.tops[1];
    if ((int)blockIdx.x < row_blocks) {  // a wave per request
        const int r = blockIdx.x * (kExpandThreads / 64) + (threadIdx.x >> 6);
        if (r < a.R) kv_write_row(a, r, free, top);
    } else {
        kv_write_slot(a, ((int)blockIdx.x - row_blocks) * kExpandThreads + threadIdx.x, a.start[a.R], free);
    }
}

hipError_t launch_kv_tables(const KvTablesArgs &a, hipStream_t st)
{
    // One launch where a wave has at most 16 rows and 256 tokens to write (its blocks are not
    // known here): 64 requests, 512 columns, 14.3 us a call and 16.4 by two launches; 256 requests
    // and 1024 tokens 16.2 and 16.4; 512 and 2000 29.0 and 16.4.
    if (a.R > 0 && a.R <= 256 && a.T <= 1024) {
        kv_scan_kernel<1024, 1, true><<<1, 1024, 0, st>>>(a);
        return hipGetLastError();
    }
    if (a.R == 0) kv_scan_kernel<1024, 0, false><<<1, 1024, 0, st>>>(a);  // (loads no request)
    else if (a.R <= 1024) kv_scan_kernel<1024, 1, false><<<1, 1024, 0, st>>>(a);
    else if (a.R <= 4096) kv_scan_kernel<1024, 4, false><<<1, 1024, 0, st>>>(a);
    else kv_scan_kernel<1024, 0, false><<<1, 1024, 0, st>>>(a);
    const int rows = (a.R + kExpandThreads / 64 - 1) / (kExpandThreads / 64);
    const int toks = (a.T + kExpandThreads - 1) / kExpandThreads;
    if (rows + toks) kv_expand_kernel<<<rows + toks, kExpandThreads, 0, st>>>(a, rows);
    return hipGetLastError();
}

// ---- store --------------------------------------------------------------------
//
// Eight components of a token a thread and step: one load, one store, kStoreSteps tokens in
// flight.  Bound by memory, if the indices and the divisions by the scale stay cheap: one
// index for all of a thread's tokens, one reciprocal.

// 8001 tokens of 8 heads of 128 components into 8 bits: 49 MB in 11.3 us; with one token in
// flight 12.5, with eight 12.8.

constexpr int kStoreThreads = 256;
constexpr int kStoreSteps = 4;

// x / s rounded to nearest (of quotients within 2^-23 of a last place of the middle of two
// floats either) for r = 1 / s, rounded to nearest, of an s far from the format's ends: the
// error x - q s is exact in one product-sum and error r corrects q.  What saturates fp8
// anyway, infinities among it, is left as x r.
__device__ __forceinline__ float quotient(float x, float s, float r)
{
    const float q = x * r;
    return fabsf(q) < 1024.0f ? __builtin_fmaf(__builtin_fmaf(-q, s, x), r, q) : q;
}

template <class T, class C>
__global__ __launch_bounds__(kStoreThreads) void kv_store_kernel(const KvStoreArgs a)
{
    const int which = blockIdx.y;
    const uint32_t per_head = a.D / 8, per_token = per_head * a.H;
    const uint32_t at_once = max(kStoreThreads / per_token, 1u);  // tokens
    const uint32_t mine = threadIdx.x / per_token;
    if (mine >= at_once) return;
    const int64_t t0 = (int64_t)blockIdx.x * at_once * kStoreSteps + mine;
    int64_t slot[kStoreSteps];
#pragma unroll
    for (int i = 0; i < kStoreSteps; ++i) {
        const int64_t t = t0 + i * at_once;
        slot[i] = t < a.T ? a.slot[t] : -1;
    }
    for (uint32_t c = threadIdx.x - mine * per_token; c < per_token; c += kStoreThreads) {
        const uint32_t h = c / per_head, d = (c - h * per_head) * 8;
        const T *x = (const T *)a.x[which] + h * a.x_head[which] + d;
        C *y = (C *)a.c[which] + h * a.c_head[which] + d;
        uint4 v[kStoreSteps];
#pragma unroll
        for (int i = 0; i < kStoreSteps; ++i)
            if (slot[i] >= 0 && slot[i] < a.slots) v[i] = *(const uint4 *)(x + (t0 + i * at_once) * a.x_token[which]);
        float s = 1.0f, r = 1.0f;
        bool far = true;
        if constexpr (sizeof(C) == 1) {
            s = a.scale[which][h];
            r = 1.0f / s;
            far = s > 0x1p-100f && s < 0x1p100f;
        }
#pragma unroll
        for (int i = 0; i < kStoreSteps; ++i) {
            if (slot[i] < 0 || slot[i] >= a.slots) continue;
            C *to = y + (slot[i] >> a.shift) * a.c_block[which] +
                    (slot[i] & ((1 << a.shift) - 1)) * a.c_token[which];
            if constexpr (sizeof(C) == 1) {
                const auto w = __builtin_bit_cast(Vec<T, 8>, v[i]);
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = far ? quotient(to_float(w[j]), s, r) : to_float(w[j]) / s;
                *(uint2 *)to = make_uint2(pack_fp8(f), pack_fp8(f + 4));
            } else {
                *(uint4 *)to = v[i];
            }
        }
    }
}

template <class T, class C> static void run_store(const KvStoreArgs &a, hipStream_t st)
{
    const int64_t at_once = std::max(kStoreThreads / (a.D / 8 * a.H), 1), per = at_once * kStoreSteps;
    kv_store_kernel<T, C><<<dim3((unsigned)((a.T + per - 1) / per), 2), kStoreThreads, 0, st>>>(a);
}

hipError_t launch_kv_store(const KvStoreArgs &a, int dtype, int cache_dtype, hipStream_t st)
{
    if (cache_dtype == DRO_FP8_E4M3) {
        if (dtype == DRO_BF16) run_store<bf16, fp8>(a, st);
        else run_store<f16, fp8>(a, st);
    } else {  // bits are copied, whichever 16-bit type they are
        run_store<bf16, bf16>(a, st);
    }
    return hipGetLastError();
}

}  // namespace dro
