// Block tables and slots of a serving step, and the store into the paged cache.
#include "kv.h"
#include "kv_types.h"
#include "wave.h"

namespace dro {

// ---- block tables -----------------------------------------------------------
//
// One workgroup takes the sums over the requests (what each gives back, what it
// grows by, where its tokens start) and leaves a record per request; a second
// kernel writes the table entries, the free stack and the tokens' slots from the
// records.  The second kernel never reads what it writes: a block that is handed
// out comes from the part of the stack that was there before, or straight from the
// table row of the request that gave it back.

constexpr int kScanThreads = 1024;
constexpr int kScanWaves = kScanThreads / 64;

struct KvRequest {
    long long n, after;
    int held, blocks, back;
    long long grow;
    bool live;
};

static __device__ KvRequest kv_request(const KvTablesArgs &a, int r)
{
    KvRequest q;
    const int add = a.add[r];
    const long long len = max(a.len[r], 0);
    q.held = min(max(a.held[r], 0), a.W);
    q.n = max(add, 0);
    q.after = len + q.n;
    const long long most = a.reserve ? max(q.after, (long long)a.reserve[r]) : q.after;
    const long long blocks = (most + (1 << a.shift) - 1) >> a.shift;
    q.live = add >= 0 && blocks <= a.W;
    q.blocks = (int)min(blocks, (long long)a.W);
    q.back = add < 0 ? q.held : 0;
    q.grow = q.live ? max(q.blocks - q.held, 0) : 0;
    return q;
}

// Inclusive sums over the workgroup's threads; `total` holds the last one's.
static __device__ uint64_t scan_threads(uint64_t x, uint64_t *part, uint64_t &total)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    x = scan_wave(x);
    if (lane == 63) part[wave] = x;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
    for (int w = 0; w < kScanWaves; ++w) {
        if (w < wave) before += part[w];
        total += part[w];
    }
    __syncthreads();
    return before + x;
}

// Each thread sums consecutive requests and walks them again with the sums before
// its own, so three scans serve any R.
// rows[r] = {held, blocks after the step, stack place of the first block taken, stack
// place (beyond the free blocks) of the first block given back}.
__global__ __launch_bounds__(kScanThreads) void kv_scan_kernel(const KvTablesArgs a)
{
    __shared__ uint64_t part[kScanWaves];
    const int per = (a.R + kScanThreads - 1) / kScanThreads;
    const int r0 = min((int)threadIdx.x * per, a.R), r1 = min(r0 + per, a.R);
    uint64_t n = 0, back = 0, grow = 0;
    for (int r = r0; r < r1; ++r) {
        const KvRequest q = kv_request(a, r);
        n += q.n;
        back += q.back;
        grow += q.grow;
    }
    uint64_t all_n, all_back, all_grow;
    uint64_t at_n = scan_threads(n, part, all_n) - n;
    uint64_t at_back = scan_threads(back, part, all_back) - back;
    uint64_t at_grow = scan_threads(grow, part, all_grow) - grow;
    const long long free = min(max(a.free_count[0], 0), a.num_blocks);
    // no more blocks than the pool has can be free, whatever the rows claim to hold
    const long long top = min(free + (long long)all_back, (long long)a.num_blocks);
    const long long kTop = 0x7fffffff;
    long long taken = 0;
    for (int r = r0; r < r1; ++r) {
        const KvRequest q = kv_request(a, r);
        const long long end = (long long)at_grow + q.grow;
        const bool ok = q.live && (q.grow == 0 || end <= top);
        a.rows[r] = make_int4(q.held, ok ? max(q.held, q.blocks) : q.held,
                              (int)max(top - 1 - (long long)at_grow, -1LL), (int)at_back);
        a.start[r] = (int)min((long long)at_n, kTop);
        a.context[r] = ok ? (int)min(q.after, kTop) : 0;
        a.granted[r] = ok;
        a.held_out[r] = q.back || a.add[r] < 0 ? 0 : ok ? max(q.held, q.blocks) : q.held;
        if (ok) taken = max(taken, q.grow ? end : 0);
        at_n += q.n;
        at_back += q.back;
        at_grow += q.grow;
    }
    // the largest sum that was granted is what leaves the stack
    for (int d = 32; d; d >>= 1) taken = max(taken, __shfl_xor(taken, d));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = taken;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 0; w < kScanWaves; ++w) taken = max(taken, (long long)part[w]);
        a.start[a.R] = (int)min((long long)all_n, kTop);
        a.tops[0] = (int)free;
        a.tops[1] = (int)top;
        a.free_out[0] = (int)(top - taken);
    }
}

// The block at place `p` of the stack: below `free` the free list's, above it one
// of the blocks just given back, found in its request's row by bisection.
static __device__ int kv_stack_block(const KvTablesArgs &a, int p, int free)
{
    if (p < 0) return -1;
    if (p < free) return a.free_list[p];
    const int x = p - free;
    int lo = 0, hi = a.R;  // the last request whose blocks start at or before x
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (a.rows[m].w <= x) lo = m;
        else hi = m;
    }
    return a.table[lo * a.table_stride + min(x - a.rows[lo].w, a.W - 1)];
}

constexpr int kExpandThreads = 256;

__global__ __launch_bounds__(kExpandThreads) void kv_expand_kernel(const KvTablesArgs a, int row_blocks)
{
    const int free = a.tops[0], top = a.tops[1];
    if ((int)blockIdx.x < row_blocks) {  // a wave per request
        const int r = blockIdx.x * (kExpandThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
        if (r >= a.R) return;
        const int4 q = a.rows[r];
        int32_t *row = a.table + r * a.table_stride;
        if (a.add[r] < 0) {
            for (int i = lane; i < q.x; i += 64)
                if (free + q.w + i < top) a.free_list[free + q.w + i] = row[i];
        } else {
            for (int i = q.x + lane; i < q.y; i += 64) row[i] = kv_stack_block(a, q.z - (i - q.x), free);
        }
        return;
    }
    const int t = ((int)blockIdx.x - row_blocks) * kExpandThreads + threadIdx.x;
    if (t >= a.T) return;
    int64_t slot = -1;
    int pos = -1;
    if (t < a.start[a.R]) {
        int lo = 0, hi = a.R;  // the last request that starts at or before t
        while (hi - lo > 1) {
            const int m = (lo + hi) >> 1;
            if (a.start[m] <= t) lo = m;
            else hi = m;
        }
        if (a.granted[lo]) {
            const int4 q = a.rows[lo];
            pos = max(a.len[lo], 0) + t - a.start[lo];
            const int b = pos >> a.shift;
            const int block = b < q.x ? a.table[lo * a.table_stride + b]
                                      : kv_stack_block(a, q.z - (b - q.x), free);
            slot = ((int64_t)block << a.shift) + (pos & ((1 << a.shift) - 1));
        }
    }
    a.slot[t] = slot;
    a.pos[t] = pos;
}

hipError_t launch_kv_tables(const KvTablesArgs &a, hipStream_t st)
{
    kv_scan_kernel<<<1, kScanThreads, 0, st>>>(a);
    const int rows = (a.R + kExpandThreads / 64 - 1) / (kExpandThreads / 64);
    const int toks = (a.T + kExpandThreads - 1) / kExpandThreads;
    kv_expand_kernel<<<rows + toks, kExpandThreads, 0, st>>>(a, rows);
    return hipGetLastError();
}

// ---- store --------------------------------------------------------------------
//
// Eight components a thread: one load, one store.  Bound by memory.

constexpr int kStoreThreads = 256;

template <class T, class C>
__global__ __launch_bounds__(kStoreThreads) void kv_store_kernel(const KvStoreArgs a)
{
    const int which = blockIdx.y, per_head = a.D / 8, per_token = per_head * a.H;
    const long long i = (long long)blockIdx.x * kStoreThreads + threadIdx.x;
    const int t = (int)(i / per_token);
    if (t >= a.T) return;
    const int c = (int)(i - (long long)t * per_token), h = c / per_head, d = (c - h * per_head) * 8;
    const int64_t slot = a.slot[t];
    if (slot < 0 || slot >= a.slots) return;
    const T *x = (const T *)a.x[which] + t * a.x_token[which] + h * a.x_head[which] + d;
    C *y = (C *)a.c[which] + (slot >> a.shift) * a.c_block[which] +
           (slot & ((1 << a.shift) - 1)) * a.c_token[which] + h * a.c_head[which] + d;
    if constexpr (sizeof(C) == 1) {
        const float s = a.scale[which][h];
        const auto v = *(const Vec<T, 8> *)x;
        float f[8];
        for (int j = 0; j < 8; ++j) f[j] = to_float(v[j]) / s;
        *(uint2 *)y = make_uint2(pack_fp8(f), pack_fp8(f + 4));
    } else {
        *(uint4 *)y = *(const uint4 *)x;
    }
}

template <class T, class C> static void run_store(const KvStoreArgs &a, hipStream_t st)
{
    const long long n = (long long)a.T * a.H * (a.D / 8);
    kv_store_kernel<T, C><<<dim3((unsigned)((n + kStoreThreads - 1) / kStoreThreads), 2),
                            kStoreThreads, 0, st>>>(a);
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
