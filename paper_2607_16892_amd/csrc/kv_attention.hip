// Attention of the new tokens over the paged cache.
//
// One wave per (row, query head): 64 keys a step, a key per lane for the scores,
// the components over the lanes for the weighted values, with the running maximum
// and sum of the softmax.
#include "kv.h"
#include "kv_types.h"

namespace dro {

constexpr int kThreads = 256;

template <class C> static __device__ float cache_at(const void *p, int64_t i)
{
    if constexpr (sizeof(C) == 1) {
        const uint32_t w = ((const uint8_t *)p)[i];
        return __builtin_bit_cast(float, unpack_fp8<bf16, false>(w) << 16);
    } else {
        return to_float(((const C *)p)[i]);
    }
}

template <class T, class C>
__global__ __launch_bounds__(kThreads) void kv_rows_kernel(const KvAttnArgs a)
{
    const long long row = (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= (long long)a.T * a.Hq) return;
    const int t = (int)(row / a.Hq), hq = (int)(row - (long long)t * a.Hq), h = hq / a.G;
    int lo = 0, hi = a.R;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (a.start[m] <= t) lo = m;
        else hi = m;
    }
    const int r = lo;
    const bool mine = a.start[r] <= t && t < a.start[r + 1];
    const long long most = (long long)a.W << a.shift;
    const int ctx = mine ? (int)min((long long)max(a.context[r], 0), most) : 0;
    const long long p = (long long)ctx - a.start[r + 1] + t;
    const int pre = a.prefix ? a.prefix[r] : 0;
    const int first = a.window ? (int)max(p - a.window + 1, 0LL) : 0;
    const int last = (int)min(max(p + 1, (long long)pre), (long long)ctx);
    const float slope = a.slopes ? a.slopes[hq] : 0.0f;
    const float ks = a.k_scale ? a.k_scale[h] * a.scale : a.scale;
    const T *q = (const T *)a.q + t * a.q_token + hq * a.q_head;
    const int32_t *table = a.table + r * a.table_stride;
    float m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
    for (int j0 = first; j0 < last; j0 += 64) {
        const int j = j0 + lane;
        float s = -INFINITY;
        int block = 0;
        if (j < last) {
            block = min(max(table[j >> a.shift], 0), a.num_blocks - 1);
            const int64_t at = block * a.k_block + (j & ((1 << a.shift) - 1)) * a.k_token + h * a.k_head;
            float x = 0.0f;
            for (int d = 0; d < a.D; ++d) x += to_float(q[d]) * cache_at<C>(a.k, at + d);
            s = x * ks;
            if (a.cap > 0) s = a.cap * tanhf(s / a.cap);
            s += slope * (float)(j - p);
        }
        float mt = s;
        for (int d = 32; d; d >>= 1) mt = fmaxf(mt, __shfl_xor(mt, d));
        const float mn = fmaxf(m, mt), mu = mn == -INFINITY ? 0.0f : mn;
        const float e = j < last ? expf(s - mu) : 0.0f, f = expf(m - mu);
        l = l * f + e;
        for (int c = 0; c < 4; ++c) o[c] *= f;
        m = mn;
        for (int jj = 0; jj < min(64, last - j0); ++jj) {
            const float w = __shfl(e, jj);
            const int b = __shfl(block, jj);
            const int64_t at = b * a.v_block + ((j0 + jj) & ((1 << a.shift) - 1)) * a.v_token + h * a.v_head;
            for (int c = 0; c < 4; ++c)
                if (c * 64 + lane < a.D) o[c] += w * cache_at<C>(a.v, at + c * 64 + lane);
        }
    }
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
    const float f = l == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[h] : 1.0f) / l;
    T *out = (T *)a.out + t * a.out_token + hq * a.out_head;
    for (int c = 0; c < 4; ++c)
        if (c * 64 + lane < a.D) out[c * 64 + lane] = (T)(l == 0.0f ? 0.0f : o[c] * f);
    if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? -INFINITY : m + logf(l);
}

template <class T, class C> static void run_rows(const KvAttnArgs &a, hipStream_t st)
{
    const long long rows = (long long)a.T * a.Hq;
    kv_rows_kernel<T, C><<<(unsigned)((rows + 3) / 4), kThreads, 0, st>>>(a);
}

hipError_t launch_kv_attention(const KvAttnArgs &a, int dtype, int cache_dtype, hipStream_t st)
{
    if (dtype == DRO_BF16) {
        if (cache_dtype == DRO_FP8_E4M3) run_rows<bf16, fp8>(a, st);
        else run_rows<bf16, bf16>(a, st);
    } else {
        if (cache_dtype == DRO_FP8_E4M3) run_rows<f16, fp8>(a, st);
        else run_rows<f16, f16>(a, st);
    }
    return hipGetLastError();
}

}  // namespace dro
