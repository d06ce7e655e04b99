// Attention of many rows a request (chunks of prompts, whole prompts).
//
// Bound by the matrix products and, beside them, by the exponentials: 4 D flops and one
// exponential a score.  A workgroup of four waves takes 128 rows (tokens x the G query
// heads of a key head), 32 a wave, and steps through the keys in tiles that pass LDS once
// for all four:
//   S^T = K Q^T        keys x rows: each lane holds half the tile's scores of one row
//   O^T = V^T P^T      components x rows
// so the softmax of a row is a lane's own work and one exchange with lane + 32, the
// weights are the second operand as they stand (the order of the keys within a product
// is theirs; V^T lies in LDS in that order), and rescaling a row is a lane's own product.
// The next tile is on its way from memory to registers while one is worked on.
#pragma once

#include "kv_math.h"
#include "kv_sched.h"

namespace dro {

constexpr int kPrefillRows = 128;

constexpr int prefill_keys(int DP) { return 8192 / DP; }  // 16 KB of keys, as much of values
constexpr int prefill_groups(int DP) { return DP == 256 ? 1 : 2; }  // workgroups a compute unit

// 32 x 32 tile over 16 products: lane holds row (column) lane % 32, products (lane / 32) 8
// .. + 8; result: column lane % 32, rows 8 b + 4 (lane / 32) + c in place 4 b + c.
template <class T> __device__ __forceinline__ f32x16 mfma32(u32x4 x, u32x4 y, f32x16 c)
{
    if constexpr (__is_same(T, bf16))
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Vec<bf16, 8>, x),
                                                       __builtin_bit_cast(Vec<bf16, 8>, y), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Vec<f16, 8>, x),
                                                      __builtin_bit_cast(Vec<f16, 8>, y), c, 0, 0, 0);
}

__device__ __forceinline__ float max_halves(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_halves(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

template <class T, class C, int DP, bool MODS>
__global__ __launch_bounds__(256, prefill_groups(DP)) void kv_prefill_kernel(
    const KvAttnArgs a, const KvCut cut, const KvTiles tiles, bool pad, float *part_o, float2 *part_ml,
    KvJoin *joins)
{
    constexpr int E = sizeof(C);
    constexpr bool F8 = E == 1;
    constexpr int KT = prefill_keys(DP);
    constexpr int S = DP / 16;           // steps of 16 components of a score
    constexpr int NT = KT / 32;          // score tiles
    constexpr int ND = DP / 32;          // component tiles
    constexpr int KRow = DP * 2 + 16;    // bytes of a key's row, and of a component's row of
    constexpr int VRow = KT * 2 + 16;    // values: 16 more, so 16 rows start on all banks
    constexpr int KG = KT / 8;           // groups of 8 keys
    constexpr int W = E * 2;             // dwords of 8 components in the cache
    __shared__ __align__(16) char sk[2][KT * KRow];
    __shared__ __align__(16) char sv[2][DP * VRow];
    __shared__ int odd[2][2];  // a tile holds such values, by the wave that staged them

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n32 = lane & 31, half = lane >> 5;
    // runs next to one another on one die: the tiles of a head share its keys in the L2
    const uint32_t per_die = gridDim.x / kDies;
    const uint32_t group = (blockIdx.x % kDies) * per_die + blockIdx.x / kDies;

    if (pad) zero_rows<T>(a);
    if (threadIdx.x == 0) joins[group].parts = 0;
    const uint64_t all1 = tiles.sums[tiles.count[0]], all = all1 * a.H;
    const uint64_t run = kv_tile_run(cut, all);
    uint64_t unit = group * run;
    const uint64_t end = min(unit + run, all);
    while (unit < end) {
        const int h = (int)(unit / all1);
        const uint64_t u1 = unit - h * all1;
        const int entry = __builtin_amdgcn_readfirstlane(kv_find(tiles.sums, tiles.count[0], u1));
        const int2 rt = tiles.tiles[entry];
        const int r = rt.x, tile = rt.y;
        const KvShare sh = kv_share(a, cut, r);
        const int item_steps = (int)(tiles.sums[entry + 1] - tiles.sums[entry]);
        const int step0 = (int)(u1 - tiles.sums[entry]);
        const int go = (int)min(end - unit, (uint64_t)(item_steps - step0));
        unit += go;
        const int first_token = min(max(a.start[r], 0), a.T);
        const int row0 = tile * kPrefillRows;
        const int rows = min(sh.n * a.G - row0, kPrefillRows);
        const int prefix = a.prefix ? a.prefix[r] : 0;
        const KvRange top = kv_row_range(a, sh.ctx, sh.n, row0 / a.G, prefix);
        const KvRange bot = kv_row_range(a, sh.ctx, sh.n, (row0 + rows - 1) / a.G, prefix);
        const int base = top.lo & ~31;
        const int k0 = min(base + step0 * KT, bot.hi), k1 = min(base + (step0 + go) * KT, bot.hi);
        const int steps = (k1 - k0 + KT - 1) / KT;

        // this wave's rows, and this lane's
        const int wrow = min(wave * 32, rows - 1), wlast = min(wave * 32 + 31, rows - 1);
        const KvRange wtop = kv_row_range(a, sh.ctx, sh.n, (row0 + wrow) / a.G, prefix);
        const KvRange wbot = kv_row_range(a, sh.ctx, sh.n, (row0 + wlast) / a.G, prefix);
        const bool idle = wave * 32 >= rows;
        const int row = row0 + min(wave * 32 + n32, rows - 1);
        const int token = row / a.G, hq = h * a.G + row - token * a.G;
        const KvRange see = kv_row_range(a, sh.ctx, sh.n, token, prefix);
        const int p_row = sh.ctx - sh.n + token;

        u32x4 q[S];
        {
            const char *p = (const char *)a.q + 2 * ((int64_t)(first_token + token) * a.q_token + hq * a.q_head);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int d = s * 16 + half * 8;
                q[s] = d < a.D ? *(const u32x4 *)(p + 2 * d) : u32x4{0, 0, 0, 0};
            }
        }
        const float ks = F8 ? a.scale * a.k_scale[h] : a.scale;
        const float to_exp = MODS ? ks : ks * kLog2e;
        const float slope = MODS && a.slopes ? a.slopes[hq] : 0.0f;
        const float inv_cap = MODS && a.cap > 0.0f ? 1.0f / a.cap : 0.0f;

        // Staging: waves 0 and 1 take the values (8 keys x 8 components a thread, in the
        // order of the products), waves 2 and 3 the keys (8 rows x 8 components).  A
        // thread's keys lie in one group of 16, so in one block.
        const bool values = wave < 2;
        const int st = threadIdx.x & 127;
        const int kg = st % KG, dg = st / KG;              // values
        const int kc = st % (DP / 8), kr = st / (DP / 8);  // keys
        const int in_tile = values ? (kg >> 1) * 16 : (kr >> 1) * 16;
        const int in_group = values ? (kg & 1) * 4 : (kr & 1) * 8;
        const int sd = (values ? dg : kc) * 8;
        const char *src = values ? (const char *)a.v + (int64_t)h * a.v_head * E
                                 : (const char *)a.k + (int64_t)h * a.k_head * E;
        const int64_t s_block = (values ? a.v_block : a.k_block) * E;
        const int s_token = (int)(values ? a.v_token : a.k_token) * E;
        const int s_skip = values ? 8 * s_token : 4 * s_token;  // from row 3 to row 4, less 4 rows
        const int32_t *table = a.table + (int64_t)r * a.table_stride;
        const int in_block = (1 << a.shift) - 1;
        int id = 0;
        auto load_id = [&](int u) { id = table[min(k0 + u * KT + in_tile, k1 - 1) >> a.shift]; };
        Words<W> reg[8];
        auto load = [&](int u) {
            const int at = ((k0 + u * KT + in_tile) & in_block) + in_group;
            const char *p = src + min(max(id, 0), a.num_blocks - 1) * s_block + (uint32_t)(at * s_token + sd * E);
            const char *p4 = p + s_skip;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                Words<W> x{};
                if (sd < a.D) x = load_words<W>((i < 4 ? p : p4) + (i & 3) * (int64_t)s_token, 0);
                reg[i] = x;
            }
        };
        auto key_of = [&](int i) { return in_tile + in_group + (values ? (i >> 2) * 8 + (i & 3) : i); };
        // registers to LDS; values that no row of the tile of rows sees become zero, and in
        // tiles that hide keys from some rows infinities and NaN do, for `odd`
        auto store = [&](int u) {
            const int b = u & 1, key0 = k0 + u * KT;
            u32x4 x[8];
            if (values) {
                const bool edge = key0 < bot.lo || key0 + KT > min(top.hi, k1);
                if (edge) {
                    uint32_t bad = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int key = key0 + key_of(i);
                        const bool keep = key >= top.lo && key < bot.hi;
#pragma unroll
                        for (int j = 0; j < W; ++j) {
                            const uint32_t w = keep ? reg[i].w[j] : 0, mask = nonfinite_mask<C>(w);
                            bad |= mask;
                            reg[i].w[j] = w & ~mask;
                        }
                    }
                    bad = __any(bad);
                    if (lane == 0) odd[b][wave] = bad;
                } else if (lane == 0) {
                    odd[b][wave] = 0;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (F8)
                    x[i] = u32x4{unpack_fp8<T, false>(reg[i].w[0]), unpack_fp8<T, true>(reg[i].w[0]),
                                 unpack_fp8<T, false>(reg[i].w[1]), unpack_fp8<T, true>(reg[i].w[1])};
                else
                    x[i] = u32x4{reg[i].w[0], reg[i].w[1], reg[i].w[2], reg[i].w[3]};
            }
            if (values) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {  // component 8 dg + j: keys in order
                    u32x4 y;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        y[c] = __builtin_amdgcn_perm(x[2 * c + 1][j / 2], x[2 * c][j / 2],
                                                     j & 1 ? 0x07060302u : 0x05040100u);
                    *(u32x4 *)&sv[b][(dg * 8 + j) * VRow + kg * 16] = y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) *(u32x4 *)&sk[b][(kr * 8 + i) * KRow + kc * 16] = x[i];
            }
        };

        float m = -INFINITY, l = 0.0f;
        f32x16 o[ND];
#pragma unroll
        for (int j = 0; j < ND; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.0f;

        __syncthreads();  // the last item's tiles are read
        if (steps) {
            load_id(0);
            load(0);
            load_id(1);
            store(0);
        }
        for (int u = 0; u < steps; ++u) {
            const int b = u & 1, key0 = k0 + u * KT;
            __syncthreads();  // tile u is in LDS, tile u - 1 is read
            if (u + 1 < steps) {
                load(u + 1);
                load_id(u + 2);
            }
            const bool none = idle || key0 >= wbot.hi || key0 + KT <= wtop.lo;
            if (!none) {
                f32x16 s[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
                    for (int x = 0; x < S; ++x)
                        s[t] = mfma32<T>(*(const u32x4 *)&sk[b][(t * 32 + n32) * KRow + x * 32 + half * 16], q[x], s[t]);
                }
                const bool edge = key0 < wbot.lo || key0 + KT > min(wtop.hi, k1);
                float mt = -INFINITY;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = key0 + t * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
                        if constexpr (MODS) {
                            float x = s[t][i] * to_exp;
                            if (a.cap > 0.0f) x = a.cap * tanh_fast(x * inv_cap);
                            s[t][i] = (x + slope * (float)(key - p_row)) * kLog2e;
                        } else {
                            s[t][i] *= to_exp;
                        }
                        if (edge) s[t][i] = key >= see.lo && key < see.hi ? s[t][i] : -INFINITY;
                        mt = fmaxf(mt, s[t][i]);
                    }
                mt = max_halves(mt);
                if (__any(mt > m + kSlack)) {
                    const float to = fmaxf(m, mt);
                    const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
                    m = to;
                    l *= f;
#pragma unroll
                    for (int j = 0; j < ND; ++j)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[j][i] *= f;
                }
                const float mu = m == -INFINITY ? 0.0f : m;
                u32x4 w[NT * 2];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        s[t][i] = __builtin_amdgcn_exp2f(s[t][i] - mu);
                        s[t][i + 1] = __builtin_amdgcn_exp2f(s[t][i + 1] - mu);
                        l += s[t][i] + s[t][i + 1];
                        w[2 * t + (i >> 3)][(i >> 1) & 3] = pack2<T>(s[t][i], s[t][i + 1]);
                    }
                if (odd[b][0] | odd[b][1]) {  // (rare) infinities and NaN, to the rows that see them
                    for (int x = 0; x < NT * 16; ++x) {
                        float mine = 0.0f;
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 16; ++i) mine = x == t * 16 + i ? s[t][i] : mine;
                        for (int g = 0; g < 2; ++g) {
                            const float wt = __shfl(mine, n32 + 32 * g);
                            const int key = key0 + (x >> 4) * 32 + ((x >> 2) & 3) * 8 + g * 4 + (x & 3);
                            const bool seen = key >= see.lo && key < see.hi;
                            const int kk = min(key, k1 - 1);
                            const int id = min(max(table[kk >> a.shift], 0), a.num_blocks - 1);
                            const char *at = (const char *)a.v + (id * a.v_block + (int64_t)(kk & in_block) * a.v_token +
                                                                  (int64_t)h * a.v_head) * E;
                            int D = a.D;
                            asm volatile("" : "+s"(D));  // compared with anew: the masks would not fit
#pragma unroll
                            for (int j = 0; j < ND; ++j)
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const int d = j * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
                                    const float y = d < D ? value_at<C>(at, d) : 0.0f;
                                    o[j][i] += seen && !__builtin_isfinite(y) ? wt * y : 0.0f;
                                    __builtin_amdgcn_sched_barrier(0);
                                }
                        }
                    }
                }
#pragma unroll
                for (int x = 0; x < NT * 2; ++x)
#pragma unroll
                    for (int j = 0; j < ND; ++j)
                        o[j] = mfma32<T>(*(const u32x4 *)&sv[b][(j * 32 + n32) * VRow + x * 32 + half * 16], w[x], o[j]);
            }
            if (u + 1 < steps) store(u + 1);
        }

        l = sum_halves(l);
        const bool whole = go >= item_steps;
        if (wave * 32 + n32 < rows) {
            const int64_t t = first_token + token;
            const int64_t at = kv_part(group, step0 == 0) * kPrefillRows + wave * 32 + n32;
            const float inv = l == 0.0f ? 0.0f : (F8 ? a.v_scale[h] : 1.0f) / l;
            T *out = (T *)a.out + t * a.out_token + hq * a.out_head;
#pragma unroll
            for (int j = 0; j < ND; ++j)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int d = j * 32 + (i >> 2) * 8 + half * 4;
                    if (!whole)
                        *(f32x4 *)&part_o[at * DP + d] = f32x4{o[j][i], o[j][i + 1], o[j][i + 2], o[j][i + 3]};
                    else if (d < a.D)
                        *(uint2 *)(out + d) = l == 0.0f ? make_uint2(0, 0)
                                                        : make_uint2(pack2<T>(o[j][i] * inv, o[j][i + 1] * inv),
                                                                     pack2<T>(o[j][i + 2] * inv, o[j][i + 3] * inv));
                }
            if (half == 0) {
                if (!whole) part_ml[at] = make_float2(m, l);
                else if (a.lse) a.lse[t * a.Hq + hq] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
            }
        }
        if (!whole && step0 == 0 && threadIdx.x == 0) {
            KvJoin &j = joins[group];
            j.parts = 1 + (int)((item_steps - go + run - 1) / run);
            j.first_token = first_token;
            j.row0 = row0;
            j.rows = rows;
            j.head = h;
        }
    }
}

template <class T, class C, int DP>
void run_kv_prefill(const KvAttnArgs &a, const KvCut &c, const KvTiles &t, bool pad, float *o, float2 *ml,
                    KvJoin *joins, hipStream_t st)
{
    if (a.cap > 0.0f || a.slopes) kv_prefill_kernel<T, C, DP, true><<<c.groups, 256, 0, st>>>(a, c, t, pad, o, ml, joins);
    else kv_prefill_kernel<T, C, DP, false><<<c.groups, 256, 0, st>>>(a, c, t, pad, o, ml, joins);
}

template <class T>
void launch_kv_prefill(const KvAttnArgs &a, const KvCut &c, const KvTiles &t, int cache_dtype, int DP, bool pad,
                       float *o, float2 *ml, KvJoin *joins, hipStream_t st)
{
    const bool f8 = cache_dtype == DRO_FP8_E4M3;
    if (DP == 64) (f8 ? run_kv_prefill<T, fp8, 64> : run_kv_prefill<T, T, 64>)(a, c, t, pad, o, ml, joins, st);
    else if (DP == 128) (f8 ? run_kv_prefill<T, fp8, 128> : run_kv_prefill<T, T, 128>)(a, c, t, pad, o, ml, joins, st);
    else (f8 ? run_kv_prefill<T, fp8, 256> : run_kv_prefill<T, T, 256>)(a, c, t, pad, o, ml, joins, st);
}

}  // namespace dro
