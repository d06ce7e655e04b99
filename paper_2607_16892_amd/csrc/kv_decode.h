// Attention of few rows a request (single tokens, short chunks).
//
// Bound by the keys and values that it reads, so every wave takes its own 32 keys at a
// time straight from memory to registers, and nothing of them passes LDS:
//   S^T = K Q^T        keys x rows: a lane holds 8 weights of one row
//   O^T = V^T P^T      components x rows
// with 16 rows a tile (the G query heads of a key head, then tokens).  The order of the
// keys within a product does not matter as long as weights and values agree, so a
// lane's 8 weights are the second operand as they stand, and V^T needs only the
// transpose of 8 rows x 16 bytes inside each lane.  A workgroup is one wave with its own
// run of steps: while one begins or ends an item, the other seven of the compute unit
// read on.  (Four waves that shared a run and met in LDS after each item: 124 us for 64
// requests of 50 to 8192 keys on 8 heads, 464 MB, against 102 now: 4.7 TB/s in
// the kernel, and 5.2 from 128 requests of 1000 to 16,384 keys in 8 bits.)
#pragma once

#include "kv_math.h"
#include "kv_sched.h"

namespace dro {

constexpr int kDecodeRows = 16;

// Waves a SIMD, so registers: the keys of the next step and this one's values (32 x 256 bytes
// each) take 64 of a wave's, beside queries and sums.  With 256 components one wave has both on
// their way where two have not: 64 requests of 50 to 8192 keys on 8 heads, 16 bits 182 us and 245 with
// two, 8 bits 117 and 129.
constexpr int decode_waves(int DP, int E) { return DP == 256 ? 1 : DP * E >= 256 ? 2 : DP * E >= 128 ? 3 : 4; }

template <class T, class C, int DP, bool FULL>
__global__ __launch_bounds__(64, decode_waves(DP, (int)sizeof(C))) void kv_decode_kernel(
    const KvAttnArgs a, const KvCut cut, const uint64_t *sums, bool pad, float *part_o, float2 *part_ml,
    KvJoin *joins)
{
    constexpr int E = sizeof(C);
    constexpr int S = DP / 32;             // steps of 32 components of a score
    constexpr int VW = DP / 16;            // components a lane reads of a value row
    constexpr bool F8 = sizeof(C) == 1;
    constexpr int KWords = F8 ? S * 2 : S * 4;   // dwords a lane reads of a key row
    constexpr int VWords = F8 ? VW / 4 : VW / 2; // and of a value row
    __shared__ KvLds lds;

    const int lane = threadIdx.x, n16 = lane & 15, grp = lane >> 4;

    KvSched sched;
    sched.init(a, cut, sums, lds);
    if (threadIdx.x == 0) joins[blockIdx.x].parts = 0;
    uint64_t unit = blockIdx.x * sched.run;
    const uint64_t end = min(unit + sched.run, sched.all);
    if (pad && (gridDim.x - 1) * sched.run < sched.all) {
        zero_rows<T>(a, blockIdx.x, gridDim.x);
    } else if (pad && unit >= end) {
        const uint32_t busy = (uint32_t)((sched.all + sched.run - 1) / sched.run);
        zero_rows<T>(a, blockIdx.x - busy, gridDim.x - busy);
    }
    while (unit < end) {
        const KvItem it = sched.item(a, cut, sums, lds, unit);
        const int go = (int)min(end - unit, (uint64_t)(it.steps - it.step));  // steps of this item
        unit += go;
        const int h = it.head, r = it.r;
        const int row0 = it.tile * kDecodeRows;
        const int rows = min(it.n * a.G - row0, kDecodeRows);
        const int prefix = a.prefix ? a.prefix[r] : 0;

        // this lane's row
        const int row = row0 + min(n16, rows - 1);
        const int token = row / a.G, hq = h * a.G + row - token * a.G;
        const KvRange see = kv_row_range(a, it.ctx, it.n, token, prefix);
        // the tile's keys: those that some row sees, and those that every row sees
        const KvRange top = kv_row_range(a, it.ctx, it.n, row0 / a.G, prefix);
        const KvRange bot = kv_row_range(a, it.ctx, it.n, (row0 + rows - 1) / a.G, prefix);
        const int all_lo = bot.lo, all_hi = top.hi;
        const int base = top.lo & ~(kStepKeys - 1);
        const int k0 = min(base + it.step * kStepKeys, bot.hi);
        const int k1 = min(base + (it.step + go) * kStepKeys, bot.hi);

        // queries: second operand of the scores
        u32x4 q[S];
        {
            const char *p = (const char *)a.q + 2 * ((int64_t)(it.first_token + token) * a.q_token + hq * a.q_head);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int d = F8 ? (s >> 1) * 64 + grp * 16 + (s & 1) * 8 : s * 32 + grp * 8;
                q[s] = FULL || d < a.D ? *(const u32x4 *)(p + 2 * d) : u32x4{0, 0, 0, 0};
            }
        }
        const float ks = F8 ? a.scale * a.k_scale[h] : a.scale;
        // scores to exponents of two: times to_exp, plus slope a key's distance; with a cap
        // to_exp leads to the exponent of its tanh
        const float slope = a.slopes ? a.slopes[hq] * kLog2e : 0.0f;
        const float cap = a.cap * kLog2e, to_exp = a.cap > 0.0f ? ks * (2.0f * kLog2e) / a.cap : ks * kLog2e;
        const int p_row = it.ctx - it.n + token;

        const char *kp = (const char *)a.k + (int64_t)h * a.k_head * E;
        const char *vp = (const char *)a.v + (int64_t)h * a.v_head * E;
        const int in_block = (1 << a.shift) - 1;
        const uint32_t k_lane = (uint32_t)(n16 * (int)a.k_token + (F8 ? grp * 16 : grp * 8)) * E;
        const uint32_t v_lane = (uint32_t)(grp * 4 * (int)a.v_token + n16 * VW) * E;
        const int32_t *table = a.table + (int64_t)r * a.table_stride;

        float m = -INFINITY, l = 0.0f;
        f32x4 o[VW];
#pragma unroll
        for (int j = 0; j < VW; ++j) o[j] = f32x4{0, 0, 0, 0};

        // Steps: keys k0 + 32 u.  A lane holds the block of one group of 16 keys, 32 steps ahead.
        const int steps = (k1 - k0 + kStepKeys - 1) / kStepKeys;
        int ids = 0;
        bool found = false;  // infinities or NaN among values that only some rows see
        auto fetch_ids = [&](int u) {
            const int key = k0 + (u + (lane >> 1)) * kStepKeys + (lane & 1) * 16;
            ids = min(max(table[min(key, k1 - 1) >> a.shift], 0), a.num_blocks - 1);
        };
        auto base_of = [&](const char *p, int64_t block_stride, int64_t token_stride, int u, int t) {
            const int id = __builtin_amdgcn_readlane(ids, 2 * (u & 31) + t);
            const int key = k0 + u * kStepKeys + t * 16;
            return p + ((int64_t)id * block_stride + (int64_t)(key & in_block) * token_stride) * E;
        };
        Words<KWords> k[2];
        auto load_k = [&](int u) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const char *p = base_of(kp, a.k_block, a.k_token, u, t);
                if constexpr (FULL) {
                    constexpr int L = F8 ? S / 2 : S;  // 16-byte loads
#pragma unroll
                    for (int s = 0; s < L; ++s) {
                        const Words<4> x = load_words<4>(p + s * 64, k_lane);
#pragma unroll
                        for (int j = 0; j < 4; ++j) k[t].w[4 * s + j] = x.w[j];
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        constexpr int N = F8 ? 2 : 4;
                        const int d = F8 ? (s >> 1) * 64 + grp * 16 + (s & 1) * 8 : s * 32 + grp * 8;
                        Words<N> x{};
                        if (d < a.D) x = load_words<N>(p + (F8 ? (s >> 1) * 64 + (s & 1) * 8 : s * 64), k_lane);
#pragma unroll
                        for (int j = 0; j < N; ++j) k[t].w[N * s + j] = x.w[j];
                    }
                }
            }
        };

        if (steps) {
            fetch_ids(0);
            load_k(0);
        }
        for (int u = 0; u < steps; ++u) {
            const int key0 = k0 + u * kStepKeys;
            const bool edge = key0 < all_lo || key0 + kStepKeys > min(all_hi, k1);
            Words<VWords> v[8];
            auto load_v = [&]() {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const char *p = base_of(vp, a.v_block, a.v_token, u, t);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const char *at = p + (int64_t)i * a.v_token * E;
                        if constexpr (FULL) {
                            v[t * 4 + i] = load_words<VWords>(at, v_lane);
                        } else {
                            constexpr int N = F8 ? 2 : 4, P = VWords < N ? VWords : N;
#pragma unroll
                            for (int x = 0; x < VWords; x += P) {
                                Words<P> y{};
                                if (n16 * VW + x * (4 / E) < a.D) y = load_words<P>(at + 4 * x, v_lane);
#pragma unroll
                                for (int j = 0; j < P; ++j) v[t * 4 + i].w[x + j] = y.w[j];
                            }
                        }
                    }
                }
            };
            load_v();

            f32x4 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int x = 0; x < S; ++x) {
                    u32x4 kf;
                    if constexpr (F8) {
                        kf = u32x4{unpack_fp8<T, false>(k[t].w[2 * x]), unpack_fp8<T, true>(k[t].w[2 * x]),
                                   unpack_fp8<T, false>(k[t].w[2 * x + 1]), unpack_fp8<T, true>(k[t].w[2 * x + 1])};
                    } else {
                        kf = u32x4{k[t].w[4 * x], k[t].w[4 * x + 1], k[t].w[4 * x + 2], k[t].w[4 * x + 3]};
                    }
                    s[t] = mfma16<T>(kf, q[x], s[t]);
                }
            }
            // the next step's keys are on their way while this one's values are used; the blocks
            // of the next 32 steps only after this step's values have been asked for
            if (u + 1 < steps) {
                if (((u + 1) & 31) == 0) fetch_ids(u + 1);
                load_k(u + 1);
            }

            // scores to exponents of two
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = s[i >> 2][i & 3] * to_exp;
            if (a.cap > 0.0f || a.slopes) {
                const float b0 = slope * (float)(key0 + grp * 4 - p_row);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float add = __builtin_fmaf((float)((i >> 2) * 16 + (i & 3)), slope, b0);
                    e[i] = a.cap > 0.0f ? tanh_scaled(e[i], cap, add) : e[i] + add;
                }
            }
            if (edge) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = key0 + (i >> 2) * 16 + grp * 4 + (i & 3);
                    e[i] = key >= see.lo && key < see.hi ? e[i] : -INFINITY;
                }
            }
            float mt = fmaxf(fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3])), fmaxf(fmaxf(e[4], e[5]), fmaxf(e[6], e[7])));
            mt = max_groups(mt);
            if (__any(has_to_raise<T>(mt, m))) {
                const float to = fmaxf(m, mt - kUnit<T>);
                const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= f;
#pragma unroll
                for (int j = 0; j < VW; ++j) o[j] *= f;
            }
            const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(e[i] - mu);
                l += e[i];
            }
            const u32x4 w = {pack2<T>(e[0], e[1]), pack2<T>(e[2], e[3]), pack2<T>(e[4], e[5]), pack2<T>(e[6], e[7])};

            if (edge) {
                // a weight of zero does not silence an infinity or a NaN: values that no row of
                // the tile sees become zero, and those that some see are added after the last
                // step, to these rows alone
                uint32_t odd = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = key0 + (i >> 2) * 16 + grp * 4 + (i & 3);
                    const bool keep = key >= top.lo && key < bot.hi;
#pragma unroll
                    for (int j = 0; j < VWords; ++j) {
                        v[i].w[j] = keep ? v[i].w[j] : 0;
                        odd |= nonfinite_mask<C>(v[i].w[j]);
                    }
                }
                if (__any(odd)) {
                    found = true;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int j = 0; j < VWords; ++j) v[i].w[j] &= ~nonfinite_mask<C>(v[i].w[j]);
                }
            }
            // V^T: dword y of column j holds rows 2y and 2y + 1
#pragma unroll
            for (int j = 0; j < VWords; ++j) {
                if constexpr (F8) {
                    u32x4 x[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t lo = v[2 * y].w[j], hi = v[2 * y + 1].w[j];
                        const uint32_t x0 = __builtin_amdgcn_perm(hi, lo, 0x05010400u);
                        const uint32_t x1 = __builtin_amdgcn_perm(hi, lo, 0x07030602u);
                        x[0][y] = unpack_fp8<T, false>(x0);
                        x[1][y] = unpack_fp8<T, true>(x0);
                        x[2][y] = unpack_fp8<T, false>(x1);
                        x[3][y] = unpack_fp8<T, true>(x1);
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[4 * j + c] = mfma16<T>(x[c], w, o[4 * j + c]);
                } else {
                    u32x4 x[2];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t lo = v[2 * y].w[j], hi = v[2 * y + 1].w[j];
                        x[0][y] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
                        x[1][y] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) o[2 * j + c] = mfma16<T>(x[c], w, o[2 * j + c]);
                }
            }
        }

        if (found) {
            // An infinity stays one here whatever its weight, and a NaN.  (In steps that all rows
            // see it goes through the product, where a weight that rounds to zero makes it NaN:
            // looking at every value of every step would cost more than it is worth.)
            for (int key = k0; key < k1; ++key) {
                const int step = k0 + ((key - k0) & ~(kStepKeys - 1));
                if (step >= all_lo && step + kStepKeys <= min(all_hi, k1)) continue;  // not zeroed
                const bool seen = key >= see.lo && key < see.hi;
                const int id = min(max(table[key >> a.shift], 0), a.num_blocks - 1);
                const char *at = vp + (id * a.v_block + (int64_t)(key & in_block) * a.v_token) * E;
                if (!row_nonfinite<C>(at, a.D * E)) continue;
                int D = a.D;
                asm volatile("" : "+s"(D));  // compared with anew: 64 addresses would not fit
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < VW; ++j) {
                        const int d = VW * (grp * 4 + c) + j;
                        const float y = value_at<C>(at, FULL ? d : min(d, D - 1));
                        if (seen && !__builtin_isfinite(y)) o[j][c] += y;
                        __builtin_amdgcn_sched_barrier(0);  // rare: few registers, not speed
                    }
            }
        }
        l = sum_groups(l);
        const bool whole = go >= it.steps;
        if (n16 < rows) {
            const int64_t t = it.first_token + token;
            const int64_t at = (int64_t)kv_part(blockIdx.x, it.step == 0) * kDecodeRows + n16;
            const float inv = l == 0.0f ? 0.0f : (F8 ? a.v_scale[h] : 1.0f) / l;
            T *out = (T *)a.out + t * a.out_token + hq * a.out_head;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int j = 0; j < VW; j += 4) {
                    const int d = VW * (grp * 4 + c) + j;
                    const f32x4 x = {o[j][c], o[j + 1][c], o[j + 2][c], o[j + 3][c]};
                    if (!whole)
                        *(f32x4 *)&part_o[at * DP + d] = x;
                    else if (FULL || d < a.D)
                        *(uint2 *)(out + d) = l == 0.0f ? make_uint2(0, 0)
                                                        : make_uint2(pack2<T>(x[0] * inv, x[1] * inv),
                                                                     pack2<T>(x[2] * inv, x[3] * inv));
                }
            if (grp == 0) {
                if (!whole) part_ml[at] = make_float2(m, l);
                else if (a.lse) a.lse[t * a.Hq + hq] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
            }
        }
        if (!whole && it.step == 0 && lane == 0) {
            // (the item's last step lies `it.steps - go` steps beyond this run's end)
            KvJoin &j = joins[blockIdx.x];
            j.parts = 1 + (int)((it.steps - go + sched.run - 1) / sched.run);
            j.first_token = it.first_token;
            j.row0 = row0;
            j.rows = rows;
            j.head = h;
            j.first = kv_part(blockIdx.x, true);
            j.next = kv_part(blockIdx.x + 1, false);
            j.stride = 2;
        }
    }
}

template <class T, class C>
void run_kv_decode(const KvAttnArgs &a, const KvCut &c, const uint64_t *sums, int DP, bool pad, float *o,
                   float2 *ml, KvJoin *joins, hipStream_t st)
{
    constexpr int kThreads = 64;
    const bool full = a.D == DP;
    if (DP == 64) {
        if (full) kv_decode_kernel<T, C, 64, true><<<c.groups, kThreads, 0, st>>>(a, c, sums, pad, o, ml, joins);
        else kv_decode_kernel<T, C, 64, false><<<c.groups, kThreads, 0, st>>>(a, c, sums, pad, o, ml, joins);
    } else if (DP == 128) {
        if (full) kv_decode_kernel<T, C, 128, true><<<c.groups, kThreads, 0, st>>>(a, c, sums, pad, o, ml, joins);
        else kv_decode_kernel<T, C, 128, false><<<c.groups, kThreads, 0, st>>>(a, c, sums, pad, o, ml, joins);
    } else {
        if (full) kv_decode_kernel<T, C, 256, true><<<c.groups, kThreads, 0, st>>>(a, c, sums, pad, o, ml, joins);
        else kv_decode_kernel<T, C, 256, false><<<c.groups, kThreads, 0, st>>>(a, c, sums, pad, o, ml, joins);
    }
}

template <class T>
void launch_kv_decode(const KvAttnArgs &a, const KvCut &c, const uint64_t *sums, int cache_dtype, int DP,
                      bool pad, float *o, float2 *ml, KvJoin *joins, hipStream_t st)
{
    if (cache_dtype == DRO_FP8_E4M3) run_kv_decode<T, fp8>(a, c, sums, DP, pad, o, ml, joins, st);
    else run_kv_decode<T, T>(a, c, sums, DP, pad, o, ml, joins, st);
}

}  // namespace dro
