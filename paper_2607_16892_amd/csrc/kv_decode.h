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

#include <type_traits>
#include <utility>

#include "kv_math.h"
#include "kv_sched.h"

namespace dro {

constexpr int kDecodeRows = 16;

// Waves a SIMD, so registers: the keys of the next step and this one's values (32 x 256 bytes
// each) take 64 of a wave's, beside queries and sums.  With 256 components one wave has both on
// their way where two have not: 64 requests of 50 to 8192 keys on 8 heads, 16 bits 182 us and 245 with
// two, 8 bits 117 and 129.
constexpr int decode_waves(int DP, int E) { return DP == 256 ? 1 : DP * E >= 256 ? 2 : DP * E >= 128 ? 3 : 4; }

// Caches in shared scales.  A lane reads 16 bytes of a key row at a time, so its codes of 4 bits are
// one whole group (with 64 components half of one), of 8 bits half a group: one power a read.  Of the
// values it reads the powers of its four rows at once, which lie next to one another.  Codes are
// widened by one instruction a pair that takes the power as well, to exactly what they stand for (in
// f16 rounded), and from there on are values of T like any other.
//
// 128 components of 4 bits: an instruction issues in 73 % of a SIMD's cycles (435 vector ones for 64 keys: 128 that
// widen, 64 that pair rows), so with two waves 184 us for 128 requests of 1000 to 16,384 keys, 64 heads
// on 8, with three 177 (4.9 TB/s in the kernel), with four 193, as registers run short; 64 keys a step
// instead of 32 were 1 % faster there with two waves, but 11 % slower for 64 requests of 50 to 8192 keys.
// In 8 bits with two waves 298 us, with three 325, where again there are too few registers; of 256
// components 89 us with one and 123 with two for 64 requests of 500 to 8192 keys, 16 heads on 4.
template <class C> constexpr int decode_waves_of(int DP)
{
    if (__is_same(C, mx4)) return DP == 256 ? 2 : DP == 128 ? 3 : 4;
    if (__is_same(C, mx8)) return DP == 256 ? 1 : DP == 128 ? 2 : 4;
    return decode_waves(DP, (int)sizeof(C));
}

// f(0), .., f(N - 1), each with its number as a constant
template <class F, int... I> __device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void each(F f) { each_of(f, std::make_integer_sequence<int, N>{}); }

template <class T, class C, int DP, bool FULL, class A>
__global__ __launch_bounds__(64, decode_waves_of<C>(DP)) void kv_decode_kernel(
    const A a, const KvCut cut, const uint64_t *sums, bool pad, float *part_o, float2 *part_ml,
    KvJoin *joins)
{
    constexpr int S = DP / 32;             // steps of 32 components of a score
    constexpr int VW = DP / 16;            // components a lane reads of a value row
    constexpr bool F8 = __is_same(C, fp8), MX = kMx<C>, FOUR = __is_same(C, mx4);
    constexpr int KWords = FOUR ? S : sizeof(C) == 1 ? S * 2 : S * 4;  // dwords a lane reads of a key row
    constexpr int VWords = F8 ? VW / 4 : VW / 2;  // and of a value row
    constexpr int KReads = FOUR ? (S + 3) / 4 : S / 2;  // shared scales: reads of a key row, a power each
    constexpr int VRaw = FOUR ? (VW + 7) / 8 : VW / 4;  // and dwords of a value row
    __shared__ KvLdsOf<A> lds;

    const int lane = threadIdx.x, n16 = lane & 15, grp = lane >> 4;
    // the first of the 8 components that this lane multiplies in step x of a score
    auto component = [&](int x) {
        if constexpr (FOUR) return DP == 64 ? grp * 16 + x * 8 : (x >> 2) * 128 + grp * 32 + (x & 3) * 8;
        else if constexpr (F8 || MX) return (x >> 1) * 64 + grp * 16 + (x & 1) * 8;
        else return x * 32 + grp * 8;
    };

    KvSched<A> sched;
    sched.init(a, cut, sums, lds);
    if (!kShared<A> && threadIdx.x == 0) joins[blockIdx.x].parts = 0;
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
        const int prefix = kv_prefix_of(a, r);

        // this lane's row
        const int row = row0 + min(n16, rows - 1);
        const int token = row / a.G, hq = h * a.G + row - token * a.G;
        KvRange see = kv_see(a, r, it.ctx, it.n, token, prefix, it.first_token + token);
        // the tile's keys: those that some row sees, and those that every row sees
        KvRange top = kv_first_range(a, r, it.ctx, it.n, row0 / a.G, prefix);
        KvRange bot = kv_last_range(a, r, it.ctx, it.n, (row0 + rows - 1) / a.G, prefix);
        // keys of a shared prefix before its own: all rows see them, and nobody what is between
        KvPrefix pre{0, 0, 0};
        const int32_t *p_table = nullptr;
        if constexpr (kJoined<A>) {
            pre.group = __builtin_amdgcn_readfirstlane(lds.prefix[r].group);
            pre.keys = __builtin_amdgcn_readfirstlane(lds.prefix[r].keys);
            pre.own = __builtin_amdgcn_readfirstlane(lds.prefix[r].own);
            p_table = a.p_table + (int64_t)pre.group * a.p_stride;
            see.hi = pre.own + max(see.hi, 0);
            top.hi = pre.own + max(top.hi, 0);
            bot.hi = pre.own + max(bot.hi, 0);
        }
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
                const int d = component(s);
                q[s] = FULL || d < a.D ? *(const u32x4 *)(p + 2 * d) : u32x4{0, 0, 0, 0};
            }
        }
        const float ks = F8 ? a.scale * a.k_scale[h] : a.scale;
        // scores to exponents of two: times to_exp, plus slope a key's distance; with a cap
        // to_exp leads to the exponent of its tanh
        const float slope = a.slopes ? a.slopes[hq] * kLog2e : 0.0f;
        const float cap = a.cap * kLog2e, to_exp = a.cap > 0.0f ? ks * (2.0f * kLog2e) / a.cap : ks * kLog2e;
        // shared scales, scores changed by nothing else: the factor is applied with the maximum's
        // subtraction, so it has to be positive
        const bool late = MX && a.cap == 0.0f && !a.slopes && ks != 0.0f;
        const float by = late ? fmaxf(fabsf(to_exp), 0x1p-126f) : 1.0f;
        if (MX && late && ks < 0.0f)
#pragma unroll
            for (int s = 0; s < S; ++s) q[s] ^= 0x80008000u;
        const int p_row = kShared<A> && !a.slopes ? 0 : kv_row_place(a, r, it.ctx, it.n, token, it.first_token + token) + pre.own;

        const char *kp = (const char *)a.k + bytes_of<C>((int64_t)h * a.k_head);
        const char *vp = (const char *)a.v + bytes_of<C>((int64_t)h * a.v_head);
        const int in_block = (1 << a.shift) - 1;
        const uint32_t k_lane = row_bytes<C>(n16, a.k_token, component(0));
        const uint32_t v_lane = row_bytes<C>(grp * 4, a.v_token, n16 * VW);
        const int32_t *table = kv_table(a, r);

        float m = -INFINITY, l = 0.0f;
        f32x4 o[VW];
#pragma unroll
        for (int j = 0; j < VW; ++j) o[j] = f32x4{0, 0, 0, 0};

        // Steps: keys k0 + 32 u.  A lane holds the block of one group of 16 keys, 32 steps ahead.
        const int steps = (k1 - k0 + kStepKeys - 1) / kStepKeys;
        int ids = 0;
        uint64_t at_k = 0, at_v = 0, at_kp = 0, at_vp = 0;  // shared scales: and where its 16 keys lie
        bool found = false;  // infinities or NaN among values that only some rows see
        auto in_of = [&](int key) { return kJoined<A> && key >= pre.own ? key - pre.own : key; };  // its own place
        auto fetch_ids = [&](int u) {
            const int key = k0 + (u + (lane >> 1)) * kStepKeys + (lane & 1) * 16;
            if constexpr (kJoined<A>)
                ids = key < pre.own ? p_table[min(key, pre.keys - 1) >> a.shift]
                                    : table[max(min(key, k1 - 1) - pre.own, 0) >> a.shift];
            else
                ids = table[min(key, k1 - 1) >> a.shift];
            ids = min(max(ids, 0), a.num_blocks - 1);
            if constexpr (MX) {
                const int64_t id = ids, in = in_of(key) & in_block;
                at_k = (uint64_t)kp + bytes_of<C>(id * a.k_block + in * a.k_token);
                at_v = (uint64_t)vp + bytes_of<C>(id * a.v_block + in * a.v_token);
                at_kp = (uint64_t)(a.k_power + h * a.kp_head + id * a.kp_block) + in * (a.D / kGroup);
                at_vp = (uint64_t)(a.v_power + h * a.vp_head + id * a.vp_block) + in * (a.D / kGroup);
            }
        };
        auto buffer_of = [&](uint64_t at, int u, int t) {
            const int from = 2 * (u & 31) + t;
            return Buffer(lane_value((uint32_t)at, from), lane_value((uint32_t)(at >> 32), from));
        };
        const uint32_t v_row = bytes_of<C>((uint32_t)a.v_token);
        auto place_of = [&](int64_t block_stride, int64_t token_stride, int u, int t) {
            const int id = __builtin_amdgcn_readlane(ids, 2 * (u & 31) + t);
            const int key = k0 + u * kStepKeys + t * 16;
            return (int64_t)id * block_stride + (int64_t)(in_of(key) & in_block) * token_stride;
        };
        auto base_of = [&](const char *p, int64_t block_stride, int64_t token_stride, int u, int t) {
            return p + bytes_of<C>(place_of(block_stride, token_stride, u, t));
        };
        Words<KWords> k[2];
        uint32_t k_pow[MX ? 2 : 1][MX ? KReads : 1];
        auto load_k = [&](int u) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const char *p = MX ? nullptr : base_of(kp, a.k_block, a.k_token, u, t);
                if constexpr (MX) {
                    constexpr int N = KWords / KReads;
                    const Buffer kb = buffer_of(at_k, u, t), pb = buffer_of(at_kp, u, t);
#pragma unroll
                    for (int x = 0; x < KReads; ++x) {
                        const int d = component(x * (S / KReads));
                        Words<N> y{};
                        k_pow[t][x] = 127;
                        if (FULL || d < a.D) {
                            y = kb.words<N>(k_lane, x * 64);
                            k_pow[t][x] = pb.byte(n16 * (a.D / kGroup) + component(0) / kGroup, x * (FOUR ? 4 : 2));
                        }
#pragma unroll
                        for (int j = 0; j < N; ++j) k[t].w[N * x + j] = y.w[j];
                    }
                } else if constexpr (FULL) {
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
                        const int d = component(s);
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
            // where a prefix ends within its last step
            const bool gap = kJoined<A> && key0 < pre.own && key0 + kStepKeys > pre.keys;
            const bool edge = gap || key0 < all_lo || key0 + kStepKeys > min(all_hi, k1);
            Words<VWords> v[MX ? 1 : 8];
            Words<MX ? VRaw : 1> raw[MX ? 8 : 1];
            uint32_t v_pow[MX ? 2 : 1];  // the power of row n16 % 4 of a tile's four (see `power`)
            auto load_v = [&]() {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if constexpr (MX) {
                        const Buffer vb = buffer_of(at_v, u, t), pb = buffer_of(at_vp, u, t);
                        const uint32_t row = (grp * 4 + (n16 & 3)) * (a.D / kGroup);
                        if constexpr (DP < 256) {
                            const int g = n16 * VW / kGroup;
                            v_pow[t] = 127;
                            if (FULL || g < a.D / kGroup) v_pow[t] = pb.byte(row + g, 0);
                        } else if constexpr (FULL) {  // of two groups
                            v_pow[t] = pb.half(row + (n16 >> 2) * 2, 0);
                        } else {
                            const int g = (n16 >> 2) * 2;
                            v_pow[t] = 127;
                            if (g < a.D / kGroup) v_pow[t] = pb.byte(row + g, 0);
                            if (g + 1 < a.D / kGroup) v_pow[t] |= pb.byte(row + g + 1, 0) << 8;
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            Words<VRaw> &y = raw[t * 4 + i];
                            y = Words<VRaw>{};
                            if (FULL || n16 * VW < a.D) {
                                if constexpr (FOUR && VW == 4) y.w[0] = vb.half(v_lane, i * v_row);
                                else y = vb.words<VRaw>(v_lane, i * v_row);
                            }
                        }
                        continue;
                    }
                    const char *p = base_of(vp, a.v_block, a.v_token, u, t);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const char *at = p + bytes_of<C>((int64_t)i * a.v_token);
                        if constexpr (FULL) {
                            v[t * 4 + i] = load_words<VWords>(at, v_lane);
                        } else {
                            constexpr int N = F8 ? 2 : 4, P = VWords < N ? VWords : N;
#pragma unroll
                            for (int x = 0; x < VWords; x += P) {
                                Words<P> y{};
                                if (n16 * VW + x * (F8 ? 4 : 2) < a.D) y = load_words<P>(at + 4 * x, v_lane);
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
                    if constexpr (MX) {
                        const float ps = group_scale(k_pow[t][x / (S / KReads)]);
                        kf = unpack_mx8of<T, C>(&k[t].w[x * KWords / S], ps);
                    } else if constexpr (F8) {
                        kf = u32x4{unpack_fp8<T, false>(k[t].w[2 * x]), unpack_fp8<T, true>(k[t].w[2 * x]),
                                   unpack_fp8<T, false>(k[t].w[2 * x + 1]), unpack_fp8<T, true>(k[t].w[2 * x + 1])};
                    } else {
                        kf = u32x4{k[t].w[4 * x], k[t].w[4 * x + 1], k[t].w[4 * x + 2], k[t].w[4 * x + 3]};
                    }
                    s[t] = mfma16<T>(kf, q[x], s[t]);
                }
                if constexpr (MX) __builtin_amdgcn_sched_barrier(0);  // (few registers)
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
            for (int i = 0; i < 8; ++i) e[i] = s[i >> 2][i & 3];
            if (!late)
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] *= to_exp;
            if (a.cap > 0.0f || a.slopes) {
                const float b0 = slope * (float)(key0 + grp * 4 - p_row + (key0 < pre.own ? pre.own - pre.keys : 0));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float add = __builtin_fmaf((float)((i >> 2) * 16 + (i & 3)), slope, b0);
                    e[i] = a.cap > 0.0f ? tanh_scaled(e[i], cap, add) : e[i] + add;
                }
            }
            if (gap)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    e[i] = (i >> 2) * 16 + (i & 3) < pre.keys - key0 - grp * 4 ? e[i] : -INFINITY;
            if (edge) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (MX) {  // (compared with constants: few registers)
                        const int from = see.lo - key0 - grp * 4;
                        e[i] = (uint32_t)((i >> 2) * 16 + (i & 3) - from) < (uint32_t)max(see.hi - see.lo, 0) ? e[i] : -INFINITY;
                    } else {
                        const int key = key0 + (i >> 2) * 16 + grp * 4 + (i & 3);
                        e[i] = key >= see.lo && key < see.hi ? e[i] : -INFINITY;
                    }
                }
            }
            float mt = fmaxf(fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3])), fmaxf(fmaxf(e[4], e[5]), fmaxf(e[6], e[7])));
            if constexpr (MX) mt *= by;
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
                e[i] = __builtin_amdgcn_exp2f(MX ? __builtin_fmaf(e[i], by, -mu) : e[i] - mu);
                l += e[i];
            }
            const u32x4 w = {pack2<T>(e[0], e[1]), pack2<T>(e[2], e[3]), pack2<T>(e[4], e[5]), pack2<T>(e[6], e[7])};

            if constexpr (MX) {
                // Four neighbouring lanes hold components of one group (of 256 components, of two), so
                // each has asked for the power of one of the four rows, and takes the others' from them.
                float ps[8];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int x = (int)(DP < 256 ? v_pow[t] << 23 : v_pow[t]);
                    const int y[4] = {quad_lane<0>(x), quad_lane<1>(x), quad_lane<2>(x), quad_lane<3>(x)};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        ps[4 * t + i] = DP < 256 ? __builtin_bit_cast(float, y[i])
                                                 : group_scale((uint32_t)y[i] >> (n16 & 2) * 4 & 0xff);
                }
                if (edge) {  // (see below)
                    const int from = top.lo - key0 - grp * 4;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const bool keep = (uint32_t)((i >> 2) * 16 + (i & 3) - from) < (uint32_t)max(bot.hi - top.lo, 0) &&
                                          !(gap && (i >> 2) * 16 + (i & 3) >= pre.keys - key0 - grp * 4);
                        ps[i] = keep ? ps[i] : 1.0f;
#pragma unroll
                        for (int j = 0; j < VRaw; ++j) raw[i].w[j] = keep ? raw[i].w[j] : 0;
                    }
                }
                if (edge) {
                    // what is not finite: a power from which on codes can be so, or a code of NaN
                    uint32_t odd = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        odd |= __builtin_bit_cast(uint32_t, ps[i]) > (uint32_t)(MxFormat<C>::template kMost<T> + 127) << 23;
                        if constexpr (!FOUR)
#pragma unroll
                            for (int j = 0; j < VRaw; ++j) odd |= nonfinite_mask<C>(raw[i].w[j]);
                    }
                    if (__any(odd)) {
                        found = true;
                        each<8>([&](auto row) {
                            constexpr int i = decltype(row)::value;
                            each<VW / 2>([&](auto pair) {
                                constexpr int p = decltype(pair)::value, of = FOUR ? 4 : 2, n = 32 / of;
                                uint32_t &y = raw[i].w[p / of];
                                const uint32_t bad = nonfinite_mask<T>(unpack_mx<T, C, p % of>(y, ps[i]));
                                y &= ~(((bad & ((1u << n / 2) - 1)) | (bad >> 16 & ((1u << n / 2) - 1)) << n / 2) << p % of * n);
                                __builtin_amdgcn_sched_barrier(0);  // rare: few registers, not speed
                            });
                            ps[i] = __builtin_isfinite(ps[i]) ? ps[i] : 1.0f;
                        });
                    }
                }
                // V^T by pairs of columns: row i's dword, of rows 2y and 2y + 1 the halves of one column
                each<VW / 2>([&](auto pc) {
                    constexpr int p = decltype(pc)::value;
                    auto widen = [&](int i) {
                        if constexpr (FOUR) return unpack_mx<T, C, p & 3>(raw[i].w[p >> 2], ps[i]);
                        else return unpack_mx<T, C, p & 1>(raw[i].w[p >> 1], ps[i]);
                    };
                    u32x4 x[2];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const uint32_t lo = widen(2 * y), hi = widen(2 * y + 1);
                        x[0][y] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
                        x[1][y] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
                    }
                    o[2 * p] = mfma16<T>(x[0], w, o[2 * p]);
                    o[2 * p + 1] = mfma16<T>(x[1], w, o[2 * p + 1]);
                    __builtin_amdgcn_sched_barrier(0);  // (few registers)
                });
            }
            if constexpr (!MX) {
                if (edge) {
                    // a weight of zero does not silence an infinity or a NaN: values that no row of
                    // the tile sees become zero, and those that some see are added after the last
                    // step, to these rows alone
                    uint32_t odd = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int key = key0 + (i >> 2) * 16 + grp * 4 + (i & 3);
                        const bool keep = key >= top.lo && key < bot.hi && !(gap && key >= pre.keys);
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
        }

        if (found) {
            // An infinity stays one here whatever its weight, and a NaN.  (In steps that all rows
            // see it goes through the product, where a weight that rounds to zero makes it NaN:
            // looking at every value of every step would cost more than it is worth.)
            for (int key = k0; key < k1; ++key) {
                const int step = k0 + ((key - k0) & ~(kStepKeys - 1));
                const bool gap = kJoined<A> && step < pre.own && step + kStepKeys > pre.keys;
                if (!gap && step >= all_lo && step + kStepKeys <= min(all_hi, k1)) continue;  // not zeroed
                if (gap && key >= pre.keys) continue;
                const bool seen = key >= see.lo && key < see.hi;
                const int place = in_of(key);
                const int id = min(max((kJoined<A> && key < pre.own ? p_table : table)[place >> a.shift], 0), a.num_blocks - 1);
                const char *at = vp + bytes_of<C>(id * a.v_block + (int64_t)(place & in_block) * a.v_token);
                const uint8_t *pw = nullptr;
                if constexpr (MX) {
                    pw = a.v_power + id * a.vp_block + (place & in_block) * (a.D / kGroup) + h * a.vp_head;
                    if (!mx_row_nonfinite<T, C>(at, pw, a.D)) continue;
                } else {
                    if (!row_nonfinite<C>(at, bytes_of<C>(a.D))) continue;
                }
                int D = a.D;
                asm volatile("" : "+s"(D));  // compared with anew: 64 addresses would not fit
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < VW; ++j) {
                        const int d = VW * (grp * 4 + c) + j;
                        float y;
                        if constexpr (MX) y = mx_value_at<T, C>(at, pw, FULL ? d : min(d, D - 1));
                        else y = value_at<C>(at, FULL ? d : min(d, D - 1));
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
            const bool raw = kShared<A> || !whole;  // (behind prefixes rows are joined afterwards)
            const int64_t row_at = t * a.Hq + hq, raw_at = kShared<A> && whole ? row_at : at;
            const KvRaw<A> to = kShared<A> && whole ? kv_raw(a, r) : KvRaw<A>{part_o, part_ml};
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int j = 0; j < VW; j += 4) {
                    const int d = VW * (grp * 4 + c) + j;
                    const f32x4 x = {o[j][c], o[j + 1][c], o[j + 2][c], o[j + 3][c]};
                    if (raw)
                        *(f32x4 *)&to.o[raw_at * DP + d] = x;
                    else if (FULL || d < a.D)
                        *(uint2 *)(out + d) = l == 0.0f ? make_uint2(0, 0)
                                                        : make_uint2(pack2<T>(x[0] * inv, x[1] * inv),
                                                                     pack2<T>(x[2] * inv, x[3] * inv));
                }
            if (grp == 0) {
                if (raw) to.ml[raw_at] = make_float2(m, l);
                else if (a.lse) a.lse[row_at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
            }
        }
        if (!kShared<A> && !whole && it.step == 0 && lane == 0) {
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

template <class T, class A>
void launch_kv_decode(const A &a, const KvCut &c, const uint64_t *sums, int cache_dtype, int DP,
                      bool pad, float *o, float2 *ml, KvJoin *joins, hipStream_t st)
{
    auto go = [&](auto kernel) { kernel<<<c.groups, 64, 0, st>>>(a, c, sums, pad, o, ml, joins); };
    auto of = [&](auto cache) {
        using C = decltype(cache);
        using K = KvKernelArgs<A, C>;
        const bool full = a.D == DP;
        if (DP == 64) full ? go(kv_decode_kernel<T, C, 64, true, K>) : go(kv_decode_kernel<T, C, 64, false, K>);
        else if (DP == 128) full ? go(kv_decode_kernel<T, C, 128, true, K>) : go(kv_decode_kernel<T, C, 128, false, K>);
        else full ? go(kv_decode_kernel<T, C, 256, true, K>) : go(kv_decode_kernel<T, C, 256, false, K>);
    };
    if (cache_dtype == DRO_FP8_E4M3) of(fp8{});
    else if (cache_dtype == DRO_MXFP4) of(mx4{});
    else if (cache_dtype == DRO_MXFP8) of(mx8{});
    else of(T{});
}

}  // namespace dro
