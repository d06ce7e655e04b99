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
// is theirs), and rescaling a row is a lane's own product.  Rows of both tiles lie in LDS
// in pieces of 16 bytes whose order is turned from row to row, so that the reads, along
// the rows and (transposed) across them, meet all banks.  16-bit caches go from memory to
// LDS directly, the next tile while one is worked on.
//
// A prompt of 8192 tokens, 64 heads on 8 of 128 components: 1.06 to 1.15 ms from card to card, 0.96 to
// 1.04 PFLOP/s, the matrix units busy 52 % of the cycles; four chunks of 512 over 4000 to 8192, 32 heads
// on 8: 234 to 251 us, 880 to 940 TFLOP/s; with lengths that fill the compute units less evenly 270 us,
// 830 TFLOP/s.
#pragma once

#include <type_traits>

#include "kv_math.h"
#include "kv_sched.h"

namespace dro {

// With 256 components the sums of 32 rows are half a wave's registers already, so two waves
// share rows there: both compute the scores, each the sums of half the components.  (Whole
// rows a wave went through scratch memory: 284 us for a mixed call of 40 requests, 8 heads on
// 4, against 141 side by side then.)
constexpr int prefill_split(int DP) { return DP == 256 ? 2 : 1; }
constexpr int prefill_rows(int DP) { return 128 / prefill_split(DP); }

constexpr int kAheadOf = 4;  // products: 128 cycles, a read of LDS

// masks of the scheduler's groups
constexpr int kMfma = 0x8, kDsRead = 0x100;

constexpr int prefill_keys(int DP) { return 8192 / DP; }  // 16 KB of keys, as much of values
constexpr int prefill_groups(int) { return 2; }              // workgroups a compute unit

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

// The larger, a NaN aside.  (fmaxf first quiets operands that a matrix product made, an
// operation each; the median with infinity does not.)
__device__ __forceinline__ float max_raw(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, INFINITY); }
__device__ __forceinline__ float max_halves(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return max_raw(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
template <int N> __device__ __forceinline__ float max_of(const f32x16 (&x)[N])
{
    // four chains of steps that take two values each
    float m[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        m[c] = x[0][c];
#pragma unroll
        for (int i = 4; i < N * 16; i += 8) {
            m[c] = max_raw(m[c], x[i / 16][i % 16 + c]);
            if (i + 4 < N * 16) m[c] = max_raw(m[c], x[(i + 4) / 16][(i + 4) % 16 + c]);
        }
    }
    return max_raw(max_raw(max_raw(m[0], m[1]), m[2]), m[3]);
}

__device__ __forceinline__ float sum_halves(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// Where piece c (8 components) of row r lies within the row: a read of one piece of 16
// rows, and one of 4 pieces of 4 rows, touch 16 different sixteenths of the banks.
template <int DP> __device__ __forceinline__ int key_turn(int r) { return DP == 64 ? (r >> 1) & 7 : r & 15; }
template <int DP> __device__ __forceinline__ int value_turn(int r)
{
    return DP == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2;
}

// (the constant address space: read through the scalar cache, so that a wait for a block's
// number is no wait for the tile that is on its way)
typedef const __attribute__((address_space(4))) int32_t *ScalarInts;
typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

template <class T, class C, int DP, bool MODS, bool FULL, class A>
__global__ __launch_bounds__(256, prefill_groups(DP)) void kv_prefill_kernel(
    const A a, const KvCut cut, const KvTiles tiles, bool pad, float *part_o, float2 *part_ml,
    KvJoin *joins)
{
    constexpr bool F8 = __is_same(C, fp8), MX = kMx<C>;
    constexpr bool REG = F8 || MX;  // widened on the way to LDS, through registers
    constexpr int GW = __is_same(C, mx4) ? 4 : 8;  // dwords of a group's codes
    constexpr bool LEAN = MODS || REG || DP == 256;  // places in LDS and memory are not kept over the steps
    constexpr int KT = prefill_keys(DP);
    constexpr int S = DP / 16;           // steps of 16 components of a score
    // keys whose scores are in registers at once: 128 beside the changes of the scores spill
    constexpr int SK = MODS && KT > 64 ? 64 : KT;
    constexpr int NT = SK / 32;          // their tiles
    constexpr int DS = prefill_split(DP);
    constexpr int ND = DP / 32 / DS;     // component tiles of a wave
    constexpr int Rows = prefill_rows(DP);
    constexpr int Row = DP * 2;          // bytes of a row in LDS
    constexpr int NC = DP / 8;           // pieces of a row
    constexpr int NG = KT / 16;          // groups of 16 keys (each within one block)
    constexpr int UP = 2 * NG / 4;       // groups of keys or of values that a wave stages
    constexpr int IP = DP / 32;          // its loads for one: 64 pieces each
    constexpr int RP = 64 / NC;          // rows of a load
    constexpr int Tile = KT * Row;
    // two tiles of keys and of values, by name: the compiler then knows that reading one waits
    // for no load into another
    __shared__ __align__(16) char k_even[Tile], k_odd[Tile], v_even[Tile], v_odd[Tile];
    __shared__ int found;  // infinities or NaN among values that only some rows see

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n32 = lane & 31, half = lane >> 5;
    const int rw = wave % (4 / DS) * 32, dt0 = wave / (4 / DS) * ND;  // rows and component tiles from there on
    if (!FULL) {  // pieces beyond the rows' ends are never written
        for (int i = threadIdx.x; i < Tile / 16; i += 256) {
            const u32x4 zero = {0, 0, 0, 0};
            ((u32x4 *)k_even)[i] = zero;
            ((u32x4 *)k_odd)[i] = zero;
            ((u32x4 *)v_even)[i] = zero;
            ((u32x4 *)v_odd)[i] = zero;
        }
        __syncthreads();
    }
    // Workgroups b, b + 8, .. run on one die.  It gets whole heads where their number allows, one
    // after the other, since the tiles of a head share its keys in the L2; else the heads take
    // turns, which with 1, 2 or 4 gives a die one head as well.
    const KvTileList list = *tiles.list;
    const uint32_t all1 = list.all, all = all1 * a.H;  // chunks of a head, and in all
    const bool by_head = a.H % kDies == 0;
    if (pad && gridDim.x <= all) zero_rows<T>(a, blockIdx.x, gridDim.x);
    else if (pad && blockIdx.x >= all) zero_rows<T>(a, blockIdx.x - all, gridDim.x - all);
    if (!kShared<A> && blockIdx.x == 0)  // places of no tile
        for (int i = list.parts * a.H + threadIdx.x; i < 2 * cut.groups; i += 256) joins[i].parts = 0;
    for (uint32_t unit = blockIdx.x; unit < all; unit += gridDim.x) {
        const uint32_t nth = unit / kDies, per = by_head ? all1 : (uint32_t)a.H, quot = (by_head ? nth : unit) / per,
                       rest = (by_head ? nth : unit) - quot * per;
        const int h = by_head ? unit % kDies * (a.H / kDies) + quot : rest;
        const uint32_t u1 = by_head ? rest : quot;
        const KvTile rt = tiles.tiles[__builtin_amdgcn_readfirstlane(kv_find(tiles.sums, list.count, u1))];
        const int r = rt.r, tile = rt.tile;
        // steps of its own
        const int chunk = (int)(u1 - rt.before), each_steps = (rt.steps + rt.chunks - 1) / rt.chunks;
        const int step0 = chunk * each_steps, go = min(each_steps, max(rt.steps - step0, 0));
        const int place = rt.part + list.parts * h + chunk;
        const bool whole = rt.chunks == 1;
        const int first_token = rt.first_token;
        const int row0 = tile * Rows;
        const int rows = min(rt.n * a.G - row0, Rows);
        const int prefix = kv_prefix_of(a, r);
        const KvRange top = kv_first_range(a, r, rt.ctx, rt.n, row0 / a.G, prefix);
        const KvRange bot = kv_last_range(a, r, rt.ctx, rt.n, (row0 + rows - 1) / a.G, prefix);
        const int base = top.lo & ~31;
        const int k0 = min(base + step0 * KT, bot.hi), k1 = min(base + (step0 + go) * KT, bot.hi);
        const int steps = (k1 - k0 + KT - 1) / KT;

        // this wave's rows, and this lane's
        const int wrow = min(rw, rows - 1), wlast = min(rw + 31, rows - 1);
        const KvRange wtop = kv_first_range(a, r, rt.ctx, rt.n, (row0 + wrow) / a.G, prefix);
        const KvRange wbot = kv_last_range(a, r, rt.ctx, rt.n, (row0 + wlast) / a.G, prefix);
        const bool idle = rw >= rows;
        const int row = row0 + min(rw + n32, rows - 1);
        const int token = row / a.G, hq = h * a.G + row - token * a.G;
        const KvRange see = kv_see(a, r, rt.ctx, rt.n, token, prefix, first_token + token);
        const int p_row = kShared<A> && (!MODS || !a.slopes) ? 0 : kv_row_place(a, r, rt.ctx, rt.n, token, first_token + token);

        u32x4 q[S];
        {
            const char *p = (const char *)a.q + 2 * ((int64_t)(first_token + token) * a.q_token + hq * a.q_head);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int d = s * 16 + half * 8;
                q[s] = FULL || d < a.D ? *(const u32x4 *)(p + 2 * d) : u32x4{0, 0, 0, 0};
            }
        }
        const float ks = F8 ? a.scale * a.k_scale[h] : a.scale;
        // scores to exponents of two: times to_exp, plus slope a key's distance; with a cap
        // to_exp leads to the exponent of its tanh
        const float slope = MODS && a.slopes ? a.slopes[hq] * kLog2e : 0.0f;
        const float cap = a.cap * kLog2e;
        float to_exp = MODS && a.cap > 0.0f ? ks * (2.0f * kLog2e) / a.cap : ks * kLog2e;
        if constexpr (!MODS) {  // scale > 0 from here on, so the largest score has the largest weight
            to_exp = fmaxf(fabsf(ks) * kLog2e, 0x1p-126f);  // (a hidden key's -infinity times zero would be NaN)
            if (ks < 0.0f)
#pragma unroll
                for (int s = 0; s < S; ++s) q[s] ^= 0x80008000u;
        }

        // Staging: piece x = lane of load i of group j goes to place 1024 i + 16 lane of the
        // group's rows, so the lane picks the piece of its row that belongs there.
        const ScalarInts table = (ScalarInts)kv_table(a, r);
        const int in_block = (1 << a.shift) - 1;
        int ids[UP];
        auto load_ids = [&](int u) {
#pragma unroll
            for (int j = 0; j < UP; ++j)
                ids[j] = table[min(k0 + u * KT + (wave + 4 * j) % NG * 16, k1 - 1) >> a.shift];
        };
        Words<2> reg[F8 ? UP * IP : 1];
        auto load = [&](auto odd_tile, int u) {
            int lane = threadIdx.x & 63;
            if constexpr (LEAN) asm volatile("" : "+v"(lane));  // (see `fresh`)
#pragma unroll
            for (int j = 0; j < UP; ++j) {
                const bool vals = (wave + 4 * j) / NG;
                const int group = (wave + 4 * j) % NG;
                const int64_t s_token = vals ? a.v_token : a.k_token;
                const int64_t id = min(max(ids[j], 0), a.num_blocks - 1);
                const int in = (k0 + u * KT + group * 16) & in_block;
                const char *base = (vals ? (const char *)a.v + bytes_of<C>(h * a.v_head) : (const char *)a.k + bytes_of<C>(h * a.k_head)) +
                                   bytes_of<C>(id * (vals ? a.v_block : a.k_block) + in * s_token);
#pragma unroll
                for (int i = 0; i < IP; ++i) {
                    const int rr = i * RP + lane / NC;
                    const int c = (lane % NC) ^ (vals ? value_turn<DP>(rr) : key_turn<DP>(rr));
                    const uint32_t off = row_bytes<C>(lane / NC, s_token, c * 8);
                    const char *p = base + bytes_of<C>(i * RP * s_token);
                    if (FULL || c * 8 < a.D) {
                        if constexpr (F8)
                            reg[j * IP + i] = load_words<2>(p, off);
                        else if (vals)
                            __builtin_amdgcn_global_load_lds(
                                (GlobalPtr)(p + off),
                                (LdsPtr)((decltype(odd_tile)::value ? v_odd : v_even) + group * 16 * Row + i * 1024), 16, 0, 0);
                        else
                            __builtin_amdgcn_global_load_lds(
                                (GlobalPtr)(p + off),
                                (LdsPtr)((decltype(odd_tile)::value ? k_odd : k_even) + group * 16 * Row + i * 1024), 16, 0, 0);
                    }
                }
            }
        };
        auto store = [&](auto odd_tile) {  // fp8: widened on the way
            if constexpr (F8) {
#pragma unroll
                for (int j = 0; j < UP; ++j) {
                    const bool vals = (wave + 4 * j) / NG;
                    const int group = (wave + 4 * j) % NG;
#pragma unroll
                    for (int i = 0; i < IP; ++i) {
                        const Words<2> &x = reg[j * IP + i];
                        const int rr = i * RP + lane / NC;
                        const int c = (lane % NC) ^ (vals ? value_turn<DP>(rr) : key_turn<DP>(rr));
                        if (FULL || c * 8 < a.D)
                            *(u32x4 *)((vals ? (decltype(odd_tile)::value ? v_odd : v_even)
                                              : (decltype(odd_tile)::value ? k_odd : k_even)) +
                                        group * 16 * Row + i * 1024 + lane * 16) =
                                u32x4{unpack_fp8<T, false>(x.w[0]), unpack_fp8<T, true>(x.w[0]),
                                      unpack_fp8<T, false>(x.w[1]), unpack_fp8<T, true>(x.w[1])};
                    }
                }
            }
        };
        // Shared scales: a tile's keys have 256 groups, so a lane stages one, of the keys and of the
        // values, 16 bytes of 4-bit codes (32 of 8-bit ones) and a power each; lanes next to one another
        // take rows next to one another.  The values' rows are turned by fours, so there a lane writes
        // its four pieces in an order by its row.  Bank conflicts are a seventh of LDS's busy cycles
        // (6.9 of 48 million in 4 bits); rows turned by their groups leave that count and the time as
        // they are.  Four chunks of 512 tokens over 4000 to 8192 keys, 32 heads on 8, of the less even
        // lengths above, one after the other on one card: 284 us in 4 bits, 303 in 8, fp8 291, 16 bits
        // 270 (which no register passes on the way to LDS).
        const int n16 = lane & 15, mx_g = DP == 64 ? lane >> 4 & 1 : DP == 128 ? lane >> 4 : (lane >> 4) + 4 * (wave & 1);
        auto mx_group = [&](int j) { return DP == 64 ? wave * 2 + j : DP == 128 ? wave : wave >> 1; };  // of 16 keys
        Words<MX ? GW : 1> mx_reg[2];
        uint32_t mx_power[2];
        constexpr int MG = MX && DP == 64 ? 2 : 1;  // groups of keys of a wave
        auto mx_ids = [&](int u) {
#pragma unroll
            for (int j = 0; j < MG; ++j) ids[j] = table[min(k0 + u * KT + mx_group(j) * 16, k1 - 1) >> a.shift];
        };
        auto mx_load = [&](int u) {
            if constexpr (MX) {
                const char *base[MG][2];
                const uint8_t *pw[MG][2];
#pragma unroll
                for (int j = 0; j < MG; ++j) {
                    const int64_t id = min(max(ids[j], 0), a.num_blocks - 1);
                    const int in = (k0 + u * KT + mx_group(j) * 16) & in_block;
                    base[j][0] = (const char *)a.k + bytes_of<C>(h * a.k_head + id * a.k_block + in * a.k_token);
                    base[j][1] = (const char *)a.v + bytes_of<C>(h * a.v_head + id * a.v_block + in * a.v_token);
                    pw[j][0] = a.k_power + h * a.kp_head + id * a.kp_block + in * (a.D / kGroup);
                    pw[j][1] = a.v_power + h * a.vp_head + id * a.vp_block + in * (a.D / kGroup);
                }
                const bool second = MG == 2 && lane >= 32;
#pragma unroll
                for (int v = 0; v < 2; ++v)
                    if (FULL || mx_g * kGroup < a.D) {
                        const uint32_t off = row_bytes<C>(n16, v ? a.v_token : a.k_token, mx_g * kGroup);
                        mx_reg[v] = load_words<GW>(second ? base[MG - 1][v] : base[0][v], off);
                        mx_power[v] = (second ? pw[MG - 1][v] : pw[0][v])[(uint32_t)(n16 * (a.D / kGroup) + mx_g)];
                    }
            }
        };
        auto mx_store = [&](auto odd_tile) {
            if constexpr (MX) {
                if (!FULL && mx_g * kGroup >= a.D) return;
                const int row = mx_group(MG == 2 ? lane >> 5 : 0) * 16 + n16, rot = n16 >> 2;
                const float ks = group_scale(mx_power[0]), vs = group_scale(mx_power[1]);
                char *kt = (decltype(odd_tile)::value ? k_odd : k_even) + row * Row;
                char *vt = (decltype(odd_tile)::value ? v_odd : v_even) + row * Row;
                constexpr int N = GW / 4;
                auto &y = mx_reg[1].w;
#pragma unroll
                for (int x = 0; x < 2 * N; ++x) {  // piece i becomes piece i ^ rot
                    const int i = x / N * 2 * N + x % N, lo = y[i], hi = y[i + N];
                    y[i] = rot & 1 ? hi : lo;
                    y[i + N] = rot & 1 ? lo : hi;
                }
#pragma unroll
                for (int i = 0; i < 2 * N; ++i) {
                    const int lo = y[i], hi = y[i + 2 * N];
                    y[i] = rot & 2 ? hi : lo;
                    y[i + 2 * N] = rot & 2 ? lo : hi;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    *(u32x4 *)(kt + ((4 * mx_g + i) ^ key_turn<DP>(row)) * 16) = unpack_mx8of<T, C>(&mx_reg[0].w[i * N], ks);
                    *(u32x4 *)(vt + ((4 * mx_g + (i ^ rot)) ^ value_turn<DP>(row)) * 16) = unpack_mx8of<T, C>(&y[i * N], vs);
                }
            }
        };
        // Where a lane reads, for piece 0 of the keys and of the values; the others follow by an
        // exclusive or and an offset.  Where registers are short (LEAN) each step computes them
        // anew: kept over the steps they take the registers of the queries, which then come back
        // from memory behind the tile on its way.
        auto key_place = [&](int lane) {
            return (uint32_t)((lane & 31) * Row + ((lane >> 5) ^ key_turn<DP>(lane & 31)) * 16);
        };
        auto value_place = [&](int lane) {
            const int i = lane & 15, rr = (lane >> 5) * 4 + (i >> 2), d = dt0 * 32 + (lane & 16) + (i & 3) * 4;
            return (uint32_t)(rr * Row + ((d >> 3) ^ value_turn<DP>(rr)) * 16 + (d & 4) * 2);
        };
        // 8 weights' worth of component n32 of tile j: keys 16 x + 4 half + {0 .. 3, 8 .. 11}
        auto value_frag = [&](const char *sv, uint32_t at, int x, int j) {
            u32x4 y;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const auto z = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) Vec<short, 4> *)(sv + (at ^ (j * 64)) + (x * 16 + e * 8) * Row));
                const Vec<uint32_t, 2> w = __builtin_bit_cast(Vec<uint32_t, 2>, z);
                y[2 * e] = w[0];
                y[2 * e + 1] = w[1];
            }
            return y;
        };

        float m = -INFINITY, l = 0.0f;
        f32x16 o[ND];
#pragma unroll
        for (int j = 0; j < ND; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.0f;

        constexpr std::integral_constant<bool, false> even{};
        constexpr std::integral_constant<bool, true> odd{};
        __syncthreads();  // the last item's tiles are read
        if (threadIdx.x == 0) found = 0;
        if (steps) {
            if constexpr (MX) {
                mx_ids(0);
                mx_load(0);
                mx_ids(1);
                mx_store(even);
            } else {
                load_ids(0);
                load(even, 0);
                load_ids(1);
                store(even);
            }
        }
        auto step = [&](auto odd_tile, int u) {
            constexpr std::integral_constant<bool, !decltype(odd_tile)::value> next{};
            const int tile0 = k0 + u * KT;
            char *sk = decltype(odd_tile)::value ? k_odd : k_even, *sv = decltype(odd_tile)::value ? v_odd : v_even;
            __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's part of tile u has landed
            __syncthreads();                     // everybody's has, and tile u - 1 is read
            if (u + 1 < steps) {
                if constexpr (MX) {
                    mx_load(u + 1);
                    mx_ids(u + 2);
                } else {
                    load(next, u + 1);
                    load_ids(u + 2);
                }
            }
            // A weight of zero does not silence an infinity or a NaN.  Where some row of the
            // workgroup does not see some key of the tile, such values become zero in LDS and are
            // added after the last step, to the rows that see them.
            const bool mixed = tile0 < bot.lo || tile0 + KT > top.hi;
            if (mixed) {
                bool bad = false;
                for (int i = threadIdx.x; i < Tile / 16; i += 256) {
                    u32x4 &y = ((u32x4 *)sv)[i];
                    u32x4 mask;
#pragma unroll
                    for (int c = 0; c < 4; ++c) mask[c] = nonfinite_mask<T>(y[c]);
                    if (mask[0] | mask[1] | mask[2] | mask[3]) {
                        y &= ~mask;
                        const int key = tile0 + i / NC;
                        bad |= key >= top.lo && key < k1;  // (what no row sees may hold anything)
                    }
                }
                if (bad) found = 1;
                __syncthreads();
            }
#pragma unroll
            for (int sub = 0; sub < KT; sub += SK) {
                const int key0 = tile0 + sub;
                const bool none = idle || key0 >= wbot.hi || key0 + SK <= wtop.lo;
                if (none) continue;
                // pieces of the keys and of the values are read kAheadOf products before their
                // use, the first of the values before the softmax
                int fresh = lane;
                if constexpr (LEAN) asm volatile("" : "+v"(fresh));
                const uint32_t k_at = key_place(fresh), v_at = value_place(fresh);
                auto key_frag = [&](int f) {
                    return *(const u32x4 *)&sk[(k_at ^ (f % S * 32)) + (sub + f / S * 32) * Row];
                };
                __builtin_amdgcn_s_setprio(1);
                f32x16 s[NT];
                u32x4 kf[kAheadOf], vf[kAheadOf];
#pragma unroll
                for (int f = 0; f < kAheadOf; ++f) kf[f] = key_frag(f);
#pragma unroll
                for (int f = 0; f < NT * S; ++f) {
                    if (f % S == 0)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[f / S][i] = 0.0f;
                    s[f / S] = mfma32<T>(kf[f % kAheadOf], q[f % S], s[f / S]);
                    if (f + kAheadOf < NT * S) kf[f % kAheadOf] = key_frag(f + kAheadOf);
                }
#pragma unroll
                for (int f = 0; f < kAheadOf; ++f) vf[f] = value_frag(sv + sub * Row, v_at, f / ND, f % ND);
                __builtin_amdgcn_sched_group_barrier(kDsRead, kAheadOf, 0);
#pragma unroll
                for (int f = 0; f < NT * S - kAheadOf; ++f) {
                    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
                }
#pragma unroll
                for (int f = 0; f < kAheadOf; ++f) {
                    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
                }
                __builtin_amdgcn_s_setprio(0);
                const bool edge = key0 < wbot.lo || key0 + SK > min(wtop.hi, k1);
                const int lane0 = key0 + half * 4, from = see.lo - lane0, dist = lane0 - p_row;
                const uint32_t seen = (uint32_t)max(see.hi - see.lo, 0);
                if constexpr (MODS) {
                    // (groups of four keys, so that few constants take registers)
                    const float b0 = slope * (float)dist, by4[4] = {0.0f, slope, 2.0f * slope, 3.0f * slope};
                    auto add = [&](int t, int i) {
                        const float b = __builtin_fmaf((float)(t * 4 + (i >> 2)), 8.0f * slope, b0);
                        return i & 3 ? b + by4[i & 3] : b;
                    };
                    if (a.cap > 0.0f) {
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                s[t][i] = tanh_scaled(s[t][i] * to_exp, cap, add(t, i));
                                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                            }
                    } else {
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                s[t][i] = __builtin_fmaf(s[t][i], to_exp, add(t, i));
                                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                            }
                    }
                }
                if (edge) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int c = t * 32 + (i >> 2) * 8 + (i & 3);
                            float x = (uint32_t)(c - from) < seen ? s[t][i] : -INFINITY;
                            asm volatile("" : "+v"(x));  // keeps the branch: most tiles have no edge
                            s[t][i] = x;
                        }
                }
                float mt = max_of(s);
                const float by = MODS ? 1.0f : to_exp;
                mt *= by;
                mt = max_halves(mt);
                if (__any(has_to_raise<T>(mt, m))) {
                    const float to = fmaxf(m, mt - kUnit<T>);
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
                        s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], by, -mu));
                        s[t][i + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i + 1], by, -mu));
                        l += s[t][i] + s[t][i + 1];
                        w[2 * t + (i >> 3)][(i >> 1) & 3] = pack2<T>(s[t][i], s[t][i + 1]);
                    }
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int f = 0; f < NT * 2 * ND; ++f) {
                    o[f % ND] = mfma32<T>(vf[f % kAheadOf], w[f / ND], o[f % ND]);
                    const int g = f + kAheadOf;
                    if (g < NT * 2 * ND) vf[f % kAheadOf] = value_frag(sv + sub * Row, v_at, g / ND, g % ND);
                }
#pragma unroll
                for (int f = 0; f < NT * 2 * ND - kAheadOf; ++f) {
                    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
                }
                __builtin_amdgcn_sched_group_barrier(kMfma, kAheadOf, 0);
                __builtin_amdgcn_s_setprio(0);
            }
            if (u + 1 < steps) {
                if constexpr (MX) mx_store(next);
                else store(next);
            }
        };
        for (int u = 0; u < steps; u += 2) {
            step(even, u);
            if (u + 1 < steps) step(odd, u + 1);
        }

        if (steps && found && !idle) {  // (the steps' barriers order `found`)
            // An infinity stays one here whatever its weight, and a NaN.  (In steps that all rows
            // see it goes through the product, where a weight that rounds to zero makes it NaN:
            // looking at every value of every step would cost more than it is worth.)
            for (int key = k0; key < k1; ++key) {
                const int at_step = (key - k0) & ~(KT - 1);
                if (k0 + at_step >= bot.lo && k0 + at_step + KT <= top.hi) continue;  // not zeroed
                const bool seen = key >= see.lo && key < see.hi;
                const int id = min(max(table[key >> a.shift], 0), a.num_blocks - 1);
                const char *at = (const char *)a.v + bytes_of<C>(id * a.v_block + (int64_t)(key & in_block) * a.v_token +
                                                                 (int64_t)h * a.v_head);
                const uint8_t *pw = nullptr;
                if constexpr (MX) {
                    pw = a.v_power + id * a.vp_block + (key & in_block) * (a.D / kGroup) + h * a.vp_head;
                    if (!mx_row_nonfinite<T, C>(at, pw, a.D)) continue;
                } else {
                    if (!row_nonfinite<C>(at, bytes_of<C>(a.D))) continue;
                }
                int D = a.D;
                asm volatile("" : "+s"(D));  // compared with anew: 64 addresses would not fit
#pragma unroll
                for (int j = 0; j < ND; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int d = (dt0 + j) * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
                        float y;
                        if constexpr (MX) y = mx_value_at<T, C>(at, pw, FULL ? d : min(d, D - 1));
                        else y = value_at<C>(at, FULL ? d : min(d, D - 1));
                        if (seen && !__builtin_isfinite(y)) o[j][i] += y;
                        __builtin_amdgcn_sched_barrier(0);  // rare: few registers, not speed
                    }
            }
        }
        l = sum_halves(l);
        if (rw + n32 < rows) {
            const int64_t t = first_token + token;
            const int64_t at = (int64_t)place * Rows + rw + n32;
            const float inv = l == 0.0f ? 0.0f : (F8 ? a.v_scale[h] : 1.0f) / l;
            T *out = (T *)a.out + t * a.out_token + hq * a.out_head;
            const bool raw = kShared<A> || !whole;  // (behind prefixes rows are joined afterwards)
            const int64_t row_at = t * a.Hq + hq, raw_at = kShared<A> && whole ? row_at : at;
            const KvRaw<A> to = kShared<A> && whole ? kv_raw(a, r) : KvRaw<A>{part_o, part_ml};
#pragma unroll
            for (int j = 0; j < ND; ++j)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int d = (dt0 + j) * 32 + (i >> 2) * 8 + half * 4;
                    if (raw)
                        *(f32x4 *)&to.o[raw_at * DP + d] = f32x4{o[j][i], o[j][i + 1], o[j][i + 2], o[j][i + 3]};
                    else if (FULL || d < a.D)
                        *(uint2 *)(out + d) = l == 0.0f ? make_uint2(0, 0)
                                                        : make_uint2(pack2<T>(o[j][i] * inv, o[j][i + 1] * inv),
                                                                     pack2<T>(o[j][i + 2] * inv, o[j][i + 3] * inv));
                }
            if (half == 0 && dt0 == 0) {
                if (raw) to.ml[raw_at] = make_float2(m, l);
                else if (a.lse) a.lse[row_at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
            }
        }
        if (!kShared<A> && !whole && threadIdx.x == 0) {
            KvJoin &j = joins[place];
            j.parts = chunk ? 0 : rt.chunks;
            j.first_token = first_token;
            j.row0 = row0;
            j.rows = rows;
            j.head = h;
            j.first = place;
            j.next = place + 1;
            j.stride = 1;
        }
    }
}

template <class T, class A>
void launch_kv_prefill(const A &a, const KvCut &c, const KvTiles &t, unsigned grid, int cache_dtype, int DP, bool pad,
                       float *o, float2 *ml, KvJoin *joins, hipStream_t st)
{
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(a, c, t, pad, o, ml, joins); };
    // A head dimension between the padded ones takes the kernel of all score changes as well.  Beyond 64
    // components its instances keep 76 to 97 registers in scratch memory, over shared scales 105 to 123;
    // those of all 128 with score changes 14 (fp8 49, MXFP4 50, MXFP8 119), of all 256 none (4, 25, 88), and
    // of MXFP8 without them 43 and 53: read back in the steps, behind the next tile's loads.  (Behind
    // shared prefixes a few more: 46 and 58.  A cap takes the four chunks above from 270 us to 370, fp8
    // from 291 to 414, MXFP4 from 284 to 445, MXFP8 from 303 to 536.)
    auto of = [&](auto cache, auto dim) {
        using C = decltype(cache);
        using K = KvKernelArgs<A, C>;
        constexpr int P = decltype(dim)::value;
        if (a.D != P) go(kv_prefill_kernel<T, C, P, true, false, K>);
        else if (a.cap > 0.0f || a.slopes || a.scale == 0.0f) go(kv_prefill_kernel<T, C, P, true, true, K>);
        else go(kv_prefill_kernel<T, C, P, false, true, K>);
    };
    auto with = [&](auto cache) {
        if (DP == 64) of(cache, std::integral_constant<int, 64>{});
        else if (DP == 128) of(cache, std::integral_constant<int, 128>{});
        else of(cache, std::integral_constant<int, 256>{});
    };
    if (cache_dtype == DRO_FP8_E4M3) with(fp8{});
    else if (cache_dtype == DRO_MXFP4) with(mx4{});
    else if (cache_dtype == DRO_MXFP8) with(mx8{});
    else with(T{});
}

}  // namespace dro
