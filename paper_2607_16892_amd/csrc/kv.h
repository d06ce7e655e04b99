// Launchers of the paged-cache kernels (block tables, store, load, attention).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dro {

// ---- block tables -----------------------------------------------------------
struct KvTablesArgs {
    int R, shift, num_blocks, W;  // block = 1 << shift tokens; W = table columns
    int64_t table_stride;
    int32_t *table;
    int32_t *free_list;
    const int32_t *held;
    const int32_t *free_count;
    const int32_t *len, *add, *reserve;  // reserve may be null
    int T;
    int32_t *held_out, *free_out, *context, *start;
    int64_t *slot;
    int32_t *pos;
    uint8_t *granted;
    int4 *rows;     // scratch [R]: what each request takes and gives (see kv_cache.hip)
    uint32_t *backs;  // scratch [R]: blocks given back before each request
    int32_t *tops;  // scratch [2]: blocks free before and after the ended requests' ones
};
hipError_t launch_kv_tables(const KvTablesArgs &a, hipStream_t st);

// ---- store and load --------------------------------------------------------------------
struct KvStoreArgs {
    int T, H, D;
    int shift;
    int64_t slots;                // num_blocks << shift
    void *x[2];                   // keys, values
    int64_t x_token[2], x_head[2];
    void *c[2];                   // the cache's
    int64_t c_block[2], c_token[2], c_head[2];
    const float *scale[2];        // fp8 caches
    uint8_t *power[2];            // caches in shared scales; D / 32 from token to token
    int64_t p_block[2], p_head[2];
    const int64_t *slot;
};
hipError_t launch_kv_store(const KvStoreArgs &a, int dtype, int cache_dtype, hipStream_t st);
// the other way: x written, the cache read
hipError_t launch_kv_load(const KvStoreArgs &a, int dtype, int cache_dtype, hipStream_t st);

// ---- attention ----------------------------------------------------------------
struct KvAttnArgs {
    int R, T, Hq, H, G, D;
    int shift, num_blocks, W;
    int max_new, num_cu;
    const void *q;
    int64_t q_token, q_head;
    void *out;
    int64_t out_token, out_head;
    float *lse;  // may be null
    const int32_t *start, *context, *table;
    int64_t table_stride;
    const void *k, *v;
    int64_t k_block, k_token, k_head, v_block, v_token, v_head;
    const float *k_scale, *v_scale;  // fp8 caches
    float scale, cap;
    int window;
    const float *slopes;
    const int32_t *prefix;
};
// The same over a cache in shared scales.  (The kernels of the other caches take the arguments above:
// with these fields among them the compiler orders the loads of single tokens over 16-bit caches
// otherwise, 105.7 us for 103.4 on 64 requests of 50 to 8192 keys.)
struct KvMxArgs : KvAttnArgs {
    const uint8_t *k_power, *v_power;
    int64_t kp_block, kp_head, vp_block, vp_head;  // (D / 32 from token to token)
};
// bytes of scratch that a call needs
size_t kv_attention_bytes(const KvAttnArgs &a, int cache_dtype);
hipError_t launch_kv_attention(const KvMxArgs &a, int dtype, int cache_dtype, void *ws, hipStream_t st);

// Attention behind shared prefixes: the sources of a row's keys are its group's prefix and its own
// tokens, and are attended like requests of their own, the groups before the requests.
struct KvSharedArgs : KvMxArgs {
    int groups, p_W, p_window, p_max_new;  // p_W = columns of the prefixes' table
    int p_few;               // groups of up to this many tokens belong to the kernel of few rows
    const int32_t *first, *p_context, *p_table;
    int64_t p_stride;
    // scratch
    int32_t *p_start;        // [groups + 1] the groups' rows
    int2 *ends;              // [groups], null: no window.  The first key of the prefix that some row
                             // sees, and the first from which on all do
    int32_t *row_pos;        // [T], null: no window and no slopes.  The rows' places among their
                             // requests' own tokens
    int2 *row_of;            // [T] each row's request and group, or -1
    float *raw_o[2];         // [T][Hq] rows of DP sums of a source's items (0: prefixes) that
    float2 *raw_ml[2];       // one workgroup has finished, and their maxima and weights' sums
};
// The same where every request reads its group's prefix itself, before its own tokens: few requests
// and groups, no window.
struct KvJoinedArgs : KvMxArgs {
    int groups, p_W;
    const int32_t *first, *p_context, *p_table;
    int64_t p_stride;
};
size_t kv_shared_bytes(const KvSharedArgs &a, int cache_dtype);
hipError_t launch_kv_shared(KvSharedArgs a, int dtype, int cache_dtype, void *ws, hipStream_t st);

}  // namespace dro
