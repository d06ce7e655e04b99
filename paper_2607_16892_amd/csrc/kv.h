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
    uint8_t *power[2];            // caches in shared scales
    int64_t p_block[2], p_token[2], p_head[2];
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
    const uint8_t *k_power, *v_power;  // caches in shared scales
    int64_t kp_block, kp_token, kp_head, vp_block, vp_token, vp_head;
    float scale, cap;
    int window;
    const float *slopes;
    const int32_t *prefix;
    // Over shared prefixes the requests are the groups: every row sees all keys, but for a window.
    float2 *raw_ml;            // null: not over prefixes.  [T][Hq] maxima and sums of the weights,
    float *raw_o;              // and sums of the values, DP floats a row, as they are
    const int32_t *row_pos;    // [T] the rows' places among their requests' own tokens
    const int2 *ends;          // [R], null: no window.  The first key that some row of the group sees,
    int prefix_window;         // and the first from which on all do
    // Behind shared prefixes: such results, to be joined with.
    const float2 *with_ml;     // null: none
    const float *with_o;
};
// bytes of scratch that a call needs
size_t kv_attention_bytes(const KvAttnArgs &a, int cache_dtype);
hipError_t launch_kv_attention(const KvAttnArgs &a, int dtype, int cache_dtype, void *ws, hipStream_t st);

// The shared prefixes of groups of requests.
struct KvSharedArgs {
    int groups, W;             // W = table columns
    int max_new, window;
    const int32_t *first, *context, *table;
    int64_t table_stride;
};
size_t kv_shared_bytes(const KvAttnArgs &a, const KvSharedArgs &s, int cache_dtype);
hipError_t launch_kv_shared(const KvAttnArgs &a, const KvSharedArgs &s, int dtype, int cache_dtype, void *ws,
                            hipStream_t st);

}  // namespace dro
