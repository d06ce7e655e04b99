// Launchers of the paged-cache kernels (block tables, store, attention).
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

// ---- store --------------------------------------------------------------------
struct KvStoreArgs {
    int T, H, D;
    int shift;
    int64_t slots;                // num_blocks << shift
    const void *x[2];             // keys, values
    int64_t x_token[2], x_head[2];
    void *c[2];                   // the cache's
    int64_t c_block[2], c_token[2], c_head[2];
    const float *scale[2];        // fp8 caches
    const int64_t *slot;
};
hipError_t launch_kv_store(const KvStoreArgs &a, int dtype, int cache_dtype, hipStream_t st);

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
// bytes of scratch that a call needs
size_t kv_attention_bytes(const KvAttnArgs &a, int cache_dtype);
hipError_t launch_kv_attention(const KvAttnArgs &a, int dtype, int cache_dtype, void *ws, hipStream_t st);

}  // namespace dro
