// C ABI of the paged cache: argument checks and launches of kv_block_tables,
// kv_store and kv_attention.  Every entry point only enqueues work on the caller's
// stream, except where the workspace has to grow: then the call waits for the device
// first.
#include <algorithm>
#include <cmath>

#include "context.h"
#include "kv.h"

namespace {

using namespace dro;

constexpr int64_t kMaxTokens = 1 << 24;
constexpr int kMaxRequests = 1 << 20;

// log2 of a block size of 16 .. 1024 tokens, or -1
int block_shift(int block)
{
    for (int s = 4; s <= 10; ++s)
        if (block == 1 << s) return s;
    return -1;
}

int check_pool_size(dro_ctx *ctx, int block, int num_blocks)
{
    if (block_shift(block) < 0)
        return fail(ctx, DRO_ELIMIT, "block=%d is not a power of two from 16 to 1024", block);
    if (num_blocks <= 0) return fail(ctx, DRO_EINVAL, "num_blocks=%d must be positive", num_blocks);
    if ((int64_t)num_blocks * block > 0x7fffffffLL)
        return fail(ctx, DRO_ELIMIT, "num_blocks * block = %lld exceeds 2^31 - 1 tokens",
                    (long long)num_blocks * block);
    return DRO_OK;
}

int check_table(dro_ctx *ctx, const int32_t *table, int R, int max_blocks, int64_t stride, int block)
{
    if (R < 0 || max_blocks <= 0)
        return fail(ctx, DRO_EINVAL, "R=%d must not be negative, max_blocks=%d be positive", R,
                    max_blocks);
    if (R && !table) return fail(ctx, DRO_EINVAL, "table is NULL");
    if (stride < max_blocks)
        return fail(ctx, DRO_EINVAL, "table_stride=%lld is less than max_blocks=%d",
                    (long long)stride, max_blocks);
    if ((int64_t)max_blocks * block > 1LL << 30)
        return fail(ctx, DRO_ELIMIT, "max_blocks * block = %lld exceeds 2^30 tokens a request",
                    (long long)max_blocks * block);
    if (R > kMaxRequests) return fail(ctx, DRO_ELIMIT, "R=%d exceeds 2^20 requests", R);
    if ((int64_t)R * max_blocks > 0x7fffffffLL || stride > (1LL << 40))
        return fail(ctx, DRO_ELIMIT, "R * max_blocks = %lld exceeds 2^31 - 1 table entries",
                    (long long)R * max_blocks);
    return DRO_OK;
}

int check_tokens(dro_ctx *ctx, int64_t T, int heads)
{
    if (T < 0) return fail(ctx, DRO_EINVAL, "T=%lld is negative", (long long)T);
    if (T > kMaxTokens || T * heads > (1LL << 30))
        return fail(ctx, DRO_ELIMIT, "T=%lld with %d heads exceeds 2^24 tokens or 2^30 rows",
                    (long long)T, heads);
    return DRO_OK;
}

int size_of(int dtype) { return dtype == DRO_FP8_E4M3 ? 1 : 2; }

bool aligned(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// A tensor of rows (token, head) of components next to one another.
int check_rows(dro_ctx *ctx, const char *name, const void *p, int64_t token, int64_t head)
{
    if (!p) return fail(ctx, DRO_EINVAL, "%s is NULL", name);
    if (!aligned(p, 16) || token % 8 || head % 8)
        return fail(ctx, DRO_EINVAL, "%s is not aligned to 16 bytes, or its strides %lld and %lld "
                    "are not multiples of 8", name, (long long)token, (long long)head);
    if (token < 0 || head < 0 || token > (1LL << 38) || head > (1LL << 38))
        return fail(ctx, DRO_ELIMIT, "the strides of %s are outside [0, 2^38]", name);
    return DRO_OK;
}

int check_cache(dro_ctx *ctx, const dro_kv_cache *c)
{
    if (!ctx) return DRO_EINVAL;
    if (!c) return fail(ctx, DRO_EINVAL, "cache is NULL");
    if (c->dtype != DRO_BF16 && c->dtype != DRO_F16 && c->dtype != DRO_FP8_E4M3)
        return fail(ctx, DRO_EINVAL, "cache type %d is unknown", c->dtype);
    if (c->heads <= 0 || c->dim <= 0)
        return fail(ctx, DRO_EINVAL, "heads and dim must be positive (heads=%d dim=%d)", c->heads,
                    c->dim);
    if (c->dim % 8 || c->dim > 256)
        return fail(ctx, DRO_ELIMIT, "dim=%d is not a multiple of 8 up to 256", c->dim);
    if (int rc = check_pool_size(ctx, c->block, c->num_blocks)) return rc;
    const int bytes = size_of(c->dtype);
    const int64_t s[6] = {c->k_block, c->k_token, c->k_head, c->v_block, c->v_token, c->v_head};
    if (!c->k || !c->v) return fail(ctx, DRO_EINVAL, "the cache's k or v is NULL");
    if (!aligned(c->k, 8 * bytes) || !aligned(c->v, 8 * bytes))
        return fail(ctx, DRO_EINVAL, "the cache's k or v is not aligned to 8 elements");
    for (int64_t x : s) {
        if (x % 8) return fail(ctx, DRO_EINVAL, "a cache stride %lld is not a multiple of 8",
                               (long long)x);
        if (x < 0 || x > (1LL << 38))
            return fail(ctx, DRO_ELIMIT, "a cache stride %lld is outside [0, 2^38]", (long long)x);
    }
    // offsets of a token within its block are 32-bit in the kernels
    if (std::max(c->k_token, c->v_token) * c->block * bytes > 0x7fffffffLL)
        return fail(ctx, DRO_ELIMIT, "the tokens of a block lie 2^31 bytes or more apart");
    const bool scaled = c->k_scale && c->v_scale;
    if (scaled != (c->dtype == DRO_FP8_E4M3) || (!c->k_scale) != (!c->v_scale))
        return fail(ctx, DRO_EINVAL, "k_scale and v_scale go with DRO_FP8_E4M3 and no other type");
    return DRO_OK;
}

int check_dtype(dro_ctx *ctx, int dtype, const dro_kv_cache *c)
{
    if (dtype != DRO_BF16 && dtype != DRO_F16)
        return fail(ctx, DRO_EINVAL, "type %d is neither DRO_BF16 nor DRO_F16", dtype);
    if (c->dtype != DRO_FP8_E4M3 && c->dtype != dtype)
        return fail(ctx, DRO_EINVAL, "type %d differs from the cache's %d", dtype, c->dtype);
    return DRO_OK;
}

}  // namespace

extern "C" {

int kv_block_tables(dro_ctx *ctx, const dro_kv_pool *p, const int32_t *len, const int32_t *add,
                    const int32_t *reserve, int64_t T, int32_t *held_out, int32_t *free_out,
                    int32_t *context, int32_t *start, int64_t *slot, int32_t *pos,
                    uint8_t *granted, dro_stream_t stream)
{
    if (!ctx) return DRO_EINVAL;
    if (!p) return fail(ctx, DRO_EINVAL, "pool is NULL");
    int rc = check_pool_size(ctx, p->block, p->num_blocks);
    if (rc) return rc;
    if ((rc = check_table(ctx, p->table, p->R, p->max_blocks, p->table_stride, p->block))) return rc;
    if ((rc = check_tokens(ctx, T, 1))) return rc;
    if (!p->free_list || !p->free_count || (p->R && (!p->held || !len || !add)))
        return fail(ctx, DRO_EINVAL, "free_list, held, free_count, len or add is NULL");
    if (!free_out || !start || (p->R && (!held_out || !context || !granted)) || (T && (!slot || !pos)))
        return fail(ctx, DRO_EINVAL, "a required output is NULL");
    ENTER_DEVICE(ctx);
    hipStream_t st = (hipStream_t)stream;
    if ((rc = ensure_ws(ctx, rup((size_t)p->R * sizeof(int4)) + rup((size_t)p->R * 4) + rup(8), st))) return rc;
    Arena ar{(char *)ctx->ws, 0};
    KvTablesArgs a{};
    a.R = p->R;
    a.shift = block_shift(p->block);
    a.num_blocks = p->num_blocks;
    a.W = p->max_blocks;
    a.table_stride = p->table_stride;
    a.table = p->table;
    a.free_list = p->free_list;
    a.held = p->held;
    a.free_count = p->free_count;
    a.len = len;
    a.add = add;
    a.reserve = reserve;
    a.T = (int)T;
    a.held_out = held_out;
    a.free_out = free_out;
    a.context = context;
    a.start = start;
    a.slot = slot;
    a.pos = pos;
    a.granted = granted;
    a.rows = ar.take<int4>(p->R);
    a.backs = ar.take<uint32_t>(p->R);
    a.tops = ar.take<int32_t>(2);
    HIPCHK(launch_kv_tables(a, st));
    return DRO_OK;
}

int kv_store(dro_ctx *ctx, const dro_kv_cache *c, int32_t dtype, int64_t T, const void *k,
             int64_t k_token, int64_t k_head, const void *v, int64_t v_token, int64_t v_head,
             const int64_t *slot, dro_stream_t stream)
{
    int rc = check_cache(ctx, c);
    if (rc) return rc;
    if ((rc = check_dtype(ctx, dtype, c))) return rc;
    if ((rc = check_tokens(ctx, T, c->heads))) return rc;
    if (T == 0) return DRO_OK;
    if ((rc = check_rows(ctx, "k", k, k_token, k_head))) return rc;
    if ((rc = check_rows(ctx, "v", v, v_token, v_head))) return rc;
    if (!slot) return fail(ctx, DRO_EINVAL, "slot is NULL");
    ENTER_DEVICE(ctx);
    KvStoreArgs a{};
    a.T = (int)T;
    a.H = c->heads;
    a.D = c->dim;
    a.shift = block_shift(c->block);
    a.slots = (int64_t)c->num_blocks * c->block;
    a.x[0] = k;
    a.x[1] = v;
    a.x_token[0] = k_token;
    a.x_token[1] = v_token;
    a.x_head[0] = k_head;
    a.x_head[1] = v_head;
    a.c[0] = c->k;
    a.c[1] = c->v;
    a.c_block[0] = c->k_block;
    a.c_block[1] = c->v_block;
    a.c_token[0] = c->k_token;
    a.c_token[1] = c->v_token;
    a.c_head[0] = c->k_head;
    a.c_head[1] = c->v_head;
    a.scale[0] = c->k_scale;
    a.scale[1] = c->v_scale;
    a.slot = slot;
    HIPCHK(launch_kv_store(a, dtype, c->dtype, (hipStream_t)stream));
    return DRO_OK;
}

int kv_attention(dro_ctx *ctx, const dro_kv_cache *c, const dro_kv_rows *q, dro_stream_t stream)
{
    int rc = check_cache(ctx, c);
    if (rc) return rc;
    if (!q) return fail(ctx, DRO_EINVAL, "rows is NULL");
    if ((rc = check_dtype(ctx, q->dtype, c))) return rc;
    if (q->Hq <= 0 || q->Hq % c->heads)
        return fail(ctx, DRO_EINVAL, "Hq=%d is not a multiple of the cache's %d heads", q->Hq, c->heads);
    if ((rc = check_table(ctx, q->table, q->R, q->max_blocks, q->table_stride, c->block))) return rc;
    if ((rc = check_tokens(ctx, q->T, q->Hq))) return rc;
    if (!std::isfinite(q->scale) || !std::isfinite(q->softcap) || q->softcap < 0 || q->window < 0 ||
        q->max_new < 0)
        return fail(ctx, DRO_EINVAL, "scale=%g must be finite, softcap=%g, window=%d and max_new=%d "
                    "finite and not negative", q->scale, q->softcap, q->window, q->max_new);
    if (q->T == 0) return DRO_OK;
    if ((rc = check_rows(ctx, "q", q->q, q->q_token, q->q_head))) return rc;
    if ((rc = check_rows(ctx, "out", q->out, q->out_token, q->out_head))) return rc;
    if (!q->start || (q->R && !q->context)) return fail(ctx, DRO_EINVAL, "start or context is NULL");
    ENTER_DEVICE(ctx);
    KvAttnArgs a{};
    a.R = q->R;
    a.T = (int)q->T;
    a.Hq = q->Hq;
    a.H = c->heads;
    a.G = q->Hq / c->heads;
    a.D = c->dim;
    a.shift = block_shift(c->block);
    a.num_blocks = c->num_blocks;
    a.W = q->max_blocks;
    a.max_new = q->max_new;
    a.num_cu = ctx->num_cu;
    a.q = q->q;
    a.q_token = q->q_token;
    a.q_head = q->q_head;
    a.out = q->out;
    a.out_token = q->out_token;
    a.out_head = q->out_head;
    a.lse = q->lse;
    a.start = q->start;
    a.context = q->context;
    a.table = q->table;
    a.table_stride = q->table_stride;
    a.k = c->k;
    a.v = c->v;
    a.k_block = c->k_block;
    a.k_token = c->k_token;
    a.k_head = c->k_head;
    a.v_block = c->v_block;
    a.v_token = c->v_token;
    a.v_head = c->v_head;
    a.k_scale = c->k_scale;
    a.v_scale = c->v_scale;
    a.scale = q->scale;
    a.cap = q->softcap;
    // a window as long as the table hides nothing
    a.window = q->window < (int64_t)q->max_blocks * c->block ? q->window : 0;
    a.slopes = q->slopes;
    a.prefix = q->prefix;
    if ((rc = ensure_ws(ctx, kv_attention_bytes(a, c->dtype), (hipStream_t)stream))) return rc;
    HIPCHK(launch_kv_attention(a, q->dtype, c->dtype, ctx->ws, (hipStream_t)stream));
    return DRO_OK;
}

}  // extern "C"
