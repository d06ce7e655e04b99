// The context of the C ABI and what its entry points share: errors, the device
// of a call, the workspace.
#pragma once

#include <stdarg.h>
#include <stdio.h>

#include <new>
#include <vector>

#include "dro_internal.h"

struct dro_ctx {
    int device = 0;
    int num_cu = 256;
    int dense_bpc = 1;  // resident dense blocks per compute unit
    void *ws = nullptr;
    size_t ws_size = 0;
    // Workspaces that graphs captured on this context may replay on: once a call has
    // been captured, one that is outgrown stays until the context's end.
    struct Kept {
        void *ws;
        Kept *next;
    };
    bool captured = false;
    Kept *kept = nullptr;
    void *scratch = nullptr;    // device address of this device's no-allocation scratch array
    // The host-validated offsets and segment map last staged on the device, and
    // the stream they were staged on: a call whose host arrays and stream match
    // uses the staged copy without uploading it again.
    void *stage = nullptr;
    size_t stage_size = 0;
    bool staged = false;
    hipStream_t staged_stream = nullptr;
    std::vector<int64_t> staged_off;
    std::vector<int32_t> staged_seg;
    dro::RowPlan staged_rows{};  // parts of the staged segments; boff points into `stage`
    // the dense plan last made for the staged problem, and its grid (K = 0: none)
    int plan_K = 0, plan_M = 0;
    dro::DensePlan plan{};
    char err[1024] = {0};
    // host staging of the configuration-space count table (kept alive until
    // the next configuration search on this context has been enqueued)
    std::vector<long long> ways_h;
    std::vector<int32_t> gpus_h;
    // host copy of the row table (segments with unequal part counts)
    std::vector<int64_t> boff_h;
};

namespace dro {

inline int fail(dro_ctx *ctx, int code, const char *fmt, ...)
{
    if (ctx) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
        va_end(ap);
    }
    return code;
}

#define HIPCHK(expr)                                                                       \
    do {                                                                                   \
        hipError_t e_ = (expr);                                                            \
        if (e_ != hipSuccess)                                                              \
            return fail(ctx, DRO_EHIP, "%s: %s", #expr, hipGetErrorString(e_));           \
    } while (0)

// Makes the context's device current for the duration of a call.
struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        if (prev != dev) ok = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard()
    {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

// Makes ctx's device current for the rest of the calling entry point, or
// returns DRO_EHIP from it when the device cannot be selected.
#define ENTER_DEVICE(ctx)                                                                   \
    DeviceGuard guard_((ctx)->device);                                                      \
    if (!guard_.ok) return fail((ctx), DRO_EHIP, "cannot select device %d", (ctx)->device)

// Bump allocator over the context workspace.
struct Arena {
    char *base = nullptr;
    size_t off = 0;
    template <class T> T *take(size_t count)
    {
        off = (off + 255) & ~size_t(255);
        T *p = reinterpret_cast<T *>(base + off);
        off += count * sizeof(T);
        return p;
    }
};

inline size_t rup(size_t v) { return (v + 255) & ~size_t(255); }

inline int ensure_ws(dro_ctx *ctx, size_t need, hipStream_t st)
{
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    const bool known = hipStreamIsCapturing(st, &capture) == hipSuccess;
    if (!known) (void)hipGetLastError();
    const bool capturing = !known || capture != hipStreamCaptureStatusNone;
    ctx->captured |= capturing;
    if (need <= ctx->ws_size) return DRO_OK;
    if (capturing)  // growing it would end the capture
        return fail(ctx, DRO_EHIP, "a captured call needs a workspace of %zu bytes and there are %zu: "
                    "make the call once before its capture", need, ctx->ws_size);
    dro_ctx::Kept *kept = nullptr;
    if (ctx->ws && ctx->captured) {
        kept = new (std::nothrow) dro_ctx::Kept{ctx->ws, ctx->kept};
        if (!kept) return fail(ctx, DRO_ENOMEM, "no host memory for a workspace record");
        ctx->kept = kept;
    } else if (ctx->ws) {
        // earlier work may still read the old buffer: on this stream, or on another
        // stream the context was used on before (growth is rare, so wait for all)
        HIPCHK(hipDeviceSynchronize());
        HIPCHK(hipFree(ctx->ws));
    }
    ctx->ws = nullptr;
    ctx->ws_size = 0;
    const size_t sz = need + need / 4 + (1u << 20);
    if (hipMalloc(&ctx->ws, sz) != hipSuccess) {
        (void)hipGetLastError();
        ctx->ws = nullptr;
        return fail(ctx, DRO_ENOMEM, "workspace allocation of %zu bytes failed", sz);
    }
    ctx->ws_size = sz;
    return DRO_OK;
}

inline void free_ws(dro_ctx *ctx)
{
    if (ctx->ws) (void)hipFree(ctx->ws);
    while (dro_ctx::Kept *k = ctx->kept) {
        ctx->kept = k->next;
        (void)hipFree(k->ws);
        delete k;
    }
}

}  // namespace dro
