// The context behind the C ABI and what its entry points share: errors,
// argument checks, workspace carving, device selection and launch timing.
#pragma once

#include <hip/hip_runtime.h>

#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <string>
#include <vector>

#include "ivf.h"

struct ivf_ctx {
    int device = 0;
    hipStream_t stream = nullptr;
    int num_cus = 1;
    void *ws = nullptr;
    size_t ws_bytes = 0;
    std::string err;
    int force_fallback = 0;
    int sample_rank = 0;
    int build_blocks = 0;
    int screen_waves = 8;
    int fp32_screen = 0;  // 1: uint8 rows also take the fp32 MFMA screen
    int two_plane_only = 0;  // 1: no single-plane int8 pre-screen
    int s1_id_order = 0;     // 1: the single plane visits centroids in id order
    int force_rescreen = 0;  // 1: the single-plane screen lists every row
    int64_t rescreen_cap = 0;  // > 0: smaller capacity of that list (tests)
    int64_t assign_slice = 0;  // > 0: shorter assignment slices (tests)
    unsigned long long *last_stats = nullptr;  // device, inside the workspace
    int64_t last_sample = 0;
    // kernel timing (IVF_OPT_PROFILE): an event pair per launch of the last call
    int profile = 0;
    std::vector<hipEvent_t> events;
    std::vector<std::string> knames;
    std::vector<std::string> retired;  // names handed out by the last read
    size_t kused = 0;
    const char *cur_call = "";
    ~ivf_ctx()
    {
        for (hipEvent_t e : events) (void)hipEventDestroy(e);
    }
};

namespace ivf {

constexpr size_t kAlign = 256;

inline ivf_status fail(ivf_ctx *ctx, ivf_status st, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    if (ctx) ctx->err = buf;
    return st;
}

// Bump allocator over the workspace (base == nullptr: sizing only).
struct Carver {
    char *base;
    size_t off = 0;
    explicit Carver(void *b) : base((char *)b) {}
    template <typename T> T *take(size_t count)
    {
        off = (off + kAlign - 1) / kAlign * kAlign;
        T *p = base ? (T *)(base + off) : nullptr;
        off += count * sizeof(T);
        return p;
    }
};

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

inline bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + nb && b0 < a0 + na;
}

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev)
    {
        if (dev < 0) {  // validation-only context
            ok = false;
            return;
        }
        if (hipGetDevice(&prev) != hipSuccess) {
            ok = false;
            return;
        }
        if (prev != dev && hipSetDevice(dev) != hipSuccess) ok = false;
    }
    ~DeviceGuard()
    {
        int cur;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

// least: what the call can do with; need: what ivf_workspace_bytes asks for
inline ivf_status check_ws(ivf_ctx *ctx, size_t least, size_t need)
{
    if (!ctx->ws || ctx->ws_bytes < least)
        return fail(ctx, IVF_ENOMEM, "workspace too small: %zu bytes required, %zu provided", need,
                    ctx->ws ? ctx->ws_bytes : (size_t)0);
    return IVF_OK;
}
inline ivf_status check_ws(ivf_ctx *ctx, size_t need) { return check_ws(ctx, need, need); }

#define HIP_TRY(expr)                                                                      \
    do {                                                                                   \
        hipError_t e_ = (expr);                                                            \
        if (e_ != hipSuccess)                                                              \
            return fail(ctx, IVF_EDEVICE, "%s failed: %s", #expr, hipGetErrorString(e_));  \
    } while (0)

// Records the start event of a kernel launch; returns its slot or -1.
inline int prof_start(ivf_ctx *ctx, const char *name)
{
    if (!ctx->profile) return -1;
    const size_t i = ctx->kused++;
    while (ctx->events.size() < 2 * ctx->kused) {
        hipEvent_t e;
        if (hipEventCreate(&e) != hipSuccess) {
            --ctx->kused;
            return -1;
        }
        ctx->events.push_back(e);
    }
    ctx->knames.push_back(std::string(ctx->cur_call) + "/" + name);
    (void)hipEventRecord(ctx->events[2 * i], ctx->stream);
    return (int)i;
}

inline void prof_stop(ivf_ctx *ctx, int slot)
{
    if (slot >= 0) (void)hipEventRecord(ctx->events[2 * slot + 1], ctx->stream);
}

// Launch with optional event timing around it.
#define TIMED(name, expr)                        \
    do {                                         \
        const int slot_ = prof_start(ctx, name); \
        HIP_TRY(expr);                           \
        prof_stop(ctx, slot_);                   \
    } while (0)

}  // namespace ivf
