// C entry point of token sampling (declared in include/ivf.h): argument checks and launch.
// The call does not synchronise with the host.
#include <hip/hip_runtime.h>

#include "ctx.h"
#include "ivf.h"
#include "sample.h"

using namespace ivf;

extern "C" {

size_t ivf_sample_bytes(int64_t T, int64_t V, int32_t cuts)
{
    if (T < 1 || T > INT32_MAX || check_threads(nullptr, T * 1024) != IVF_OK || V < 1 || V > kSampleMaxVocab) return 0;
    int num_cus = 256, dev = 0;
    if (hipGetDevice(&dev) == hipSuccess) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0) num_cus = n;
    }
    return sample_workspace(T, sample_parts(T, V, num_cus), cuts != 0, nullptr, nullptr);
}

ivf_status ivf_sample(ivf_ctx *ctx, const void *logits, int dt, int64_t row_stride, int64_t T, int64_t V,
                      const float *uniform, const float *temperature, const int32_t *top_k, const float *top_p,
                      const float *min_p, int32_t *out_token, float *out_logprob)
{
    return guarded(ctx, "sample", [&]() -> ivf_status {
        if (dt != IVF_F32 && dt != IVF_F16 && dt != IVF_BF16)
            return fail(ctx, IVF_EUNSUPPORTED, "logits must be IVF_F32, IVF_F16 or IVF_BF16 (got %d)", dt);
        if (T < 0 || V < 1) return fail(ctx, IVF_EINVAL, "T >= 0 and V >= 1 are wanted");
        if (T == 0) return IVF_OK;
        if (V > kSampleMaxVocab) return fail(ctx, IVF_EUNSUPPORTED, "V must be at most %lld", (long long)kSampleMaxVocab);
        if (row_stride < 0 || row_stride > ((int64_t)1 << 40)) return fail(ctx, IVF_EINVAL, "row_stride must be in [0, 2^40]");
        if (!logits || !uniform || !out_token) return fail(ctx, IVF_EINVAL, "null pointer argument");
        ivf_status st = IVF_OK;
        if (T > INT32_MAX || (st = check_threads(ctx, T * 1024)) != IVF_OK)
            return fail(ctx, IVF_EUNSUPPORTED, "too many rows for one call");
        const size_t element = dt == IVF_F32 ? 4 : 2;
        const void *rows[] = {logits};
        const void *words[] = {uniform, temperature, top_k, top_p, min_p, out_token, out_logprob};
        if ((st = check_elements(ctx, rows, element)) != IVF_OK || (st = check_elements(ctx, words, 4)) != IVF_OK) return st;
        const Span ins[] = {{logits, ((size_t)(T - 1) * row_stride + V) * element}, {uniform, (size_t)T * 4},
                            {temperature, (size_t)T * 4}, {top_k, (size_t)T * 4}, {top_p, (size_t)T * 4}, {min_p, (size_t)T * 4}};
        const Span outs[] = {{out_token, (size_t)T * 4}, {out_logprob, (size_t)T * 4}};
        if ((st = no_overlap(ctx, outs, 2, ins, 6)) != IVF_OK) return st;
        Sample a = {logits, dt, row_stride, T, (int)V, uniform, temperature, top_k, top_p, min_p, out_token, out_logprob, 0, 0};
        const int parts = sample_parts(T, V, ctx->num_cus);
        const bool cuts = top_k || top_p;
        const size_t need = sample_workspace(T, parts, cuts, nullptr, nullptr);
        if (need && (st = check_ws(ctx, need)) != IVF_OK) return st;
        SampleShare share;
        sample_workspace(T, parts, cuts, need ? (char *)ctx->ws : nullptr, &share);
        DeviceGuard g(ctx->device);
        if (!g.ok) return fail(ctx, IVF_EDEVICE, "no usable device (context device %d)", ctx->device);
        TIMED("sample", launch_sample(a, parts, share, ctx->stream));
        ctx->last_stats = nullptr;
        return IVF_OK;
    });
}

}  // extern "C"
