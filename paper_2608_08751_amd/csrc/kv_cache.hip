// Writing tokens into the 4-bit cache, the summaries of its full blocks, and
// reading both back.
//
// A lane holds 8 channels of one token's key and of its value (16 bytes of
// each), four neighbouring lanes the 32 that share a scale: two exchanges give
// their largest magnitude, v_cvt_scalef32_pk_fp4_f32 the codes (to nearest, ties to
// even), and each lane writes one dword of key and one of value codes. What has
// to move, 4 bytes read and 17 / 16 written per channel of key and value together,
// bounds a prompt: 29,000 tokens of 8 heads x 128 f16 (120 MB in, 32 MB out) 28 us,
// 5.4 TB/s, reading them back 24 us, 6.2 TB/s, their summaries (fp64 sums, from L2)
// 11 us. A call of few tokens is one launch, 3 us.
#include "kv.h"
#include "kv_types.h"

namespace ivf {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float max4(float x)
{
    x = fmaxf(x, __shfl_xor(x, 1));
    return fmaxf(x, __shfl_xor(x, 2));
}

// The scale byte of 32 channels whose largest magnitude is amax.
template <typename TT> __device__ __forceinline__ uint32_t scale_byte(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 129 + ((u & 0x7fffffu) > 0x600000u);  // amax in (3.5, 7] 2^e
    return (uint32_t)(min(max(e, TT::kMinExp), TT::kMaxExp) + 127);
}

struct Eight {
    float x[8];
};
template <typename TT> __device__ __forceinline__ Eight widen(u32x4 w)
{
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.x[2 * i] = TT::lo(w[i]);
        r.x[2 * i + 1] = TT::hi(w[i]);
    }
    return r;
}

__device__ __forceinline__ float top_of(const Eight &v, bool &bad)
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(v.x[i]);
        bad |= !(a <= 3.402823466e38f);
        m = fmaxf(m, a);
    }
    return m;
}

__device__ __forceinline__ uint32_t encode(const Eight &v, float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v.x[0], v.x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v.x[2], v.x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v.x[4], v.x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v.x[6], v.x[7], scale, 3);
    return w;
}

// A workgroup takes 256 / (D / 8) consecutive tokens of one head, so that the bytes it
// writes, tokens of a block side by side, meet in one L2 (single scale bytes and
// 64-byte rows from workgroups on several would each be a write of their own). Four times
// as many tokens, for more loads in flight a thread, were slower at every length from 64
// to 31,000 tokens (8 heads x 128: 5.6 -> 7.1 us, 36.3 -> 37.9).
template <int D> constexpr int tokens_at_once() { return kThreads / (D / 8); }

// The codes and scale bytes of 8 channels of a token's key and value; four lanes that share a
// scale call it together.
struct Coded {
    uint32_t kc, vc, ke, ve;
};
template <typename TT> __device__ __forceinline__ Coded code_token(u32x4 kw, u32x4 vw)
{
    const Eight kx = widen<TT>(kw), vx = widen<TT>(vw);
    bool bad = false;
    const float ka = max4(top_of(kx, bad)), va = max4(top_of(vx, bad));
    uint32_t b = bad;
    b |= __shfl_xor(b, 1);
    b |= __shfl_xor(b, 2);
    const uint32_t ke = scale_byte<TT>(ka), ve = scale_byte<TT>(va);
    if (b) return {0, 0, 255, 0};
    return {encode(kx, kv_scale(ke)), encode(vx, kv_scale(ve)), ke, ve};
}

template <typename TT, int D>
__device__ __forceinline__ void append_tokens(const KvCache &c, const KvRows &k, const KvRows &v,
                                              const int64_t *__restrict__ slots, int64_t T, uint32_t group, int h)
{
    constexpr int kPer = D / 8, kTok = tokens_at_once<D>();
    const int row = threadIdx.x / kPer, g8 = threadIdx.x % kPer;
    const int64_t t = (int64_t)group * kTok + row;
    u32x4 kw = {0, 0, 0, 0}, vw = {0, 0, 0, 0};
    int64_t slot = -1;
    if (row < kTok && t < T) {
        slot = slots[t];
        kw = *(const u32x4 *)((const typename TT::elem *)k.p + t * k.ts + h * k.hs + 8 * g8);
        vw = *(const u32x4 *)((const typename TT::elem *)v.p + t * v.ts + h * v.hs + 8 * g8);
    }
    const Coded x = code_token<TT>(kw, vw);
    if (slot < 0 || (slot >> c.shift) >= c.blocks) return;
    const int place = (int)(slot & (c.bs - 1));
    uint8_t *rec = c.rec + ((slot >> c.shift) * c.heads + h) * c.rec_bytes();
    *(uint32_t *)(rec + place * (D / 2) + 4 * g8) = x.kc;
    *(uint32_t *)(rec + c.v_codes() + place * (D / 2) + 4 * g8) = x.vc;
    if ((g8 & 3) == 0) {
        rec[c.k_scales() + place * (D / 32) + g8 / 4] = (uint8_t)x.ke;
        rec[c.v_scales() + g8 / 4 * c.bs + place] = (uint8_t)x.ve;
    }
}

template <typename TT, int D>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvCache c, KvRows k, KvRows v,
                                                             const int64_t *__restrict__ slots, int64_t T)
{
    append_tokens<TT, D>(c, k, v, slots, T, blockIdx.x / (uint32_t)c.heads, blockIdx.x % (uint32_t)c.heads);
}

// Eight stored values: codes w, scale byte e of the key beside them 255 = NaN.
template <typename TT> __device__ __forceinline__ u32x4 stored(uint32_t w, uint32_t e, uint32_t ke)
{
    const float s = kv_scale(e);
    u32x4 r = {TT::template decode<0>(w, s), TT::template decode<1>(w, s), TT::template decode<2>(w, s),
               TT::template decode<3>(w, s)};
    if (ke == 255) r = (u32x4){0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
    return r;
}

// Summaries of the blocks whose last slot is among 64 consecutive tokens, one
// head: the workgroup sums such a block's keys, thread (token row, 8 channels),
// in fp64 (exact for all but keys of far more than 2^40 different magnitudes,
// so the order does not show). FRESH: the tokens of this call are not in the cache yet;
// the workgroup finds the block's ones among the slots and codes them itself.
template <typename TT, int D, bool FRESH>
__device__ __forceinline__ void summarise(const KvCache &c, const KvRows &k, const KvRows &v,
                                          const int64_t *__restrict__ slots, int64_t T, uint32_t group, int h)
{
    constexpr int kPer = D / 8, kTok = tokens_at_once<D>(), kAhead = 4;
    __shared__ double sums[kTok * D];
    __shared__ float top[kThreads / 64];
    __shared__ int from[FRESH ? 128 : 1];  // the token of this call in each slot of the block, or -1
    const int tid = threadIdx.x;
    const int64_t t = (int64_t)group * 64 + (tid & 63);
    const int64_t mine = t < T ? slots[t] : -1;
    uint64_t full = __ballot(mine >= 0 && (mine & (c.bs - 1)) == c.bs - 1 && (mine >> c.shift) < c.blocks);
    const int row = tid / kPer, g8 = tid % kPer;
    while (full) {
        const int l = __ffsll((unsigned long long)full) - 1;
        full &= full - 1;
        const int64_t block = __shfl(mine, l) >> c.shift;
        const int64_t at = block * c.heads + h;
        const uint8_t *rec = c.rec + at * c.rec_bytes();
        if (FRESH) {
            if (tid < 128) from[tid] = -1;
            __syncthreads();
            for (int64_t i = tid; i < T; i += kThreads) {
                const int64_t slot = slots[i];
                if (slot >= 0 && slot >> c.shift == block) from[slot & (c.bs - 1)] = (int)i;
            }
            __syncthreads();
        }
        if (row < kTok) {
            double s[8] = {};
            for (int p0 = row; p0 < c.bs; p0 += kTok * kAhead) {
                uint32_t w[kAhead], e[kAhead];
                u32x4 kw[kAhead], vw[kAhead];
                bool fresh[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int p = p0 + i * kTok;
                    w[i] = 0;
                    e[i] = 127;
                    const int64_t x = FRESH && p < c.bs ? from[p] : -1;
                    fresh[i] = x >= 0;
                    if (fresh[i]) {
                        kw[i] = *(const u32x4 *)((const typename TT::elem *)k.p + x * k.ts + h * k.hs + 8 * g8);
                        vw[i] = *(const u32x4 *)((const typename TT::elem *)v.p + x * v.ts + h * v.hs + 8 * g8);
                    } else if (p < c.bs) {
                        w[i] = *(const uint32_t *)(rec + p * (D / 2) + 4 * g8);
                        e[i] = rec[c.k_scales() + p * (D / 32) + g8 / 4];
                    }
                }
                if (FRESH) {
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        if (!fresh[i]) continue;  // the same for the lanes that share a scale
                        const Coded x = code_token<TT>(kw[i], vw[i]);
                        w[i] = x.kc;
                        e[i] = x.ke;
                    }
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const Eight x = widen<TT>(stored<TT>(w[i], e[i] == 255 ? 0 : e[i], 0));  // NaN counts 0 (its codes are)
#pragma unroll
                    for (int d = 0; d < 8; ++d) s[d] += (double)x.x[d];
                }
            }
#pragma unroll
            for (int d = 0; d < 8; ++d) sums[(row * kPer + g8) * 8 + d] = s[d];
        }
        __syncthreads();
        float mean = 0.f;
        if (tid < D) {
            double a = 0.;
#pragma unroll
            for (int q = 0; q < kTok; ++q) a += sums[q * D + tid];
            mean = (float)a * (1.f / (float)c.bs);
        }
        float m = fabsf(mean);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
        if ((tid & 63) == 0) top[tid >> 6] = m;
        __syncthreads();
        float amax = top[0];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) amax = fmaxf(amax, top[w]);
        const bool live = amax >= 0x1p-100f && amax <= 3.402823466e38f;
        if (tid < D) {
            const float inv = 127.f / amax;
            c.summary[at * D + tid] = live ? (int8_t)(int)rintf(mean * inv) : (int8_t)0;
        }
        if (tid == 0) c.weight[at] = live ? amax / 127.f : 0.f;
        __syncthreads();
    }
}

template <typename TT, int D>
__global__ __launch_bounds__(kThreads) void kv_summary_kernel(KvCache c, const int64_t *__restrict__ slots, int64_t T)
{
    summarise<TT, D, false>(c, {}, {}, slots, T, blockIdx.x / (uint32_t)c.heads, blockIdx.x % (uint32_t)c.heads);
}

// Tokens and summaries in one launch: the first `token_groups` workgroups a head write, the others sum.
template <typename TT, int D>
__global__ __launch_bounds__(kThreads) void kv_append_few_kernel(KvCache c, KvRows k, KvRows v,
                                                                 const int64_t *__restrict__ slots, int64_t T,
                                                                 uint32_t token_groups)
{
    const uint32_t group = blockIdx.x / (uint32_t)c.heads;
    const int h = blockIdx.x % (uint32_t)c.heads;
    if (group < token_groups) append_tokens<TT, D>(c, k, v, slots, T, group, h);
    else summarise<TT, D, true>(c, k, v, slots, T, group - token_groups, h);
}

// The first `token_groups` workgroups a head read tokens, the others means.
template <typename TT, int D>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache c, const int64_t *__restrict__ slots, int64_t T,
                                                           typename TT::elem *k, typename TT::elem *v,
                                                           const int32_t *__restrict__ blocks, int64_t n,
                                                           float *__restrict__ mean, uint32_t token_groups)
{
    constexpr int kPer = D / 8, kTok = tokens_at_once<D>();
    const int h = blockIdx.x % (uint32_t)c.heads;
    const uint32_t group = blockIdx.x / (uint32_t)c.heads;
    const int row = threadIdx.x / kPer, g8 = threadIdx.x % kPer;
    if (row >= kTok) return;
    if (group < token_groups) {
        const int64_t t = (int64_t)group * kTok + row;
        if (t >= T) return;
        const int64_t slot = slots[t], at = (t * c.heads + h) * D + 8 * g8;
        uint32_t kc = 0, vc = 0, ke = 255, ve = 0;
        if (slot >= 0 && (slot >> c.shift) < c.blocks) {
            const int place = (int)(slot & (c.bs - 1));
            const uint8_t *rec = c.rec + ((slot >> c.shift) * c.heads + h) * c.rec_bytes();
            ke = rec[c.k_scales() + place * (D / 32) + g8 / 4];
            ve = rec[c.v_scales() + g8 / 4 * c.bs + place];
            kc = *(const uint32_t *)(rec + place * (D / 2) + 4 * g8);
            vc = *(const uint32_t *)(rec + c.v_codes() + place * (D / 2) + 4 * g8);
        }
        if (k) *(u32x4 *)(k + at) = stored<TT>(kc, ke, ke);
        if (v) *(u32x4 *)(v + at) = stored<TT>(vc, ve, ke);
        return;
    }
    const int64_t b = (int64_t)(group - token_groups) * kTok + row;
    if (b >= n) return;
    const int64_t block = blocks[b], at = (b * c.heads + h) * D + 8 * g8;
    f32x4 lo, hi;
    lo = hi = (f32x4){__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
    if (block >= 0 && block < c.blocks) {
        const int64_t s = block * c.heads + h;
        const float w = c.weight[s];
        const int8_t *q = c.summary + s * D + 8 * g8;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            lo[d] = (float)q[d] * w;
            hi[d] = (float)q[4 + d] * w;
        }
    }
    *(f32x4 *)(mean + at) = lo;
    *(f32x4 *)(mean + at + 4) = hi;
}

// Calls of at most kKvFewTokens tokens take one launch: a workgroup that sums a block codes the call's
// tokens in it anew and scans the call's slots for them. 8 heads x 128, consecutive tokens (every
// block of 64 full): 1 token 2.8 us in one launch and 4.0 in two, 64 tokens 5.3 and 5.6, 512 tokens 5.8 and 5.9,
// 1,024 tokens 6.5 and 6.0, 4,096 tokens 11.1 and 8.5; the host's share 4.0 and 6.0.
template <typename TT, int D> struct Launch {
    static unsigned groups(int64_t n) { return (unsigned)((n + tokens_at_once<D>() - 1) / tokens_at_once<D>()); }
    static hipError_t append(const KvCache &c, KvRows k, KvRows v, const int64_t *slots, int64_t T, hipStream_t s)
    {
        const unsigned sixties = (unsigned)((T + 63) / 64);
        if (T <= kKvFewTokens) {
            hipLaunchKernelGGL((kv_append_few_kernel<TT, D>), dim3((groups(T) + sixties) * c.heads), dim3(kThreads), 0, s, c, k,
                               v, slots, T, groups(T));
            return hipGetLastError();
        }
        hipLaunchKernelGGL((kv_append_kernel<TT, D>), dim3(groups(T) * c.heads), dim3(kThreads), 0, s, c, k, v, slots, T);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((kv_summary_kernel<TT, D>), dim3(sixties * c.heads), dim3(kThreads), 0, s, c, slots, T);
        return hipGetLastError();
    }
    static hipError_t read(const KvCache &c, const int64_t *slots, int64_t T, void *k, void *v, const int32_t *blocks,
                           int64_t n, float *mean, hipStream_t s)
    {
        typedef typename TT::elem elem;
        hipLaunchKernelGGL((kv_read_kernel<TT, D>), dim3((groups(T) + groups(n)) * c.heads), dim3(kThreads), 0, s, c, slots, T,
                           (elem *)k, (elem *)v, blocks, n, mean, groups(T));
        return hipGetLastError();
    }
};

// f(Launch<type, dim>()) for the cache's type and dim.
template <typename TT, typename F> hipError_t by_dim(const KvCache &c, F f)
{
    switch (c.dim) {
    case 64: return f(Launch<TT, 64>());
    case 96: return f(Launch<TT, 96>());
    case 128: return f(Launch<TT, 128>());
    case 192: return f(Launch<TT, 192>());
    default: return f(Launch<TT, 256>());
    }
}
template <typename F> hipError_t by_cache(const KvCache &c, F f)
{
    return c.bf16 ? by_dim<KvBf16>(c, f) : by_dim<KvF16>(c, f);
}

}  // namespace

hipError_t launch_kv_append(const KvCache &c, KvRows k, KvRows v, const int64_t *slots, int64_t T, hipStream_t s)
{
    return by_cache(c, [&](auto l) { return decltype(l)::append(c, k, v, slots, T, s); });
}

hipError_t launch_kv_read(const KvCache &c, const int64_t *slots, int64_t T, void *k, void *v, const int32_t *blocks,
                          int64_t n, float *mean, hipStream_t s)
{
    if (!k && !v) T = 0;
    if (T + n == 0) return hipSuccess;
    return by_cache(c, [&](auto l) { return decltype(l)::read(c, slots, T, k, v, blocks, n, mean, s); });
}

}  // namespace ivf
