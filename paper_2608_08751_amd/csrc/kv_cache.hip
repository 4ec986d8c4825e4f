// Writing tokens into the 4-bit cache, the summaries of its full blocks, and
// reading both back.
//
// A lane holds 8 channels of one token's key and of its value (16 bytes of
// each), four neighbouring lanes the 32 that share a scale: two exchanges give
// their largest magnitude, v_cvt_scalef32_pk_fp4_f32 the codes (to nearest, ties to
// even), and each lane writes one dword of key and one of value codes. What has
// to move, 4 bytes read and 17 / 16 written per channel of key and value together,
// bounds a prompt; a single token is one launch.
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

// Item = (token, head, 8 channels); dim / 8 is a multiple of 4, so the lanes of
// a scale group are neighbours of one wave.
template <typename TT>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvCache c, KvRows k, KvRows v,
                                                             const int64_t *__restrict__ slots, int64_t T)
{
    const uint32_t per = (uint32_t)c.dim / 8, row = per * (uint32_t)c.heads;
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = item / row;
    const bool in = t < T;
    const uint32_t r = (uint32_t)(item - t * row), h = r / per, g8 = r - h * per;
    u32x4 kw = {0, 0, 0, 0}, vw = {0, 0, 0, 0};
    int64_t slot = -1;
    if (in) {
        slot = slots[t];
        kw = *(const u32x4 *)((const typename TT::elem *)k.p + t * k.ts + h * k.hs + 8 * g8);
        vw = *(const u32x4 *)((const typename TT::elem *)v.p + t * v.ts + h * v.hs + 8 * g8);
    }
    const Eight kx = widen<TT>(kw), vx = widen<TT>(vw);
    bool bad = false;
    const float ka = max4(top_of(kx, bad)), va = max4(top_of(vx, bad));
    uint32_t b = bad;
    b |= __shfl_xor(b, 1);
    b |= __shfl_xor(b, 2);
    uint32_t ke = scale_byte<TT>(ka), ve = scale_byte<TT>(va);
    uint32_t kc = encode(kx, kv_scale(ke)), vc = encode(vx, kv_scale(ve));
    if (b) {
        ke = 255;
        ve = kc = vc = 0;
    }
    if (slot < 0 || (slot >> c.shift) >= c.blocks) return;
    const int place = (int)(slot & (c.bs - 1));
    uint8_t *rec = c.rec + ((slot >> c.shift) * c.heads + h) * c.rec_bytes();
    *(uint32_t *)(rec + place * (c.dim / 2) + 4 * g8) = kc;
    *(uint32_t *)(rec + c.v_codes() + place * (c.dim / 2) + 4 * g8) = vc;
    if ((g8 & 3) == 0) {
        rec[c.k_scales() + place * (c.dim / 32) + g8 / 4] = (uint8_t)ke;
        rec[c.v_scales() + (int)(g8 / 4) * c.bs + place] = (uint8_t)ve;
    }
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
// so the order does not show).
template <typename TT>
__global__ __launch_bounds__(kThreads) void kv_summary_kernel(KvCache c, const int64_t *__restrict__ slots, int64_t T)
{
    __shared__ double sums[kThreads * 8];
    __shared__ float top[kThreads / 64];
    const int tid = threadIdx.x, h = blockIdx.y;
    const int64_t t = (int64_t)blockIdx.x * 64 + (tid & 63);
    const int64_t mine = t < T ? slots[t] : -1;
    uint64_t full = __ballot(mine >= 0 && (mine & (c.bs - 1)) == c.bs - 1 && (mine >> c.shift) < c.blocks);
    const int per = c.dim / 8, rows = kThreads / per;
    const int row = tid / per, g8 = tid - row * per;
    while (full) {
        const int l = __ffsll((unsigned long long)full) - 1;
        full &= full - 1;
        const int64_t block = __shfl(mine, l) >> c.shift;
        const int64_t at = block * c.heads + h;
        const uint8_t *rec = c.rec + at * c.rec_bytes();
        double s[8] = {};
        if (row < rows) {
            for (int p = row; p < c.bs; p += rows) {
                const uint32_t w = *(const uint32_t *)(rec + p * (c.dim / 2) + 4 * g8);
                const uint32_t e = rec[c.k_scales() + p * (c.dim / 32) + g8 / 4];
                if (e != 255) {
                    const Eight x = widen<TT>(stored<TT>(w, e, e));
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] += (double)x.x[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[(row * per + g8) * 8 + i] = s[i];
        }
        __syncthreads();
        float mean = 0.f;
        if (tid < c.dim) {
            double a = 0.;
            for (int q = 0; q < rows; ++q) a += sums[q * c.dim + tid];
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
        if (tid < c.dim) {
            const float inv = 127.f / amax;
            c.summary[at * c.dim + tid] = live ? (int8_t)(int)rintf(mean * inv) : (int8_t)0;
        }
        if (tid == 0) c.weight[at] = live ? amax / 127.f : 0.f;
        __syncthreads();
    }
}

template <typename TT>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache c, const int64_t *__restrict__ slots, int64_t T,
                                                           typename TT::elem *k, typename TT::elem *v,
                                                           const int32_t *__restrict__ blocks, int64_t n,
                                                           float *__restrict__ mean)
{
    const uint32_t per = (uint32_t)c.dim / 8, row = per * (uint32_t)c.heads;
    const int64_t item = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    int64_t t = item / row;
    const uint32_t r = (uint32_t)(item - t * row), h = r / per, g8 = r - h * per;
    const int64_t tokens = k || v ? T : 0;
    if (t < tokens) {
        const int64_t slot = slots[t];
        u32x4 kw = {0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu}, vw = kw;
        if (slot >= 0 && (slot >> c.shift) < c.blocks) {
            const int place = (int)(slot & (c.bs - 1));
            const uint8_t *rec = c.rec + ((slot >> c.shift) * c.heads + h) * c.rec_bytes();
            const uint32_t ke = rec[c.k_scales() + place * (c.dim / 32) + g8 / 4];
            const uint32_t ve = rec[c.v_scales() + (int)(g8 / 4) * c.bs + place];
            kw = stored<TT>(*(const uint32_t *)(rec + place * (c.dim / 2) + 4 * g8), ke, ke);
            vw = stored<TT>(*(const uint32_t *)(rec + c.v_codes() + place * (c.dim / 2) + 4 * g8), ve, ke);
        }
        const int64_t at = (t * c.heads + h) * c.dim + 8 * g8;
        if (k) *(u32x4 *)(k + at) = kw;
        if (v) *(u32x4 *)(v + at) = vw;
        return;
    }
    t -= tokens;
    if (t >= n) return;
    const int64_t block = blocks[t], at = (t * c.heads + h) * c.dim + 8 * g8;
    f32x4 lo, hi;
    lo = hi = (f32x4){__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
    if (block >= 0 && block < c.blocks) {
        const int64_t b = block * c.heads + h;
        const float w = c.weight[b];
        const int8_t *q = c.summary + b * c.dim + 8 * g8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = (float)q[i] * w;
            hi[i] = (float)q[4 + i] * w;
        }
    }
    *(f32x4 *)(mean + at) = lo;
    *(f32x4 *)(mean + at + 4) = hi;
}

}  // namespace

hipError_t launch_kv_append(const KvCache &c, KvRows k, KvRows v, const int64_t *slots, int64_t T, hipStream_t s)
{
    const int64_t items = T * c.heads * (c.dim / 8);
    const unsigned grid = (unsigned)((items + kThreads - 1) / kThreads);
    if (c.bf16)
        hipLaunchKernelGGL((kv_append_kernel<KvBf16>), dim3(grid), dim3(kThreads), 0, s, c, k, v, slots, T);
    else
        hipLaunchKernelGGL((kv_append_kernel<KvF16>), dim3(grid), dim3(kThreads), 0, s, c, k, v, slots, T);
    return hipGetLastError();
}

hipError_t launch_kv_summaries(const KvCache &c, const int64_t *slots, int64_t T, hipStream_t s)
{
    const dim3 grid((unsigned)((T + 63) / 64), (unsigned)c.heads);
    if (c.bf16)
        hipLaunchKernelGGL((kv_summary_kernel<KvBf16>), grid, dim3(kThreads), 0, s, c, slots, T);
    else
        hipLaunchKernelGGL((kv_summary_kernel<KvF16>), grid, dim3(kThreads), 0, s, c, slots, T);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvCache &c, const int64_t *slots, int64_t T, void *k, void *v, const int32_t *blocks,
                          int64_t n, float *mean, hipStream_t s)
{
    const int64_t items = ((k || v ? T : 0) + n) * c.heads * (c.dim / 8);
    if (items == 0) return hipSuccess;
    const unsigned grid = (unsigned)((items + kThreads - 1) / kThreads);
    if (c.bf16)
        hipLaunchKernelGGL((kv_read_kernel<KvBf16>), dim3(grid), dim3(kThreads), 0, s, c, slots, T, (__bf16 *)k,
                           (__bf16 *)v, blocks, n, mean);
    else
        hipLaunchKernelGGL((kv_read_kernel<KvF16>), dim3(grid), dim3(kThreads), 0, s, c, slots, T, (_Float16 *)k,
                           (_Float16 *)v, blocks, n, mean);
    return hipGetLastError();
}

}  // namespace ivf
