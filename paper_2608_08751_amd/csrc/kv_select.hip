// The blocks that a token's queries read: a score per block, then the best.
//
// For a token and key/value head, u is the sum of the group's query rows and c
// its int8 code; a block scores <c, summary> * weight. The products are exact
// integers (int8, at most 256 channels), so the ranking does not depend on how
// the sum is split, and the selection is the one of the definition whatever
// kernel forms it. Keys are the scores' bits in ascending order of uint32 (0: not
// to be chosen); the best m are found by bisecting the key range on counts of
// keys at or above a trial value, then one pass in index order writes what is
// kept.
//
// Two kernels. kv_select_one: a workgroup per token and head, 8 lanes per block
// (16 bytes of summary each, v_dot4_i32_i8), for single tokens: their time is the
// gather of the summaries, dim bytes a block. kv_select_tile: 16 tokens of one
// request share every summary through v_mfma_i32_16x16x64_i8, each wave then selects
// for its own tokens. Both keep the keys in LDS.
#include "kv.h"
#include "kv_types.h"

#include <algorithm>

namespace ivf {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Orders fp32 by uint32; every score's key is above 0 (NaN does not occur).
__device__ __forceinline__ uint32_t key_of(float score)
{
    const uint32_t u = __float_as_uint(score + 0.f);  // -0 as +0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The sum over a head's group of query rows of channel pair d, d + 1 of token t, as fp32
// with non-finite sums 0.
template <typename TT>
__device__ __forceinline__ float2 group_sum(const KvSelect &a, int64_t t, int h, int d)
{
    const typename TT::elem *q = (const typename TT::elem *)a.q.p + t * a.q.ts + (int64_t)h * a.group * a.q.hs + d;
    double s0 = 0., s1 = 0.;
    for (int g = 0; g < a.group; ++g, q += a.q.hs) {
        const uint32_t w = *(const uint32_t *)q;
        s0 += (double)TT::lo(w);
        s1 += (double)TT::hi(w);
    }
    float2 u = make_float2((float)s0, (float)s1);
    if (!(fabsf(u.x) <= 3.402823466e38f)) u.x = 0.f;
    if (!(fabsf(u.y) <= 3.402823466e38f)) u.y = 0.f;
    return u;
}

__device__ __forceinline__ int code_of(float u, float amax)
{
    return amax >= 0x1p-100f ? (int)rintf(u * (127.f / amax)) : 0;
}

__device__ __forceinline__ float wave_max(float m)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    return m;
}

// Keeps of keys[0, n) those of `forced` places and the best `want` of the others
// (key descending, index ascending) and writes their indexes, ascending, to
// out[0, count), -1 behind. forced(j): j < first or j >= tail; a key of 0 is never
// kept. One wave. keys stay as they are.
__device__ void wave_select(const uint32_t *keys, int n, int first, int tail, int want, int count, int32_t *out)
{
    const int lane = threadIdx.x & 63;
    // extent of the candidates' keys
    uint32_t lo = UINT32_MAX, hi = 0;
    for (int j = first + lane; j < tail; j += 64) {
        const uint32_t k = keys[j];
        if (k) lo = min(lo, k);
        hi = max(hi, k);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, d));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, d));
    }
    auto at_least = [&](uint32_t v) {
        int c = 0;
        for (int j0 = first; j0 < tail; j0 += 64) {
            const int j = j0 + lane;
            c += __popcll(__ballot(j < tail && keys[j] >= v));
        }
        return c;
    };
    // tau: the want-th largest key; more = 0 where there are no more than `want` keys (tau = 1: all)
    uint32_t tau = 1;
    int ties = 0;  // how many keys equal to tau are kept
    if (want <= 0) {
        tau = UINT32_MAX;
        ties = 0;
    } else if (hi == 0 || at_least(lo) <= want) {
        tau = 1;
        ties = 1 << 30;
    } else {
        // at_least(a) > want >= at_least(b)
        uint32_t a = lo, b = hi + 1;  // hi < UINT32_MAX: no key of a number is that high
        int cb = 0;
        while (b - a > 1 && cb != want) {
            const uint32_t mid = a + (b - a) / 2;
            const int c = at_least(mid);
            if (c > want) a = mid;
            else b = mid, cb = c;
        }
        if (cb == want) {
            tau = b;
            ties = 1 << 30;
        } else {
            tau = a;  // b = a + 1: cb keys are above it
            ties = want - cb;
        }
    }
    int kept = 0, used = 0;
    for (int j0 = 0; j0 < n; j0 += 64) {
        const int j = j0 + lane;
        const uint32_t k = j < n ? keys[j] : 0u;
        const bool forced = j < first || j >= tail;
        const bool eq = !forced && k == tau && want > 0;
        const uint64_t me = __ballot(eq);
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        const bool take = k != 0 && (forced || (want > 0 && k > tau) || (eq && used + __popcll(me & below) < ties));
        used += __popcll(me);
        const uint64_t mt = __ballot(take);
        const int at = kept + __popcll(mt & below);
        if (take && at < count) out[at] = j;
        kept += __popcll(mt);
    }
    for (int i = kept + lane; i < count; i += 64) out[i] = -1;
}

// How many blocks token t ranks, and which of them are kept anyway.
struct Extent {
    int b, n, first, tail, want;
};
__device__ __forceinline__ Extent extent_of(const KvSelect &a, int64_t t)
{
    Extent e;
    const int b = a.request[t], p = a.position[t];
    e.b = b;
    e.n = b < 0 || b >= a.B || p < 0 ? 0 : min((p >> a.c.shift) + 1, a.cols);
    e.first = min(a.first, e.n);
    e.tail = max(e.n - a.last, e.first);
    e.want = a.count - e.first - (e.n - e.tail);
    return e;
}

constexpr int kOneThreads = 512;

template <typename TT>
__global__ __launch_bounds__(kOneThreads) void kv_select_one_kernel(KvSelect a)
{
    extern __shared__ uint32_t lds[];  // keys [cols]
    __shared__ __align__(16) int8_t code[256];
    __shared__ float top[kOneThreads / 64];
    const int tid = threadIdx.x;
    const int h = blockIdx.x % a.c.heads;
    const int64_t t = blockIdx.x / a.c.heads;
    const Extent e = extent_of(a, t);
    int32_t *out = a.out + (t * a.c.heads + h) * a.count;
    if (e.n <= a.count) {  // all of them, but for holes in the table
        for (int j = tid; j < e.n; j += kOneThreads) {
            const int32_t id = a.table[(int64_t)e.b * a.cols + j];
            lds[j] = id >= 0 && id < a.c.blocks;
        }
    } else {
        float2 u = make_float2(0.f, 0.f);
        if (2 * tid < a.c.dim) u = group_sum<TT>(a, t, h, 2 * tid);
        const float m = wave_max(fmaxf(fabsf(u.x), fabsf(u.y)));
        if ((tid & 63) == 0) top[tid >> 6] = m;
        if (tid < 128) *(uint16_t *)&code[2 * tid] = 0;
        __syncthreads();
        const float amax = fmaxf(top[0], top[1]);  // at most 256 channels: two waves hold them
        if (2 * tid < a.c.dim) {
            code[2 * tid] = (int8_t)code_of(u.x, amax);
            code[2 * tid + 1] = (int8_t)code_of(u.y, amax);
        }
        __syncthreads();
        const int part = tid & 7;  // 16 bytes of a summary, and 16 more 128 further on
        const i32x4 q0 = *(const i32x4 *)&code[16 * part], q1 = *(const i32x4 *)&code[128 + 16 * part];
        const bool has0 = 16 * part < a.c.dim, has1 = 128 + 16 * part < a.c.dim;
        for (int j0 = 0; j0 < e.n; j0 += kOneThreads / 8) {
            const int j = j0 + (tid >> 3);
            int32_t id = -1;
            if (j < e.n) id = a.table[(int64_t)e.b * a.cols + j];
            const bool ok = id >= 0 && id < a.c.blocks;
            int s = 0;
            if (ok) {
                const int8_t *p = a.c.summary + ((int64_t)id * a.c.heads + h) * a.c.dim + 16 * part;
                if (has0) {
                    const i32x4 x = *(const i32x4 *)p;
#pragma unroll
                    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_sdot4(x[i], q0[i], s, false);
                }
                if (has1) {
                    const i32x4 x = *(const i32x4 *)(p + 128);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_sdot4(x[i], q1[i], s, false);
                }
            }
            s += __shfl_xor(s, 1);
            s += __shfl_xor(s, 2);
            s += __shfl_xor(s, 4);
            if (part == 0 && j < e.n)
                lds[j] = ok ? key_of((float)s * a.c.weight[(int64_t)id * a.c.heads + h]) : 0u;
        }
    }
    __syncthreads();
    if (tid < 64) wave_select(lds, e.n, e.first, e.tail, e.want, a.count, out);
}

constexpr int kTileTokens = 16, kTileThreads = 512;

// Dynamic LDS: keys [16][ld], ld >= cols.
template <typename TT>
__global__ __launch_bounds__(kTileThreads) void kv_select_tile_kernel(KvSelect a, int ld)
{
    extern __shared__ uint32_t lds[];
    __shared__ __align__(16) int8_t code[kTileTokens][256];
    __shared__ Extent ext[kTileTokens];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = blockIdx.x % a.c.heads;
    const int64_t t0 = (int64_t)(blockIdx.x / a.c.heads) * kTileTokens;
    const int tokens = (int)min((int64_t)kTileTokens, a.T - t0);
    if (tid < kTileTokens) {
        Extent e = {-1, 0, 0, 0, 0};
        if (tid < tokens) e = extent_of(a, t0 + tid);
        ext[tid] = e;
    }
    for (int i = tid; i < kTileTokens * 64; i += kTileThreads) ((uint32_t *)code)[i] = 0;
    __syncthreads();
    for (int i = wave; i < tokens; i += kTileThreads / 64) {
        float2 u[2];
        float m = 0.f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int d = 2 * (lane + 64 * s);
            u[s] = d < a.c.dim ? group_sum<TT>(a, t0 + i, h, d) : make_float2(0.f, 0.f);
            m = fmaxf(m, fmaxf(fabsf(u[s].x), fabsf(u[s].y)));
        }
        m = wave_max(m);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            code[i][2 * (lane + 64 * s)] = (int8_t)code_of(u[s].x, m);
            code[i][2 * (lane + 64 * s) + 1] = (int8_t)code_of(u[s].y, m);
        }
    }
    __syncthreads();
    // scores, request by request (the tokens of one follow each other)
    const int col = lane & 15, hi = lane >> 4, steps = (a.c.dim + 63) / 64;
    i32x4 qf[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[s] = *(const i32x4 *)&code[col][64 * s + 16 * hi];
    for (int i0 = 0; i0 < tokens;) {
        const int b = ext[i0].b;
        int i1 = i0, n = 0;
        for (; i1 < tokens && ext[i1].b == b; ++i1) n = max(n, ext[i1].n);
        const bool mine = col >= i0 && col < i1;
        for (int j0 = 16 * wave; j0 < n; j0 += 16 * (kTileThreads / 64)) {
            const int jr = j0 + col;  // the block that this lane loads
            int32_t id = jr < n ? a.table[(int64_t)b * a.cols + jr] : -1;
            if (id >= a.c.blocks) id = -1;
            const int8_t *p = a.c.summary + ((int64_t)max(id, 0) * a.c.heads + h) * a.c.dim + 16 * hi;
            i32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s < steps) {
                    i32x4 x = {0, 0, 0, 0};
                    if (64 * s + 16 * hi < a.c.dim) x = *(const i32x4 *)(p + 64 * s);
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, qf[s], acc, 0, 0, 0);
                }
            }
            const float w = id >= 0 ? a.c.weight[(int64_t)id * a.c.heads + h] : 0.f;
            uint32_t k[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int src = 4 * hi + r;  // the block of row src was loaded by lane src
                const float wr = __shfl(w, src);
                const int idr = __shfl(id, src);
                k[r] = idr >= 0 ? key_of((float)acc[r] * wr) : 0u;
            }
            if (mine) {
#pragma unroll
                for (int r = 0; r < 4; ++r) lds[col * ld + j0 + 4 * hi + r] = k[r];
            }
        }
        i0 = i1;
    }
    __syncthreads();
    for (int i = wave; i < tokens; i += kTileThreads / 64)
        wave_select(lds + i * ld, ext[i].n, ext[i].first, ext[i].tail, ext[i].want, a.count,
                    a.out + ((t0 + i) * a.c.heads + h) * a.count);
}

}  // namespace

hipError_t launch_kv_select(const KvSelect &a, int num_cus, hipStream_t s)
{
    const int ld = (a.cols + 15) / 16 * 16 + 4;
    const size_t tile_lds = (size_t)kTileTokens * ld * 4;
    // 16 tokens of a tile share the summaries where a batch brings more tokens than requests
    if (a.T > 2 * a.B && tile_lds <= 128 * 1024) {
        const unsigned grid = (unsigned)((a.T + kTileTokens - 1) / kTileTokens * a.c.heads);
        const void *f = a.c.bf16 ? (const void *)kv_select_tile_kernel<KvBf16> : (const void *)kv_select_tile_kernel<KvF16>;
        if (tile_lds > 48 * 1024) {
            const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)tile_lds);
            if (e != hipSuccess) return e;
        }
        if (a.c.bf16)
            hipLaunchKernelGGL((kv_select_tile_kernel<KvBf16>), dim3(grid), dim3(kTileThreads), tile_lds, s, a, ld);
        else
            hipLaunchKernelGGL((kv_select_tile_kernel<KvF16>), dim3(grid), dim3(kTileThreads), tile_lds, s, a, ld);
        return hipGetLastError();
    }
    const size_t one_lds = (size_t)a.cols * 4;
    const unsigned grid = (unsigned)(a.T * a.c.heads);
    if (one_lds > 48 * 1024) {
        const void *f = a.c.bf16 ? (const void *)kv_select_one_kernel<KvBf16> : (const void *)kv_select_one_kernel<KvF16>;
        const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)one_lds);
        if (e != hipSuccess) return e;
    }
    if (a.c.bf16)
        hipLaunchKernelGGL((kv_select_one_kernel<KvBf16>), dim3(grid), dim3(kOneThreads), one_lds, s, a);
    else
        hipLaunchKernelGGL((kv_select_one_kernel<KvF16>), dim3(grid), dim3(kOneThreads), one_lds, s, a);
    return hipGetLastError();
}

}  // namespace ivf
