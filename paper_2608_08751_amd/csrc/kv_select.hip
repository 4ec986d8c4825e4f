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
//
// 32 tokens x 8 heads over up to 1,016 blocks of 128 channels take 13 us, of which the
// scores (17 MB of summaries) are a third and the rounds of the selection the rest;
// 2,048 tokens x 8 heads over 1,000 blocks of 96 channels 55 us, bound by the selection's
// vector instructions (16,384 times the best 48 of 1,000; the products are 4 us).
#include "kv.h"
#include "kv_types.h"

#include <algorithm>
#include <type_traits>

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

// A block's weight as its score takes it. That of a block whose last slot has not been written
// may be anything: no number, or one below 0, counts 0.
__device__ __forceinline__ float weight_of(float w) { return w >= 0.f && w <= 3.402823466e38f ? w : 0.f; }

// 127 / amax, or 0 where amax is too small: code = rint(u times it).
__device__ __forceinline__ float code_scale(float amax) { return amax >= 0x1p-100f ? 127.f / amax : 0.f; }
__device__ __forceinline__ uint16_t two_codes(float2 u, float scale)
{
    const int c0 = (int)rintf(u.x * scale), c1 = (int)rintf(u.y * scale);
    return (uint16_t)((c0 & 255) | (c1 & 255) << 8);
}

__device__ __forceinline__ float wave_max(float m)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    return m;
}

// The score of a key (the inverse of key_of).
__device__ __forceinline__ float score_of(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// x summed over the wave, by lanes of a row of 16 and then over the rows.
__device__ __forceinline__ float wave_sum(float x)
{
    auto step = [&](auto ctrl) {
        constexpr int c = decltype(ctrl)::value;
        x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), c, 0xf, 0xf, true));
    };
    step(std::integral_constant<int, 0xb1>());   // quad_perm 1 0 3 2
    step(std::integral_constant<int, 0x4e>());   // quad_perm 2 3 0 1
    step(std::integral_constant<int, 0x141>());  // row_half_mirror
    step(std::integral_constant<int, 0x140>());  // row_mirror
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        s += __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 16 * r));
    return s;
}

// The point that a normal variable passes with probability p, for p up to 1/2 to 0.003
// (Abramowitz and Stegun, Handbook of Mathematical Functions, 26.2.22).
__device__ __forceinline__ float upper_quantile(float p)
{
    const float t = __builtin_amdgcn_sqrtf(-1.38629436f * __builtin_amdgcn_logf(p));  // sqrt(-2 ln p)
    return t - (0.27061f * t + 2.30753f) * __builtin_amdgcn_rcpf((0.04481f * t + 0.99229f) * t + 1.f);
}

// Sums over WAVES waves: two rows in turn, so that one barrier a sum is enough.
template <int WAVES> struct Exchange {
    uint32_t v[2][WAVES];
};
template <typename T, int WAVES>
__device__ __forceinline__ T add_rows16(T x)  // over lanes 0 ... 15, in lane 0
{
    auto step = [&](auto ctrl) {
        constexpr int c = decltype(ctrl)::value;
        x += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), c, 0xf, 0xf, true));
    };
    step(std::integral_constant<int, 0xb1>());
    step(std::integral_constant<int, 0x4e>());
    step(std::integral_constant<int, 0x141>());
    step(std::integral_constant<int, 0x140>());
    return __builtin_bit_cast(T, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}
// The sum of the waves' x (uniform in each); *before: of the waves before this one.
template <typename T, int WAVES>
__device__ __forceinline__ T sum_waves(Exchange<WAVES> &e, int &turn, int wave, T x, T *before = nullptr)
{
    static_assert(WAVES <= 16, "a lane a wave");
    if (WAVES == 1) {
        if (before) *before = 0;
        return x;
    }
    const int lane = threadIdx.x & 63;
    if (lane == 0) e.v[turn][wave] = __builtin_bit_cast(uint32_t, x);
    __syncthreads();
    const T y = lane < WAVES ? __builtin_bit_cast(T, e.v[turn][lane % WAVES]) : T(0);
    turn ^= 1;
    if (before) *before = add_rows16<T, WAVES>(lane < wave ? y : T(0));
    return add_rows16<T, WAVES>(y);
}

// `from` and the number of lanes below this one in the mask.
__device__ __forceinline__ int lanes_below(uint64_t mask, int from)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, (uint32_t)from));
}

// Keeps of keys 0 ... n - 1 those of forced places (j < first or j >= tail) and the
// best `want` of the others (key descending, index ascending), and writes their
// indexes, ascending, to out[0, count), -1 behind; a key of 0 is never kept. WAVES
// waves (all threads of the workgroup, or one wave by itself): lane l of wave w holds keys
// (w KPT + i) 64 + l in k[i], zero from n on.
template <int WAVES, int KPT>
__device__ __forceinline__ void select_best(const uint32_t (&k)[KPT], int wave, int n, int first, int tail, int want,
                                            int count, int32_t *out, Exchange<WAVES> &ex)
{
    const int lane = threadIdx.x & 63, j0 = wave * KPT * 64 + lane;
    int turn = 0;
    uint32_t c[KPT];  // keys; forced ones the largest
    float sum = 0.f, squares = 0.f, count_s = 0.f;  // of a quarter of the scores
    int forced = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        c[i] = k[i];
        const int base = (wave * KPT + i) * 64;
        if (base < first || base + 64 > tail) {  // the same for the wave: most 64 keys have no forced one
            const int j = j0 + 64 * i;
            const bool kept = (j < first || j >= tail) && k[i] != 0;
            c[i] = kept ? UINT32_MAX : k[i];
            forced += __popcll(__ballot(kept));
        }
        if (i % 4 == 0) {
            const bool sample = c[i] + 1 > 1;  // neither 0 nor forced
            const float x = sample ? score_of(k[i]) : 0.f;
            sum += x;
            squares += x * x;
            count_s += sample ? 1.f : 0.f;
        }
    }
    forced = sum_waves<int, WAVES>(ex, turn, wave, forced);
    // keys at or above v (no number's key is UINT32_MAX), the forced ones left out
    auto at_least = [&](uint32_t v) {
        int x = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) x += __popcll(__ballot(c[i] >= v));
        return sum_waves<int, WAVES>(ex, turn, wave, x) - forced;
    };
    // kept are keys at or above tau, and the first `ties` equal to tau - 1
    uint32_t tau = 1;
    int ties = 0, candidates = 0;
    if (want <= 0) {
        tau = UINT32_MAX;
    } else if ((candidates = at_least(1)) > want) {
        // The want-th largest key lies between a and b: at_least(a) > want >= at_least(b) = cb.
        // The first trial value is where a normal
        // distribution of the scores' mean and variance has `want` keys above, the next ones step away
        // from it until both sides are known, then the bracket is halved by value (by key where
        // that leaves it): for the best 45 of 1,000 normal scores 6.8 counts on average, at most 11 in 95 of
        // 100 (of 400, run on the host), where halving the keys' range takes 16.5.
        auto over_waves = [&](float x) { return sum_waves<float, WAVES>(ex, turn, wave, wave_sum(x)); };
        const float per = __builtin_amdgcn_rcpf(over_waves(count_s)), mean = over_waves(sum) * per;
        const float sigma = __builtin_amdgcn_sqrtf(fmaxf(over_waves(squares) * per - mean * mean, 0.f));
        const float share = (float)want * __builtin_amdgcn_rcpf((float)candidates);
        float trial = mean + sigma * (share <= 0.5f ? upper_quantile(share) : -upper_quantile(1.f - share));
        float step = 0.125f * sigma;
        uint32_t a = 1, b = UINT32_MAX;
        int cb = 0;
        while (b - a > 1 && cb != want) {
            uint32_t mid = (uint32_t)__builtin_amdgcn_readfirstlane((int)key_of(trial));
            if (!(mid > a && mid < b)) mid = a + (b - a) / 2;
            const int x = at_least(mid);
            if (x > want) a = mid;
            else b = mid, cb = x;
            if (a > 1 && b < UINT32_MAX) {
                trial = 0.5f * score_of(a) + 0.5f * score_of(b);
            } else {
                trial += x > want ? step : -step;
                step *= 2.f;
            }
        }
        tau = b;
        ties = want - cb;  // where more than 0, b = a + 1
    }
    uint64_t take[KPT];  // lanes whose key i is kept, in scalar registers
    int kept = 0;
    static_assert(KPT <= 32, "two scalar registers a key");
    if (ties > 0) {
        int eq = 0, used = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) eq += __popcll(__ballot(c[i] == tau - 1));
        sum_waves<int, WAVES>(ex, turn, wave, eq, &used);
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const bool same = c[i] == tau - 1;
            const uint64_t me = __ballot(same);
            take[i] = __ballot(c[i] >= tau || (same && lanes_below(me, used) < ties));
            used += __popcll(me);
            kept += __popcll(take[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            take[i] = __ballot(c[i] >= tau);
            kept += __popcll(take[i]);
        }
    }
    int at = 0;
    const int total = sum_waves<int, WAVES>(ex, turn, wave, kept, &at);
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int to = lanes_below(take[i], at);
        if (__builtin_amdgcn_inverse_ballot_w64(take[i]) && to < count) out[to] = j0 + 64 * i;
        at += __popcll(take[i]);
    }
    for (int i = total + wave * 64 + lane; i < count; i += WAVES * 64) out[i] = -1;
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

constexpr int kOneThreads = 1024, kOneWaves = kOneThreads / 64;

// KPT keys a lane of the TEAM waves that select: tables of up to 64 KPT TEAM columns. PARTS: 128
// channels each. Dynamic LDS: [cols] block ids, then keys. One wave selects among up to 2,048 keys
// (a count is three instructions for 64 keys there, and no barrier), all 16 beyond.
template <typename TT, int KPT, int PARTS, int TEAM>
__global__ __launch_bounds__(kOneThreads) void kv_select_one_kernel(KvSelect a)
{
    extern __shared__ uint32_t lds[];
    __shared__ __align__(16) int8_t code[128 * PARTS];
    __shared__ float top[PARTS];
    __shared__ Exchange<TEAM> ex;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.x % (uint32_t)a.c.heads;
    const int64_t t = blockIdx.x / (uint32_t)a.c.heads;
    float2 u = make_float2(0.f, 0.f);
    if (2 * tid < a.c.dim) u = group_sum<TT>(a, t, h, 2 * tid);
    const Extent e = extent_of(a, t);
    int32_t *out = a.out + (t * a.c.heads + h) * a.count;
    const bool ranked = e.n > a.count;
    for (int j = tid; j < e.n; j += kOneThreads) {
        int32_t id = a.table[(int64_t)e.b * a.cols + j];
        if (id >= a.c.blocks) id = -1;
        lds[j] = ranked ? (uint32_t)id : (uint32_t)(id >= 0);  // all are kept, but for holes in the table
    }
    if (ranked) {
        if (tid < 64 * PARTS) {  // the waves that hold channels
            const float m = wave_max(fmaxf(fabsf(u.x), fabsf(u.y)));
            if (lane == 0) top[wave] = m;
        }
        __syncthreads();
        if (tid < 64 * PARTS)
            *(uint16_t *)&code[2 * tid] = two_codes(u, code_scale(PARTS > 1 ? fmaxf(top[0], top[PARTS - 1]) : top[0]));
        __syncthreads();
        const int part = tid & 7;  // 16 bytes of every 128 of a summary
        i32x4 q[PARTS];
        bool has[PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            q[p] = *(const i32x4 *)&code[128 * p + 16 * part];
            has[p] = 128 * p + 16 * part < a.c.dim;
        }
        constexpr int kAhead = 8 / PARTS, kStep = kOneThreads / 8;
        for (int j0 = tid >> 3; j0 < e.n; j0 += kStep * kAhead) {
            i32x4 x[kAhead][PARTS];
            float w[kAhead];
            int32_t id[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int j = j0 + kStep * i;
                id[i] = j < e.n ? (int32_t)lds[j] : -1;
                w[i] = 0.f;
                const int64_t at = (int64_t)max(id[i], 0) * a.c.heads + h;
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    x[i][p] = (i32x4){0, 0, 0, 0};
                    if (id[i] >= 0 && has[p]) x[i][p] = *(const i32x4 *)(a.c.summary + at * a.c.dim + 128 * p + 16 * part);
                }
                if (id[i] >= 0 && part == 0) w[i] = a.c.weight[at];
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                int s = 0;
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s = __builtin_amdgcn_sdot4(x[i][p][r], q[p][r], s, false);
                s += __shfl_xor(s, 1);
                s += __shfl_xor(s, 2);
                s += __shfl_xor(s, 4);
                const int j = j0 + kStep * i;
                if (part == 0 && j < e.n) lds[j] = id[i] >= 0 ? key_of((float)s * weight_of(w[i])) : 0u;
            }
        }
    }
    __syncthreads();
    if (wave >= TEAM) return;
    uint32_t k[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int j = (wave * KPT + i) * 64 + lane;
        k[i] = j < e.n ? lds[j] : 0u;
    }
    select_best<TEAM, KPT>(k, wave, e.n, e.first, e.tail, e.want, a.count, out, ex);
}

constexpr int kTileTokens = 16, kTileThreads = 1024;  // a wave a token

// KPT keys a lane: tables of up to 64 KPT columns. Dynamic LDS: keys [16][ld], then
// block ids [ld] and weights [ld] of the request at hand, ld >= cols + 4 a multiple of 4.
template <typename TT, int KPT>
__global__ __launch_bounds__(kTileThreads) void kv_select_tile_kernel(KvSelect a, int ld)
{
    extern __shared__ uint32_t lds[];
    int32_t *ids = (int32_t *)lds + kTileTokens * ld;
    float *weights = (float *)(ids + ld);
    __shared__ __align__(16) int8_t code[kTileTokens][256];
    __shared__ Extent ext[kTileTokens];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.x % (uint32_t)a.c.heads;
    const int64_t t0 = (int64_t)(blockIdx.x / (uint32_t)a.c.heads) * kTileTokens;
    const int tokens = (int)min((int64_t)kTileTokens, a.T - t0);
    if (tid < kTileTokens) {
        Extent e = {-1, 0, 0, 0, 0};
        if (tid < tokens) e = extent_of(a, t0 + tid);
        ext[tid] = e;
    }
    // the code of a token a wave (missing ones are zero)
    {
        float2 u[2];
        float m = 0.f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int d = 2 * (lane + 64 * s);
            u[s] = d < a.c.dim && wave < tokens ? group_sum<TT>(a, t0 + wave, h, d) : make_float2(0.f, 0.f);
            m = fmaxf(m, fmaxf(fabsf(u[s].x), fabsf(u[s].y)));
        }
        const float scale = code_scale(wave_max(m));
#pragma unroll
        for (int s = 0; s < 2; ++s) *(uint16_t *)&code[wave][2 * (lane + 64 * s)] = two_codes(u[s], scale);
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
        for (int j = tid; j < (n + 15) / 16 * 16; j += kTileThreads) {
            int32_t id = j < n ? a.table[(int64_t)b * a.cols + j] : -1;
            if (id >= a.c.blocks) id = -1;
            ids[j] = max(id, 0);
            weights[j] = id >= 0 ? weight_of(a.c.weight[(int64_t)id * a.c.heads + h]) : -1.f;  // below 0: no block
        }
        __syncthreads();
        const bool mine = col >= i0 && col < i1;
        constexpr int kAhead = 4, kStep = 16 * (kTileThreads / 64);
        for (int j0 = 16 * wave; j0 < n; j0 += kStep * kAhead) {
            i32x4 acc[kAhead];
#pragma unroll
            for (int x = 0; x < kAhead; ++x) {
                acc[x] = (i32x4){0, 0, 0, 0};
                const int j = j0 + kStep * x;
                const int32_t id = j < n ? ids[j + col] : 0;
                const int8_t *p = a.c.summary + ((int64_t)id * a.c.heads + h) * a.c.dim + 16 * hi;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    if (s < steps) {
                        i32x4 y = {0, 0, 0, 0};
                        if (64 * s + 16 * hi < a.c.dim) y = *(const i32x4 *)(p + 64 * s);
                        acc[x] = __builtin_amdgcn_mfma_i32_16x16x64_i8(y, qf[s], acc[x], 0, 0, 0);
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < kAhead; ++x) {
                const int j = j0 + kStep * x + 4 * hi;  // the lane's four blocks
                if (j0 + kStep * x >= n) break;
                const f32x4 w = *(const f32x4 *)&weights[j];
                u32x4 k;
#pragma unroll
                for (int r = 0; r < 4; ++r) k[r] = w[r] >= 0.f ? key_of((float)acc[x][r] * w[r]) : 0u;
                if (mine) *(u32x4 *)&lds[col * ld + j] = k;
            }
        }
        i0 = i1;
        __syncthreads();
    }
    if (wave >= tokens) return;
    Exchange<1> ex;
    const Extent x = ext[wave];
    const auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };  // the lanes agree: scalar registers
    const Extent e = {same(x.b), same(x.n), same(x.first), same(x.tail), same(x.want)};
    uint32_t k[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const uint32_t y = lds[wave * ld + 64 * i + lane];  // past the row's end: another row, or what the launch adds
        k[i] = 64 * i + lane < e.n ? y : 0u;
    }
    select_best<1, KPT>(k, 0, e.n, e.first, e.tail, e.want, a.count, a.out + ((t0 + wave) * a.c.heads + h) * a.count, ex);
}

template <typename F, typename... A>
hipError_t launch_lds(F *f, unsigned grid, int threads, size_t lds, hipStream_t s, A... args)
{
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(f, dim3(grid), dim3(threads), lds, s, args...);
    return hipGetLastError();
}

template <typename TT, int PARTS> hipError_t launch_one(const KvSelect &a, unsigned grid, size_t lds, hipStream_t s)
{
    return a.cols <= 512    ? launch_lds(kv_select_one_kernel<TT, 8, PARTS, 1>, grid, kOneThreads, lds, s, a)
           : a.cols <= 1024 ? launch_lds(kv_select_one_kernel<TT, 16, PARTS, 1>, grid, kOneThreads, lds, s, a)
           : a.cols <= 2048 ? launch_lds(kv_select_one_kernel<TT, 32, PARTS, 1>, grid, kOneThreads, lds, s, a)
           : a.cols <= 8192 ? launch_lds(kv_select_one_kernel<TT, 8, PARTS, 16>, grid, kOneThreads, lds, s, a)
                            : launch_lds(kv_select_one_kernel<TT, 32, PARTS, 16>, grid, kOneThreads, lds, s, a);
}

template <typename TT> hipError_t launch_select(const KvSelect &a, hipStream_t s)
{
    // 16 tokens of a tile share the summaries where there are enough of them a request and the tiles fill
    // the device: 500 blocks, 8 heads x 128, one request of 64 tokens 14.9 us in tiles and 11.3 one by one, of 96
    // tokens 15.4 and 15.5, of 512 tokens 16 and 60; 32 requests of 4 tokens 26 and 19, of 8 tokens 19 and 32
    if (a.T >= 6 * a.B && a.T * a.c.heads >= 768 && a.cols <= 2048) {
        const int ld = (a.cols + 15) / 16 * 16 + 4;
        const int keys = a.cols <= 512 ? 512 : a.cols <= 1024 ? 1024 : 2048;  // that a wave reads from its row on
        const size_t lds = (size_t)std::max((kTileTokens + 2) * ld, (kTileTokens - 1) * ld + keys) * 4;
        const unsigned grid = (unsigned)((a.T + kTileTokens - 1) / kTileTokens * a.c.heads);
        return a.cols <= 512    ? launch_lds(kv_select_tile_kernel<TT, 8>, grid, kTileThreads, lds, s, a, ld)
               : a.cols <= 1024 ? launch_lds(kv_select_tile_kernel<TT, 16>, grid, kTileThreads, lds, s, a, ld)
                                : launch_lds(kv_select_tile_kernel<TT, 32>, grid, kTileThreads, lds, s, a, ld);
    }
    const size_t lds = (size_t)a.cols * 4;
    const unsigned grid = (unsigned)(a.T * a.c.heads);
    return a.c.dim <= 128 ? launch_one<TT, 1>(a, grid, lds, s) : launch_one<TT, 2>(a, grid, lds, s);
}

}  // namespace

hipError_t launch_kv_select(const KvSelect &a, hipStream_t s)
{
    // a launch holds fewer than 2^32 threads: at most this many tokens of 1,024 threads a head
    const int64_t most = (int64_t)UINT32_MAX / kOneThreads / a.c.heads / kTileTokens * kTileTokens;
    for (int64_t t = 0; t < a.T; t += most) {
        KvSelect part = a;
        part.T = a.T - t < most ? a.T - t : most;
        part.q.p = (const uint16_t *)a.q.p + t * a.q.ts;
        part.request += t;
        part.position += t;
        part.out += t * a.c.heads * a.count;
        const hipError_t e = a.c.bf16 ? launch_select<KvBf16>(part, s) : launch_select<KvF16>(part, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ivf
