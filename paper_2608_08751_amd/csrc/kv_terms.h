// What a call may put into the scores of the cache's attention: a cap, a bias that grows
// with distance, and the keys that a row sees.
//
// A row at position p sees the keys j with first <= j <= p or j < prefix. Keys that rows of
// a group see between them lie in [0, most prefix) and [least first, most p], so that a
// kernel's steps (of 32, 64 or 128 keys) are those of the two ranges one after the other,
// and what lies between is neither read nor computed.
#pragma once

#include <type_traits>

#include "kv.h"
#include "kv_types.h"

namespace ivf {

template <typename Terms> constexpr bool has_terms = !std::is_same<Terms, KvNoTerms>::value;

// Terms of a kernel of their own: with a cap or not, with a bias or not (always with sights).
template <bool CAP, bool BIAS> struct KvTermsOf : KvTerms {
    static constexpr bool kCap = CAP, kBias = BIAS;
};

// A head's slope, to the base 2. One of 2^14 leaves a key that is one further away no weight, and the biases of a step's
// 64 keys stay within 63 x 2^14 x 1.443 < 2^21, where fp32 numbers lie 2^-3 apart: the prompt kernel subtracts them in
// another order for the reference than for the probabilities, a rounding of the bias, of its sum with the score and of
// the sum with the reference, 2^-4 each (scores are small beside such biases), so that the two differ by less than a
// unit of the exponent (beyond 2^30 they would be infinite). Comparisons leave a slope that is no number as it is.
__device__ __forceinline__ float slope_of(const KvTerms &x, int head)
{
    const float s = x.slopes[head];
    return (s > 0x1p14f ? 0x1p14f : s < -0x1p14f ? -0x1p14f : s) * 1.44269504089f;
}

// The keys that a row sees; last_key: the last that its table has room for. A row that does not count or stands
// at no position sees nothing.
struct KvSight {
    int pos, first, prefix;
    static __device__ __forceinline__ KvSight of(const KvAttend &a, const KvTerms &x, int64_t t, bool counts, int last_key)
    {
        const int p = counts ? a.position[t] : -1;
        KvSight s = {min(p, last_key), 0, 0};
        if (p < 0) return {-1, 0, 0};
        if (x.first) s.first = max(x.first[t], 0);
        if (x.prefix) s.prefix = min(max(x.prefix[t], 0), last_key + 1);
        return s;
    }
    __device__ __forceinline__ bool sees(int key) const { return (key <= pos && key >= first) || key < prefix; }
};

// The same of several rows: what any of them sees, and what all do.
struct KvSights {
    int pos_max = -1, pos_min = INT32_MAX, first_min = INT32_MAX, first_max = 0, prefix_max = 0, prefix_min = INT32_MAX;
    __device__ __forceinline__ void add(const KvSight &s)
    {
        const bool window = s.first <= s.pos;  // else the row sees its prefix alone
        pos_max = max(pos_max, window ? s.pos : -1);
        pos_min = min(pos_min, window ? s.pos : -1);
        first_min = min(first_min, window ? s.first : INT32_MAX);
        first_max = max(first_max, s.first);
        prefix_max = max(prefix_max, s.prefix);
        prefix_min = min(prefix_min, s.prefix);
    }
    // over the 16 columns of a wave's lanes; the result is uniform
    __device__ __forceinline__ void join_columns()
    {
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) {
            pos_max = max(pos_max, __shfl_xor(pos_max, d));
            pos_min = min(pos_min, __shfl_xor(pos_min, d));
            first_min = min(first_min, __shfl_xor(first_min, d));
            first_max = max(first_max, __shfl_xor(first_max, d));
            prefix_max = max(prefix_max, __shfl_xor(prefix_max, d));
            prefix_min = min(prefix_min, __shfl_xor(prefix_min, d));
        }
        pos_max = __builtin_amdgcn_readfirstlane(pos_max);
        pos_min = __builtin_amdgcn_readfirstlane(pos_min);
        first_min = __builtin_amdgcn_readfirstlane(first_min);
        first_max = __builtin_amdgcn_readfirstlane(first_max);
        prefix_max = __builtin_amdgcn_readfirstlane(prefix_max);
        prefix_min = __builtin_amdgcn_readfirstlane(prefix_min);
    }
    // the last key that any row sees
    __device__ __forceinline__ int last() const { return max(pos_max, prefix_max - 1); }
    // whether any row sees one of the n keys from `key` on, and whether all rows see all of them
    __device__ __forceinline__ bool any(int key, int n) const
    {
        return key < prefix_max || (key <= pos_max && key + (n - 1) >= first_min);
    }
    __device__ __forceinline__ bool all(int key, int n) const
    {
        return (key >= first_max && key + (n - 1) <= pos_min) || key + (n - 1) < prefix_min;
    }
    // whether no row sees the key: it may be a slot that was never written
    __device__ __forceinline__ bool nobody(int key) const
    {
        return key > last() || (key >= prefix_max && key < first_min);
    }
};

// Steps of 2^SHIFT keys that cover what rows see.
struct KvSteps {
    int before, gap, count;  // steps over the prefixes; what lies between them and the rest; all
    template <int SHIFT> static __device__ __forceinline__ KvSteps of(int prefix_max, int first_min, int pos_max)
    {
        KvSteps s;
        s.before = (int)(((int64_t)prefix_max + (1 << SHIFT) - 1) >> SHIFT);
        const int from = max(s.before, first_min >> SHIFT), end = pos_max < 0 ? 0 : (pos_max >> SHIFT) + 1;
        s.gap = end > from ? from - s.before : 0;
        s.count = s.before + max(end - from, 0);
        return s;
    }
    __device__ __forceinline__ int at(int i) const { return i < before ? i : i + gap; }
};

// tanh x. Up to 1 by a polynomial in x^2 (fitted to the relative error over [0, 1]: 1.6e-7 with its roundings), beyond
// that by 1 - 2 / (1 + exp 2x), whose last subtraction costs at most a bit there (at 0 it would leave an absolute
// error of the whole cap's rounding). Up to 0.6 five terms do (1.8e-7): they come with the cap multiplied in
// (KvTerms::near), two instructions a score less.
__device__ __forceinline__ float tanh_near(float x)
{
    const float z = x * x;
    float p = 0.00104102271f;
    p = __builtin_fmaf(p, z, -0.00620337948f);
    p = __builtin_fmaf(p, z, 0.0202899817f);
    p = __builtin_fmaf(p, z, -0.0534570292f);
    p = __builtin_fmaf(p, z, 0.13325204f);
    p = __builtin_fmaf(p, z, -0.333328396f);
    p = __builtin_fmaf(p, z, 0.99999994f);
    return x * p;
}
__device__ __forceinline__ float tanh_far(float x)
{
    return 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * 2.88539008f));
}

// The N capped scores of a lane, to the base 2, from its products with the query (scale: by the cap). Which form is
// taken goes by the largest score of the wave's lanes.
template <int N> __device__ __forceinline__ void cap_scores(float (&t)[N], float scale, const KvTerms &x)
{
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(t[i]));
    if (!__ballot(most * scale > 0.6f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = t[i] * scale, z = y * y;
            float p = __builtin_fmaf(x.near[4], z, x.near[3]);
            p = __builtin_fmaf(p, z, x.near[2]);
            p = __builtin_fmaf(p, z, x.near[1]);
            t[i] = y * __builtin_fmaf(p, z, x.near[0]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] *= scale;
    if (!__ballot(most * scale > 1.f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = tanh_near(t[i]) * x.cap;
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float near = tanh_near(t[i]), far = tanh_far(t[i]);
        t[i] = (fabsf(t[i]) <= 1.f ? near : far) * x.cap;
    }
}

// Scores to the base 2, capped or scaled.
template <int N> __device__ __forceinline__ void scale_scores(float (&t)[N], float scale, const KvTerms &x)
{
    if (x.cap != 0.f) {
        cap_scores(t, scale, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] *= scale;
}

}  // namespace ivf
