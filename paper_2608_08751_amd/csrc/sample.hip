// A token for each row of logits: temperature, top-k, top-p and min-p, drawn by a given number.
//
// With the row's largest logit m the weight of logit x is w = exp((x - m) / t). All three
// limits keep a leading part of the order (x descending, index ascending): the first k;
// of these the shortest part whose weights reach top_p of theirs; of that the weights of
// at least min_p. So what is kept is given by one element, the cut, and the token is
// the first index at which the running sum of kept weights passes u times their whole.
//
// Weights are whole numbers of 2^-43 of the largest one (64 bits), from an fp64 exponential: their
// sums are exact, so that no order of additions matters (atomics included), and
// a border between two tokens, or of top_p, is off by at most 2^-43 a weight. With fp32
// sums one in some hundred draws from 128,000 tokens would take a neighbour of the right token.
#include "sample.h"

#include "ivf.h"

#include <algorithm>

namespace ivf {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kTile = kThreads * 8;      // elements of a step: eight a thread
constexpr int kSegments = ((int)kSampleMaxVocab / kTile + 2) * kWaves;  // of 512 elements, a wave's share of a step
constexpr int kBins = 2048;              // the last one holds what weighs nothing
constexpr int kList = 1024;              // elements of a bin that are put in order one by one
constexpr double kUnit = 8796093022208.0;  // 2^43

typedef unsigned long long u64;

// Numbers as unsigned ones of the same order, and back.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number_of(uint32_t o)
{
    return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
// The place of an element in the row's order: larger ones come first.
__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)order_of(x) << 32 | (uint32_t)~i; }
__device__ __forceinline__ int index_of(u64 place) { return (int)~(uint32_t)place; }

// A logit as it counts: no number as -infinity, +infinity as the largest number, -0 as 0.
__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, -INFINITY), 3.40282347e38f) + 0.f; }

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(_Float16 x) { return (float)x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

// A row of V logits, taken in groups of eight that begin at multiples of 16 bytes.
template <typename E> struct Row {
    const E *p;
    int V, pad;  // elements of the first group that lie before the row
    __device__ __forceinline__ int end() const { return V + pad; }
    // x[j]: element v + j - pad, -infinity outside the row
    __device__ __forceinline__ void load(int v, float (&x)[8]) const
    {
        const int i = v - pad;
        if (i >= 0 && i + 8 <= V) {
            union {
                uint4 w[sizeof(E) / 2];
                E e[8];
            } y;
#pragma unroll
            for (int k = 0; k < (int)sizeof(E) / 2; ++k) y.w[k] = ((const uint4 *)(p + i))[k];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = clean(widen(y.e[j]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = i + j >= 0 && i + j < V ? clean(widen(p[i + j])) : -INFINITY;
        }
    }
};

// w = 2^43 exp((x - m) / t) to the nearest whole number; 2^f by a polynomial of degree 9 in f (fitted on
// [-1/2, 1/2] with 2^0 = 1, relative error 2^-44.6).
__device__ __forceinline__ u64 weight(float x, float m, double inv_t)
{
    // -infinity with any temperature (no number with an infinite one) weighs nothing
    const double d = fmax(((double)x - (double)m) * inv_t, -60.0);
    const double n = rint(d), f = d - n;
    double r = 1.020312117214188e-07;
    r = fma(r, f, 1.325522487405178e-06);
    r = fma(r, f, 1.5252686845751567e-05);
    r = fma(r, f, 0.00015403455852473414);
    r = fma(r, f, 0.0013333558179043862);
    r = fma(r, f, 0.009618129159402536);
    r = fma(r, f, 0.055504108664760424);
    r = fma(r, f, 0.2402265069581299);
    r = fma(r, f, 0.6931471805599453);
    r = fma(r, f, 1.0);
    const double w = ldexp(r, (int)n + 43) + 4503599627370496.0;  // 2^52: rounds, the whole number in the low bits
    return (u64)__double_as_longlong(w) & 0xfffffffffffffull;
}

__device__ __forceinline__ u64 shfl_up64(u64 x, int d) { return (u64)__shfl_up((long long)x, d); }
__device__ __forceinline__ u64 wave_sum(u64 x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += (u64)__shfl_xor((long long)x, d);
    return x;
}

struct Shared {
    uint32_t count[kBins];
    u64 sum[kBins];       // weights
    u64 segment[kSegments];
    u64 list[kList], sorted[kList];
    u64 waves[kWaves];
    uint32_t cursor, bin;
    u64 cut, before, through;
    uint32_t rest;
};

// The sum of x over the threads before this one; *all: over all of them.
__device__ __forceinline__ u64 sum_before(Shared &s, u64 x, u64 *all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 up = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 y = shfl_up64(up, d);
        if (lane >= d) up += y;
    }
    __syncthreads();
    if (lane == 63) s.waves[wave] = up;
    __syncthreads();
    u64 before = up - x, total = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s.waves[w];
        total += s.waves[w];
    }
    *all = total;
    return before;
}

// Calls f(x[8], index of x[0], segment) for all of the row; indexes outside it come with -infinity.
template <typename E, typename F> __device__ __forceinline__ void for_row(const Row<E> &row, F f)
{
    const int tid = threadIdx.x;
    for (int v0 = 0; v0 < row.end(); v0 += kTile) {
        float x[8];
        row.load(v0 + 8 * tid, x);
        f(x, v0 + 8 * tid - row.pad, v0 / kTile * kWaves + (tid >> 6));
    }
}

// What a row's elements are put into bins by: the distance to the largest, in steps.
struct Binning {
    float m, per;
    __device__ __forceinline__ int operator()(float x) const { return (int)fminf((m - x) * per, (float)(kBins - 1)); }
};

// The element at which a leading part of the order ends: the first whose elements number `need`, or
// whose weights reach `need` (by_weight), which lies in `bin` (`count` and `sum` come before it).
// Writes s.cut (its place) and s.through (the weights up to it). All threads call it.
template <typename E>
__device__ void find_cut(Shared &s, const Row<E> &row, Binning bins, double inv_t, int bin, uint32_t count, u64 sum, u64 need,
                         bool by_weight)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const uint32_t n = s.count[bin];
    if (n <= kList) {
        // put the bin's elements in order, each by the number of larger ones
        if (tid == 0) s.cursor = 0;
        __syncthreads();
        for_row(row, [&](const float (&x)[8], int i, int) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (bins(x[j]) == bin && i + j >= 0 && i + j < row.V) s.list[atomicAdd(&s.cursor, 1u)] = place_of(x[j], i + j);
        });
        __syncthreads();
        u64 mine = 0;
        if (tid < (int)n) {
            mine = s.list[tid];
            int larger = 0;
            for (uint32_t j = 0; j < n; ++j) larger += s.list[j] > mine;
            s.sorted[larger] = mine;
        }
        __syncthreads();
        mine = tid < (int)n ? s.sorted[tid] : 0;
        const u64 w = tid < (int)n ? weight(number_of((uint32_t)(mine >> 32)), bins.m, inv_t) : 0;
        u64 all;
        const u64 before = sum + sum_before(s, w, &all);
        const bool here = by_weight ? before < need && before + w >= need : count + tid + 1 == need;
        if (here && tid < (int)n) {
            s.cut = mine;
            s.through = before + w;
        }
        __syncthreads();
        return;
    }
    // many elements: the cut's number eight bits at a time, then its index among equal ones
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) {
            s.list[tid] = 0;
            s.sorted[tid] = 0;
        }
        __syncthreads();
        for_row(row, [&](const float (&x)[8], int i, int) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t o = order_of(x[j]);
                if (bins(x[j]) == bin && i + j >= 0 && i + j < row.V && (shift == 24 || (o ^ prefix) >> (shift + 8) == 0)) {
                    atomicAdd(&s.list[o >> shift & 255], 1ull);
                    atomicAdd(&s.sorted[o >> shift & 255], weight(x[j], bins.m, inv_t));
                }
            }
        });
        __syncthreads();
        // digits from the largest down
        const u64 c = tid < 256 ? s.list[255 - tid] : 0;
        u64 all;
        const u64 cb = count + sum_before(s, c, &all);
        const u64 w = tid < 256 ? s.sorted[255 - tid] : 0;
        const u64 wb = sum + sum_before(s, w, &all);
        if (c && (by_weight ? wb < need && wb + w >= need : cb < need && cb + c >= need)) {
            s.cursor = 255 - tid;
            s.rest = (uint32_t)cb;
            s.before = wb;
        }
        __syncthreads();
        prefix |= s.cursor << shift;
        count = s.rest;
        sum = s.before;
        __syncthreads();
    }
    // the elements equal to it weigh the same
    const u64 w = weight(number_of(prefix), bins.m, inv_t);
    const uint32_t rank = by_weight ? (uint32_t)((need - sum + w - 1) / w) : (uint32_t)(need - count);  // from 1
    for_row(row, [&](const float (&x)[8], int i, int seg) {
        int equal = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) equal += order_of(x[j]) == prefix && i + j >= 0 && i + j < row.V;
        const u64 of_wave = wave_sum(equal);
        if (lane == 0) s.segment[seg] = of_wave;
    });
    __syncthreads();
    const int segments = (row.end() + kTile - 1) / kTile * kWaves, per = (segments + kThreads - 1) / kThreads;
    u64 mine = 0, all;
    for (int k = 0; k < per; ++k)
        if (tid * per + k < segments) mine += s.segment[tid * per + k];
    u64 at = sum_before(s, mine, &all);
    for (int k = 0; k < per; ++k)
        if (tid * per + k < segments) {
            const u64 c = s.segment[tid * per + k];
            if (at < rank && at + c >= rank) {
                s.bin = tid * per + k;
                s.before = at;
            }
            at += c;
        }
    __syncthreads();
    if (tid < 64) {
        const int v = (int)s.bin * 512 + 8 * lane;
        float x[8];
        row.load(v, x);
        int equal = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) equal += order_of(x[j]) == prefix && v - row.pad + j >= 0 && v - row.pad + j < row.V;
        u64 up = equal;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const u64 y = shfl_up64(up, d);
            if (lane >= d) up += y;
        }
        u64 n = s.before + up - equal;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (order_of(x[j]) == prefix && v - row.pad + j >= 0 && v - row.pad + j < row.V && ++n == rank) {
                s.cut = place_of(x[j], v - row.pad + j);
                s.through = sum + rank * w;
            }
    }
    __syncthreads();
}

template <typename E> __global__ __launch_bounds__(kThreads) void sample_kernel(Sample a)
{
    __shared__ Shared s;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Row<E> row;
    row.p = (const E *)a.logits + t * a.stride;
    row.V = a.V;
    row.pad = (int)((uintptr_t)row.p % 16 / sizeof(E));
    // (beyond 2^60 the range of the bins would not hold in fp32; no number stays none)
    const float given = a.temperature ? a.temperature[t] : 1.f, temp = given > 0x1p60f ? 0x1p60f : given;
    const int top_k = a.top_k ? a.top_k[t] : 0;
    const float top_p = a.top_p ? a.top_p[t] : 1.f, min_p = a.min_p ? a.min_p[t] : 0.f;
    const double inv_t = 1.4426950408889634 / (double)temp;

    // the largest logit, the first of its value, and the least finite one
    u64 top = 0;
    float least = INFINITY;
    for_row(row, [&](const float (&x)[8], int i, int) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u64 p = place_of(x[j], i + j);
            if (i + j >= 0 && i + j < row.V && p > top) top = p;
            if (x[j] > -INFINITY) least = fminf(least, x[j]);
        }
    });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        top = max(top, (u64)__shfl_xor((long long)top, d));
        least = fminf(least, __shfl_xor(least, d));
    }
    if (lane == 0) {
        s.list[wave] = top;
        s.sorted[wave] = __float_as_uint(least);
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        top = max(top, s.list[w]);
        least = fminf(least, __uint_as_float((uint32_t)s.sorted[w]));
    }
    __syncthreads();
    const float m = number_of((uint32_t)(top >> 32));
    if (m == -INFINITY || !(temp > 0.f)) {
        if (tid == 0) {
            a.token[t] = m == -INFINITY ? -1 : index_of(top);
            if (a.logprob) a.logprob[t] = m == -INFINITY ? -INFINITY : 0.f;
        }
        return;
    }

    u64 cut = 0;  // what is kept has this place or a larger one
    const bool by_k = top_k > 0 && top_k < a.V, by_p = top_p < 1.f;
    if (by_k || by_p) {
        Binning bins;
        bins.m = m;
        // beyond 31 temperatures a weight is below 2^-44
        bins.per = ((float)(kBins - 1) - 0.5f) / fmaxf(fminf(m - least, 31.f * temp), 1e-30f);
        for (int b = tid; b < kBins; b += kThreads) {
            s.count[b] = 0;
            s.sum[b] = 0;
        }
        __syncthreads();
        for_row(row, [&](const float (&x)[8], int i, int) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int b = bins(x[j]);
                if (b < kBins - 1) {
                    atomicAdd(&s.count[b], 1u);
                    if (by_p) atomicAdd(&s.sum[b], weight(x[j], m, inv_t));
                }
            }
        });
        __syncthreads();
        uint32_t c[kBins / kThreads];
        u64 w[kBins / kThreads], cs = 0, ws = 0, call, wall;
#pragma unroll
        for (int k = 0; k < kBins / kThreads; ++k) {
            c[k] = s.count[tid * (kBins / kThreads) + k];
            w[k] = s.sum[tid * (kBins / kThreads) + k];
            cs += c[k];
            ws += w[k];
        }
        const u64 cb = sum_before(s, cs, &call), wb = sum_before(s, ws, &wall);
        // the bin where a leading part ends that has `need` elements, or weights
        auto bin_of = [&](u64 need, bool by_weight) {
            u64 cn = cb, wn = wb;
#pragma unroll
            for (int k = 0; k < kBins / kThreads; ++k) {
                if (by_weight ? wn < need && wn + w[k] >= need : cn < need && cn + c[k] >= need) {
                    s.bin = tid * (kBins / kThreads) + k;
                    s.rest = (uint32_t)cn;
                    s.before = wn;
                }
                cn += c[k];
                wn += w[k];
            }
            __syncthreads();
        };
        u64 whole = wall;  // weights of the first top_k
        if (by_k && (u64)top_k <= call) {
            bin_of((u64)top_k, false);
            find_cut(s, row, bins, inv_t, (int)s.bin, s.rest, s.before, (u64)top_k, false);
            cut = s.cut;
            whole = s.through;
            __syncthreads();
        }
        if (by_p) {
            const u64 need = max((u64)1, (u64)ceil((double)fmaxf(top_p, 0.f) * (double)whole));
            bin_of(need, true);
            find_cut(s, row, bins, inv_t, (int)s.bin, s.rest, s.before, need, true);
            cut = max(cut, s.cut);
            __syncthreads();
        }
    }

    // kept weights, segment by segment
    const double least_w = (double)fminf(fmaxf(min_p, 0.f), 1.f) * kUnit;
    auto kept = [&](float x, int i) -> u64 {
        if (i < 0 || i >= row.V || x == -INFINITY || place_of(x, i) < cut) return 0;
        const u64 w = weight(x, m, inv_t);
        return (double)w >= least_w ? w : 0;
    };
    for_row(row, [&](const float (&x)[8], int i, int seg) {
        u64 sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += kept(x[j], i + j);
        sum = wave_sum(sum);
        if (lane == 0) s.segment[seg] = sum;
    });
    __syncthreads();
    const int segments = (row.end() + kTile - 1) / kTile * kWaves, per = (segments + kThreads - 1) / kThreads;
    u64 mine = 0, whole;
    for (int k = 0; k < per; ++k)
        if (tid * per + k < segments) mine += s.segment[tid * per + k];
    u64 at = sum_before(s, mine, &whole);
    const float u = fmaxf(a.uniform[t], 0.f);
    const u64 goal = u < 1.f ? min((u64)((double)u * (double)whole), whole - 1) : whole - 1;  // the first running sum above it
    for (int k = 0; k < per; ++k)
        if (tid * per + k < segments) {
            const u64 x = s.segment[tid * per + k];
            if (at <= goal && at + x > goal) {
                s.bin = tid * per + k;
                s.before = at;
            }
            at += x;
        }
    __syncthreads();
    if (wave == 0) {
        const int v = (int)s.bin * 512 + 8 * lane, i = v - row.pad;
        float x[8];
        row.load(v, x);
        u64 sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += kept(x[j], i + j);
        u64 up = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const u64 y = shfl_up64(up, d);
            if (lane >= d) up += y;
        }
        u64 running = s.before + up - sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u64 w = kept(x[j], i + j);
            if (running <= goal && running + w > goal) {
                a.token[t] = i + j;
                if (a.logprob)
                    a.logprob[t] = (float)(((double)x[j] - (double)m) * inv_t * 0.6931471805599453 - log((double)whole / kUnit));
            }
            running += w;
        }
    }
}

}  // namespace

hipError_t launch_sample(const Sample &a, hipStream_t s)
{
    const dim3 grid((unsigned)a.T), block(kThreads);
    if (a.dt == IVF_F32) hipLaunchKernelGGL((sample_kernel<float>), grid, block, 0, s, a);
    else if (a.dt == IVF_F16) hipLaunchKernelGGL((sample_kernel<_Float16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((sample_kernel<__bf16>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace ivf
