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
//
// A row is gone over two to four times (from the caches after the first):
//   ends     the largest and the least logit;
//   bins     with top_k or top_p: numbers and weights of 2,048 bins by distance to the largest
//            (of 31 temperatures at most), from which follows the bin in which the kept part ends;
//   collect  the elements of the bins up to it, where they are few, which are then put in order
//            and drawn from in LDS; else those of that bin alone, with the sums of all before it;
//   draw     the range of the row that the running sum ends in, once more.
// Rows without top_k and top_p take their weights' sums, range by range, in place of bins and collect.
//
// One workgroup takes a row in one launch, or up to eight share it in four. Bound, where weights are needed, by the
// fp64 exponential's instructions: 250 whole rows of 100,003 in f16 (50 MB) 39 us, vector units 73 % busy, a pass over
// them by itself 11; 64 rows of 128,000 in bf16, limits mixed, 53 us (ends 4.9, bins 14.6, collect 18.9, draw 16.3): a
// workgroup of 32,000 elements a CU, in rounds that wait for LDS, barriers and the caches. One row of 32,000: 29 us, four
// launches; of 1,000: 14, in one. Rows that take the largest logit: 64 of 128,000 16 us, 250 of 100,003 20. With top_k of
// 40,000 and top_p, which end in a bin of more elements than a list holds, one row of 128,000 takes 234 us and 64 take 219: draw's
// one workgroup a row goes over it some ten times (top_p alone 40 and 57).
#include "sample.h"

#include "ivf.h"

#include <algorithm>

namespace ivf {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;              // the last one holds what weighs nothing
constexpr int kList = kSampleList;       // elements that are put in order in LDS
constexpr int kTile = kThreads * 8;
constexpr int kSegments = ((int)kSampleMaxVocab / kTile + 2) * kWaves;  // of 512 elements, a wave's share of a tile
constexpr double kUnit = 8796093022208.0;  // 2^43

typedef unsigned long long u64;

// Numbers as unsigned ones of the same order (0 and -0 as one), and back.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number_of(uint32_t o)
{
    return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
// The place of an element in the row's order: larger ones come first.
__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)order_of(x) << 32 | (uint32_t)~i; }
__device__ __forceinline__ int index_of(u64 place) { return (int)~(uint32_t)place; }

constexpr float kLargest = 3.40282347e38f;  // what +infinity counts as

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(_Float16 x) { return (float)x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

// The larger of a number and a logit; a logit that is no number is passed over (by a comparison: the maximum
// instruction passes on a signaling NaN).
__device__ __forceinline__ float larger(float most, float x) { return x > most ? x : most; }

// A logit that is no number has no weight and no bin but the last as it is: d and the bin's number below, which
// differences have quieted, are kept in range by maximum and minimum. +infinity, which would make differences of no kind, is
// replaced, in rows whose largest logit it is.
//
// A row of V logits, taken in groups of eight that begin at multiples of 16 bytes. A range is the groups that one
// wave goes over, `per` of them; a row has parts * kWaves ranges.
template <typename E> struct Row {
    const E *p;
    int V, pad;  // elements of the first group that lie before the row
    int per, parts;
    bool infinite = false;  // whether there is +infinity
    __device__ __forceinline__ Row(const Sample &a, int64_t t)
    {
        p = (const E *)a.logits + t * a.stride;
        V = a.V;
        pad = (int)((uintptr_t)p % 16 / sizeof(E));
        per = a.per;
        parts = a.parts;
    }
    __device__ __forceinline__ int groups() const { return (V + pad + 7) >> 3; }
    __device__ __forceinline__ int first_of(int g) const { return 8 * g - pad; }
    __device__ __forceinline__ int range_of(int i) const { return ((i + pad) >> 3) / per; }
    // Eight elements as they lie in memory.
    struct Group {
        uint4 w[sizeof(E) / 2];
        __device__ __forceinline__ void to(float (&x)[8], bool infinite) const
        {
            typedef E E8 __attribute__((ext_vector_type(8)));
            const E8 y = __builtin_bit_cast(E8, *this);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = widen((E)y[j]);
            if (infinite) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = x[j] == INFINITY ? kLargest : x[j];
            }
        }
    };
    // group g, -infinity outside the row and from group `end` on
    __device__ __forceinline__ Group load(int g, int end) const
    {
        Group y;
        const int i = first_of(g);
        if (g < end && i >= 0 && i + 8 <= V) {
#pragma unroll
            for (int k = 0; k < (int)sizeof(E) / 2; ++k) y.w[k] = ((const uint4 *)(p + i))[k];
        } else {
            typedef E E8 __attribute__((ext_vector_type(8)));
            E8 z;
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = g < end && i + j >= 0 && i + j < V ? p[i + j] : (E)-INFINITY;
            y = __builtin_bit_cast(Group, z);
        }
        return y;
    }
    // Calls f(x[8], index of x[0]) for the groups of range r, all lanes each time (-infinity past its end). Four
    // groups a lane are loaded at a time: a wave alone waits for each otherwise.
    template <typename F> __device__ __forceinline__ void for_range(int r, F f) const
    {
        constexpr int U = 4;
        const int lane = threadIdx.x & 63, end = min((r + 1) * per, groups());
        for (int g = r * per; g < end; g += 64 * U) {
            Group y[U];
#pragma unroll
            for (int k = 0; k < U; ++k) y[k] = load(g + 64 * k + lane, end);
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (g + 64 * k < end) {
                    float x[8];
                    y[k].to(x, infinite);
                    f(x, first_of(g + 64 * k + lane));
                }
            }
        }
    }
};

// w = 2^43 exp((x - m) / t) to the nearest whole number; 2^f by a polynomial of degree 9 in f (fitted on
// [-1/2, 1/2] with 2^0 = 1, relative error 2^-44.6). -infinity weighs nothing. Bound by its instructions: 22 and some
// ten around it, 16 of them in fp64, for each logit. The coefficients are kept in scalar registers: in vector
// registers each addition would first copy its own (16 instructions; 250 rows of 100,003 without limits 47 us, so 42).
struct Coefficients {
    double c[8];
    __device__ __forceinline__ Coefficients()
    {
        const double k[8] = {1.325522487405178e-06,  1.5252686845751567e-05, 0.00015403455852473414, 0.0013333558179043862,
                             0.009618129159402536,   0.055504108664760424,   0.2402265069581299,     0.6931471805599453};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = k[i];
            asm("" : "+s"(c[i]));
        }
    }
};
__device__ __forceinline__ u64 weight(float x, double m, double inv_t, const Coefficients &k)
{
    constexpr double kRound = 6755399441055744.0;  // 1.5 2^52: the sum's low bits are the nearest whole number
    const double d = fmax(((double)x - m) * inv_t, -60.0);
    const double n = d + kRound, f = d - (n - kRound);
    double r = 1.020312117214188e-07;
#pragma unroll
    for (int i = 0; i < 8; ++i) r = fma(r, f, k.c[i]);
    r = fma(r, f, 1.0);
    // times 2^(n + 43) in the exponent; + 2^52 rounds
    const u64 b = (u64)__double_as_longlong(r) + ((u64)(uint32_t)((int)__double_as_longlong(n) + 43) << 52);
    return (u64)__double_as_longlong(__longlong_as_double((long long)b) + 4503599627370496.0) & 0xfffffffffffffull;
}

// Lane exchanges without LDS: x of the lane that CTRL names in the rows of MASK, 0 where there is none.
template <int CTRL, int MASK> __device__ __forceinline__ u64 moved(u64 x)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, MASK, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, MASK, 0xf, false);
    return (u64)hi << 32 | lo;
}
// The sum of x over this lane and those before it in its row of 16.
__device__ __forceinline__ u64 row_scan(u64 x)
{
    x += moved<0x111, 0xf>(x);  // one lane up, two, four, eight
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    return x + moved<0x118, 0xf>(x);
}
// ... in the wave.
__device__ __forceinline__ u64 wave_scan(u64 x)
{
    x = row_scan(x);
    x += moved<0x142, 0xa>(x);         // the last lane of rows 0 and 2 to rows 1 and 3
    return x + moved<0x143, 0xc>(x);   // lane 31 to rows 2 and 3
}
__device__ __forceinline__ u64 of_lane(u64 x, int lane)
{
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}
__device__ __forceinline__ u64 wave_sum(u64 x) { return of_lane(wave_scan(x), 63); }

// How the kept part of a row ends: nowhere; in a bin that is listed with all bins before it; in one that is listed
// alone; or in one of more elements than a list holds.
enum Mode { kWhole, kFew, kInBin, kMany };

struct Shared {
    uint32_t count[kBins];
    u64 sum[kBins];          // weights
    u64 list[kList];         // places
    u64 segment[kSegments];  // or, of a list, indexes and weights
    u64 range[kSampleMaxParts * kWaves];
    u64 waves[kWaves];
    float low[kWaves], high[kWaves];
    // the bin where a leading part ends, and what comes before it
    int bin;
    uint32_t rest;
    u64 before;
    uint32_t cursor[2];  // of the list: elements of the bins before (from its front on) and of the bin (from its end back)
    uint32_t at[2];
    u64 cut, through;
    int found;
};

// What `decide` finds, for the launch that draws.
struct Decision {
    int mode, bin;
    uint32_t rest;
    int k_cuts;
    u64 before, all_w;
};

// The sum of x over the threads before this one; *all: over all of them.
__device__ __forceinline__ u64 sum_before(Shared &s, u64 x, u64 *all)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u64 up = wave_scan(x);
    __syncthreads();
    if (lane == 63) s.waves[wave] = up;
    __syncthreads();
    const u64 waves = row_scan(s.waves[lane % kWaves]);
    *all = of_lane(waves, kWaves - 1);
    return up - x + (wave ? of_lane(waves, wave - 1) : 0);
}

// What a row asks for, with its largest and least logit.
struct Limits {
    float m;
    double md, inv_t;
    float per;  // bins a unit of distance to the largest
    bool none, greedy, by_k, by_p;
    int top_k;
    float top_p;
    u64 least_w;  // of what min_p keeps
    // (beyond 2^60 the range of the bins would not hold in fp32; no number stays none)
    static __device__ __forceinline__ float temperature_of(const Sample &a, int64_t t)
    {
        const float given = a.temperature ? a.temperature[t] : 1.f;
        return given > 0x1p60f ? 0x1p60f : given;
    }
    __device__ __forceinline__ Limits(const Sample &a, int64_t t, float high, float low)
        : m(fminf(high, kLargest)), md((double)fminf(high, kLargest)), inv_t(1.4426950408889634 / (double)temperature_of(a, t))
    {
        const float temp = temperature_of(a, t);
        none = high == -INFINITY;
        greedy = !(temp > 0.f);
        // beyond 31 temperatures a weight is below 2^-44
        per = ((float)(kBins - 1) - 0.5f) / fmaxf(fminf(m - low, 31.f * temp), 1e-30f);
        top_k = a.top_k ? a.top_k[t] : 0;
        top_p = a.top_p ? a.top_p[t] : 1.f;
        by_k = top_k > 0 && top_k < a.V;
        by_p = top_p < 1.f;
        least_w = a.min_p ? (u64)ceil((double)fminf(fmaxf(a.min_p[t], 0.f), 1.f) * kUnit) : 0;
    }
    __device__ __forceinline__ bool cuts() const { return !none && !greedy && (by_k || by_p); }
    __device__ __forceinline__ int bin(float x) const { return (int)fminf((m - x) * per, (float)(kBins - 1)); }
    __device__ __forceinline__ u64 weigh(float x, const Coefficients &k = Coefficients()) const { return weight(x, md, inv_t, k); }
    // the weight of an element that is kept, else 0
    __device__ __forceinline__ u64 kept(float x, int i, u64 cut, const Coefficients &k = Coefficients()) const
    {
        if (cut && place_of(x, i) < cut) return 0;
        const u64 w = weigh(x, k);
        if (!least_w) return w;  // uniform over the workgroup
        return w >= least_w ? w : 0;
    }
    // the weights that top_p of `whole` asks for
    __device__ __forceinline__ u64 need(u64 whole) const
    {
        return max((u64)1, (u64)ceil((double)fmaxf(top_p, 0.f) * (double)whole));
    }
};

// The largest and the least logit of a part (16 ranges), the least of those above -infinity; all threads get them.
template <typename E> __device__ __forceinline__ float2 ends_of(Shared &s, const Row<E> &row, int part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float high = -INFINITY, low = INFINITY;
    row.for_range(part * kWaves + wave, [&](const float (&x)[8], int) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            high = larger(high, x[j]);
            low = fminf(low, x[j] > -INFINITY ? x[j] : INFINITY);
        }
    });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        high = fmaxf(high, __shfl_xor(high, d));
        low = fminf(low, __shfl_xor(low, d));
    }
    if (lane == 0) {
        s.low[wave] = low;
        s.high[wave] = high;
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        high = fmaxf(high, s.high[w]);
        low = fminf(low, s.low[w]);
    }
    return make_float2(high, low);
}

// The lowest index of the part at which the largest logit stands; thread 0 gets it.
template <typename E> __device__ __forceinline__ int first_of(Shared &s, const Row<E> &row, float m, int part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int first = INT32_MAX;
    row.for_range(part * kWaves + wave, [&](const float (&x)[8], int i) {
#pragma unroll
        for (int j = 7; j >= 0; --j)
            if (x[j] == m) first = min(first, i + j);
    });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) first = min(first, __shfl_xor(first, d));
    if (lane == 0) s.waves[wave] = (u64)first;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) first = min(first, (int)s.waves[w]);
    return first;
}

// Kept weights of range r (a wave): of all of it, of bins before `bin`, or from the cut on.
enum Part { kAll, kBefore, kFromCut };
template <Part PART, typename E> __device__ __forceinline__ u64 sum_of(const Row<E> &row, const Limits &l, int r, u64 cut, int bin)
{
    const Coefficients k;
    u64 sum = 0;
    row.for_range(r, [&](const float (&x)[8], int i) {
        if (PART != kAll) {
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) most = larger(most, x[j]);
            if (!__any(PART == kBefore ? l.bin(most) < bin : order_of(most) >= (uint32_t)(cut >> 32))) return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u64 w = l.kept(x[j], i + j, PART == kFromCut ? cut : 0, k);
            if (PART != kBefore || l.bin(x[j]) < bin) sum += w;
        }
    });
    return wave_sum(sum);
}

// Numbers and weights of the part's bins, in LDS.
template <typename E> __device__ __forceinline__ void fill_bins(Shared &s, const Row<E> &row, const Limits &l, int part)
{
    const int tid = threadIdx.x;
    for (int b = tid; b < kBins; b += kThreads) {
        s.count[b] = 0;
        s.sum[b] = 0;
    }
    __syncthreads();
    const Coefficients k;
    row.for_range(part * kWaves + (tid >> 6), [&](const float (&x)[8], int) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int b = l.bin(x[j]);
            if (b < kBins - 1) {
                atomicAdd(&s.count[b], 1u);
                if (l.by_p) atomicAdd(&s.sum[b], l.weigh(x[j], k));
            }
        }
    });
    __syncthreads();
}

// The bin where a leading part ends that has `need` elements, or weights: s.bin, and what comes before it, s.rest and
// s.before. c, w: two bins of this thread, cn, wn: what comes before them.
struct Scan {
    uint32_t c[kBins / kThreads];
    u64 w[kBins / kThreads], cn, wn, all_c, all_w;
    __device__ __forceinline__ explicit Scan(Shared &s)
    {
        u64 cs = 0, ws = 0;
#pragma unroll
        for (int k = 0; k < kBins / kThreads; ++k) {
            c[k] = s.count[threadIdx.x * (kBins / kThreads) + k];
            w[k] = s.sum[threadIdx.x * (kBins / kThreads) + k];
            cs += c[k];
            ws += w[k];
        }
        cn = sum_before(s, cs, &all_c);
        wn = sum_before(s, ws, &all_w);
    }
    __device__ __forceinline__ void find(Shared &s, u64 need, bool by_weight) const
    {
        u64 a = cn, b = wn;
#pragma unroll
        for (int k = 0; k < kBins / kThreads; ++k) {
            if (by_weight ? b < need && b + w[k] >= need : a < need && a + c[k] >= need) {
                s.bin = threadIdx.x * (kBins / kThreads) + k;
                s.rest = (uint32_t)a;
                s.before = b;
            }
            a += c[k];
            b += w[k];
        }
        __syncthreads();
    }
};

// Where the kept part ends (without min_p), from the row's bins in LDS. All threads get it; s.bin, s.rest and s.before
// hold what it says too.
__device__ __forceinline__ Decision decide(Shared &s, const Limits &l, const Scan &scan)
{
    Decision d;
    // (where top_k leaves out only what weighs nothing it cuts nothing)
    d.k_cuts = l.by_k && (u64)l.top_k <= scan.all_c;
    d.all_w = scan.all_w;
    if (!d.k_cuts && !l.by_p) {
        d.mode = kWhole;
        d.bin = kBins - 1;
        d.rest = 0;
        d.before = 0;
        return d;
    }
    if (d.k_cuts) scan.find(s, (u64)l.top_k, false);
    else scan.find(s, l.need(scan.all_w), true);
    d.bin = s.bin;
    d.rest = s.rest;
    d.before = s.before;
    const uint32_t here = s.count[d.bin];
    // (with both, top_p goes by what top_k leaves)
    d.mode = d.rest + here <= kList ? kFew : !(d.k_cuts && l.by_p) && here <= kList ? kInBin : kMany;
    return d;
}

// The part's elements of bin `last` in no order, in s.list (what would not find room is left out); and of the bins before
// it the elements too (FEW), or the wave's sum of kept weights. All threads call it.
template <bool FEW, typename E>
__device__ __forceinline__ u64 collect(Shared &s, const Row<E> &row, const Limits &l, int part, int last)
{
    if (threadIdx.x < 2) s.cursor[threadIdx.x] = 0;
    __syncthreads();
    const Coefficients c;
    u64 sum = 0;
    row.for_range(part * kWaves + (threadIdx.x >> 6), [&](const float (&x)[8], int i) {
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = larger(most, x[j]);
        if (!__any(l.bin(most) <= last)) return;
        uint32_t hits[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int b = l.bin(x[j]);
            if (FEW) hits[0] |= (uint32_t)(b < last) << j;
            hits[1] |= (uint32_t)(b == last) << j;
            if (!FEW) {
                const u64 w = l.kept(x[j], i + j, 0, c);
                if (b < last) sum += w;
            }
        }
#pragma unroll
        for (int h = FEW ? 0 : 1; h < 2; ++h) {
            if (!hits[h]) continue;
            uint32_t at = atomicAdd(&s.cursor[h], (uint32_t)__popc(hits[h]));
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (hits[h] >> j & 1) {
                    if (at < kList) s.list[h ? kList - 1 - at : at] = place_of(x[j], i + j);
                    ++at;
                }
        }
    });
    return FEW ? 0 : wave_sum(sum);
}

// Sorts list[0, n), descending, in LDS; up to the next power of two it is filled with zeros. Strides of up to 64
// stay inside what a wave holds.
__device__ __forceinline__ void sort_list(u64 *list, int n)
{
    const int tid = threadIdx.x;
    __syncthreads();
    if (n <= 128) {
        // each by the number of larger ones (equal ones by their position)
        const u64 mine = tid < n ? list[tid] : 0;
        int larger = 0;
        if (tid < n)
            for (int e = 0; e < n; ++e) {
                const u64 other = list[e];
                larger += other > mine || (other == mine && e < tid);
            }
        __syncthreads();
        if (tid < n) list[larger] = mine;
        __syncthreads();
        return;
    }
    int m = 256;
    while (m < n) m <<= 1;
    for (int i = n + tid; i < m; i += kThreads) list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= m; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            if (tid < m / 2) {
                const int i = 2 * tid - (tid & (j - 1));
                const u64 a = list[i], b = list[i + j];
                if ((a < b) == ((i & k) == 0)) {
                    list[i] = b;
                    list[i + j] = a;
                }
            }
            if (j > 64 || (j == 1 && k >= 128)) {  // else a wave's own
                __syncthreads();
            } else {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
    __syncthreads();
}

// Finds the token whose running sum passes `goal` among w[N], in the order of threads and of N: called
// with the sum before this thread's.
template <int N>
__device__ __forceinline__ void pick(Shared &s, const Sample &a, const Limits &l, int64_t t, u64 running, u64 goal, u64 whole,
                                     const u64 (&w)[N], const float (&x)[N], const int (&index)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (running <= goal && running + w[j] > goal) {
            a.token[t] = index[j];
            if (a.logprob)
                a.logprob[t] = (float)(((double)x[j] - l.md) * l.inv_t * 0.6931471805599453 - log((double)whole / kUnit));
        }
        running += w[j];
    }
}

// The running sum that the row's number asks for: the first above it is the token's.
__device__ __forceinline__ u64 goal_of(const Sample &a, int64_t t, u64 whole)
{
    const float u = fmaxf(a.uniform[t], 0.f);
    return u < 1.f ? min((u64)((double)u * (double)whole), whole - 1) : whole - 1;
}

// The element of s.segment[0, n) (places, any order; put in order here) at which a leading part ends: the
// rank-th (from 1), or with rank 0 the first whose weights, on top of `before`, reach `need`. Writes s.cut (its place) and
// s.through (the weights up to it).
__device__ __forceinline__ void cut_listed(Shared &s, const Limits &l, int n, uint32_t rank, u64 before, u64 need)
{
    const int tid = threadIdx.x;
    sort_list(s.segment, n);
    u64 place[2], w[2], all;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        place[k] = 2 * tid + k < n ? s.segment[2 * tid + k] : 0;
        w[k] = place[k] ? l.weigh(number_of((uint32_t)(place[k] >> 32))) : 0;
    }
    before += sum_before(s, w[0] + w[1], &all);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (place[k] && (rank ? 2 * tid + k + 1 == (int)rank : before < need && before + w[k] >= need)) {
            s.cut = place[k];
            s.through = before + w[k];
        }
        before += w[k];
    }
    __syncthreads();
}

// The place of the last element that is kept (min_p apart), with what `decide` asks for in the list; n: the
// list's elements of the bins before the last one, m: of that one.
__device__ __forceinline__ u64 last_kept(Shared &s, const Limits &l, const Decision &d, int n, int m)
{
    const int tid = threadIdx.x;
    for (int i = tid; i < m; i += kThreads) s.segment[i] = s.list[kList - 1 - i];
    __syncthreads();
    if (!d.k_cuts) {
        cut_listed(s, l, m, 0, d.before, l.need(d.all_w));
        return s.cut;
    }
    cut_listed(s, l, m, (uint32_t)l.top_k - d.rest, d.before, 0);
    u64 cut = s.cut;
    if (!l.by_p) return cut;
    // top_p of what top_k leaves: in the same bin or in one before it
    const u64 need = l.need(s.through);
    __syncthreads();
    if (need > d.before) {
        cut_listed(s, l, m, 0, d.before, need);
    } else {
        // (all their elements are listed)
        for (int b = tid; b < kBins; b += kThreads) {
            s.count[b] = 0;
            s.sum[b] = 0;
        }
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
            const float x = number_of((uint32_t)(s.list[i] >> 32));
            atomicAdd(&s.count[l.bin(x)], 1u);
            atomicAdd(&s.sum[l.bin(x)], l.weigh(x));
        }
        __syncthreads();
        Scan(s).find(s, need, true);
        const int bin = s.bin;
        const u64 before = s.before;
        if (tid == 0) s.found = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
            const u64 p = s.list[i];
            if (l.bin(number_of((uint32_t)(p >> 32))) == bin) s.segment[atomicAdd(&s.found, 1)] = p;
        }
        __syncthreads();
        cut_listed(s, l, s.found, 0, before, need);
    }
    return max(cut, s.cut);
}

// kFew: the token from the list alone. Weights are summed in up to 2,048 buckets of neighbouring indexes; the
// elements of the one where the running sum passes the goal are put in order.
template <typename E>
__device__ __forceinline__ void draw_listed(Shared &s, const Sample &a, const Row<E> &row, const Limits &l, int64_t t, int n, int m, u64 cut)
{
    const int tid = threadIdx.x;
    int shift = 0;
    while (a.V - 1 >> shift >= kBins) ++shift;
    const bool few = n + m <= 128;  // all in order at once: no buckets
    if (!few)
        for (int b = tid; b < kBins; b += kThreads) s.sum[b] = 0;
    if (tid == 0) s.found = 0;
    __syncthreads();
    u64 w[2], whole, goal;
    int bucket[2];
    uint32_t index[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int e = tid + k * kThreads;
        const bool there = e < n || e >= kList - m;
        const u64 place = there ? s.list[e] : 0;
        index[k] = (uint32_t)index_of(place);
        w[k] = there ? l.kept(number_of((uint32_t)(place >> 32)), (int)index[k], cut) : 0;
        bucket[k] = w[k] ? few ? 0 : (int)(index[k] >> shift) : -1;
        if (!few && w[k]) atomicAdd(&s.sum[bucket[k]], w[k]);
    }
    if (few) {
        if (tid == 0) {
            s.bin = 0;
            s.before = 0;
        }
    } else {
        __syncthreads();
        const u64 x0 = s.sum[2 * tid], x1 = s.sum[2 * tid + 1];
        const u64 at = sum_before(s, x0 + x1, &whole);
        goal = goal_of(a, t, whole);
        if (at <= goal && at + x0 + x1 > goal) {
            const bool second = at + x0 <= goal;
            s.bin = 2 * tid + second;
            s.before = second ? at + x0 : at;
        }
    }
    __syncthreads();
    // a weight takes 44 bits, an index 20; the lowest index first
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (bucket[k] == s.bin) s.segment[atomicAdd(&s.found, 1)] = (u64)(uint32_t)(kSampleMaxVocab - 1 - index[k]) << 44 | w[k];
    __syncthreads();
    const int found = s.found;
    sort_list(s.segment, found);
    float x[2];
    int i[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const u64 e = 2 * tid + k < found ? s.segment[2 * tid + k] : 0;
        w[k] = e & 0xfffffffffffull;
        i[k] = w[k] ? (int)(kSampleMaxVocab - 1) - (int)(e >> 44) : 0;  // (no entry: weighs nothing)
    }
    u64 all;
    const u64 running = s.before + sum_before(s, w[0] + w[1], &all);
    if (few) {
        whole = all;
        goal = goal_of(a, t, whole);
    }
    if (running <= goal && running + w[0] + w[1] > goal) {
#pragma unroll
        for (int k = 0; k < 2; ++k) x[k] = fminf(widen(row.p[i[k]]), kLargest);
        pick(s, a, l, t, running, goal, whole, w, x, i);
    }
}

// The token from the ranges' kept weights (s.range): the range where the running sum passes the goal, once more.
template <typename E> __device__ __forceinline__ void draw_ranges(Shared &s, const Sample &a, const Row<E> &row, const Limits &l, int64_t t, u64 cut)
{
    const int tid = threadIdx.x, ranges = row.parts * kWaves;
    u64 whole, x = tid < ranges ? s.range[tid] : 0;
    const u64 at = sum_before(s, x, &whole);
    const u64 goal = goal_of(a, t, whole);
    if (at <= goal && at + x > goal) {
        s.bin = tid;
        s.before = at;
    }
    __syncthreads();
    u64 base = s.before;
    const int end = min((s.bin + 1) * row.per, row.groups());
    for (int g0 = s.bin * row.per; g0 < end; g0 += kThreads) {
        float y[8];
        int index[8];
        u64 w[8], sum = 0, all;
        row.load(g0 + tid, end).to(y, row.infinite);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            index[j] = row.first_of(g0 + tid) + j;
            w[j] = l.kept(y[j], index[j], cut);
            sum += w[j];
        }
        const u64 before = base + sum_before(s, sum, &all);
        if (before <= goal && before + sum > goal) pick(s, a, l, t, before, goal, whole, w, y, index);
        base += all;
        if (base > goal) break;  // uniform
    }
}

// kMany: the cut of one limit by going over the row, in one workgroup. It is the first element whose elements number
// `need`, or whose weights reach `need` (by_weight), and lies in s.bin (s.rest and s.before come before it).
// Writes s.cut (its place) and s.through (the weights up to it). All threads call it.
template <typename E> __device__ __forceinline__ void find_cut(Shared &s, const Row<E> &row, const Limits &l, u64 need, bool by_weight)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ranges = row.parts * kWaves;
    const int bin = s.bin;
    u64 count = s.rest, sum = s.before;
    u64 *number = s.list, *heavy = s.list + 256;
    // its number eight bits at a time, then its index among equal ones
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) number[tid] = heavy[tid] = 0;
        __syncthreads();
        for (int r = wave; r < ranges; r += kWaves)
            row.for_range(r, [&](const float (&x)[8], int) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t o = order_of(x[j]);
                    if (l.bin(x[j]) == bin && (shift == 24 || (o ^ prefix) >> (shift + 8) == 0)) {
                        atomicAdd(&number[o >> shift & 255], 1ull);
                        if (l.by_p) atomicAdd(&heavy[o >> shift & 255], l.weigh(x[j]));
                    }
                }
            });
        __syncthreads();
        // digits from the largest down
        const u64 c = tid < 256 ? number[255 - tid] : 0, w = tid < 256 ? heavy[255 - tid] : 0;
        u64 all;
        const u64 cb = count + sum_before(s, c, &all), wb = sum + sum_before(s, w, &all);
        if (c && (by_weight ? wb < need && wb + w >= need : cb < need && cb + c >= need)) {
            s.cursor[0] = 255 - tid;
            s.rest = (uint32_t)cb;
            s.before = wb;
        }
        __syncthreads();
        prefix |= s.cursor[0] << shift;
        count = s.rest;
        sum = s.before;
    }
    // the elements equal to it weigh the same
    const u64 w = l.weigh(number_of(prefix));
    const uint32_t rank = by_weight ? (uint32_t)((need - sum + w - 1) / w) : (uint32_t)(need - count);  // from 1
    const int segments = (row.groups() + 63) / 64, per = (segments + kThreads - 1) / kThreads;
    auto equal_of = [&](int seg, float (&x)[8]) {
        u64 equal = 0;
        if (64 * seg + lane < row.groups()) {
            row.load(64 * seg + lane, row.groups()).to(x, row.infinite);
#pragma unroll
            for (int j = 0; j < 8; ++j) equal += order_of(x[j]) == prefix;
        }
        return equal;
    };
    float x[8];
    for (int seg = wave; seg < segments; seg += kWaves) {
        const u64 of_wave = wave_sum(equal_of(seg, x));
        if (lane == 0) s.segment[seg] = of_wave;
    }
    __syncthreads();
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
    if (wave == 0) {
        const u64 equal = equal_of(s.bin, x);
        u64 n = s.before + wave_scan(equal) - equal;
        if (equal)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (order_of(x[j]) == prefix && ++n == rank) {
                    s.cut = place_of(x[j], row.first_of(64 * s.bin + lane) + j);
                    s.through = sum + rank * w;
                }
    }
    __syncthreads();
}

// The row's token, with what `decide` asks for in the list and in s.range.
template <typename E, typename Bins>
__device__ __forceinline__ void finish(Shared &s, const Sample &a, const Row<E> &row, const Limits &l, int64_t t, const Decision &d, Bins bins)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, ranges = row.parts * kWaves;
    const int n = (int)min(s.cursor[0], (uint32_t)kList), m = (int)min(s.cursor[1], (uint32_t)(kList - n));
    u64 cut = 0;
    if (d.mode == kFew || d.mode == kInBin) {
        cut = last_kept(s, l, d, n, m);
        __syncthreads();
        if (d.mode == kFew) {
            draw_listed(s, a, row, l, t, n, m, cut);
            return;
        }
        for (int e = kList - m + tid; e < kList; e += kThreads) {
            const u64 place = s.list[e];
            const u64 w = l.kept(number_of((uint32_t)(place >> 32)), index_of(place), cut);
            if (w) atomicAdd(&s.range[row.range_of(index_of(place))], w);
        }
        __syncthreads();
    } else if (d.mode == kMany) {
        bins();
        u64 whole = d.all_w;
#pragma unroll 1
        for (int by_p = !d.k_cuts; by_p <= (int)l.by_p; ++by_p) {
            const u64 need = by_p ? l.need(whole) : (u64)l.top_k;
            Scan(s).find(s, need, by_p);
            find_cut(s, row, l, need, by_p);
            cut = max(cut, s.cut);
            whole = s.through;
            __syncthreads();
        }
        for (int r = wave; r < ranges; r += kWaves) {
            const u64 sum = sum_of<kFromCut>(row, l, r, cut, 0);
            if (lane == 0) s.range[r] = sum;
        }
        __syncthreads();
    }
    draw_ranges(s, a, row, l, t, cut);
}

// A workgroup a row.
template <typename E> __global__ __launch_bounds__(kThreads) void sample_kernel(Sample a)
{
    __shared__ Shared s;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    Row<E> row(a, t);
    const float2 ends = ends_of(s, row, 0);
    const Limits l(a, t, ends.x, ends.y);
    row.infinite = l.m == kLargest;
    if (l.none || l.greedy) {
        const int first = l.none ? -1 : first_of(s, row, l.m, 0);
        if (tid == 0) {
            a.token[t] = first;
            if (a.logprob) a.logprob[t] = l.none ? -INFINITY : 0.f;
        }
        return;
    }
    if (!l.cuts()) {
        const u64 sum = sum_of<kAll>(row, l, wave, 0, 0);
        if (lane == 0) s.range[wave] = sum;
        __syncthreads();
        draw_ranges(s, a, row, l, t, 0);
        return;
    }
    fill_bins(s, row, l, 0);
    const Decision d = decide(s, l, Scan(s));
    u64 sum = 0;
    if (d.mode == kFew) collect<true>(s, row, l, 0, d.bin);
    else if (d.mode == kInBin) sum = collect<false>(s, row, l, 0, d.bin);
    else if (d.mode == kWhole) sum = sum_of<kBefore>(row, l, wave, 0, d.bin);
    if (lane == 0) s.range[wave] = sum;
    __syncthreads();
    finish(s, a, row, l, t, d, [] {});
}

// The same in four launches, parts of a row by workgroups of their own (blockIdx.x = row * parts + part); what
// one finds is in device memory (SampleShare) for the next.
template <typename E> __global__ __launch_bounds__(kThreads) void sample_ends_kernel(Sample a, SampleShare x)
{
    __shared__ Shared s;
    const int64_t t = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    const float2 ends = ends_of(s, Row<E>(a, t), part);
    if (threadIdx.x == 0) x.ends[blockIdx.x] = ends;
    if (part == 0 && threadIdx.x < 2) x.cursor[2 * t + threadIdx.x] = 0;
}

__device__ __forceinline__ Limits shared_limits(const Sample &a, const SampleShare &x, int64_t t)
{
    float2 ends = x.ends[t * a.parts];
    for (int p = 1; p < a.parts; ++p) {
        const float2 y = x.ends[t * a.parts + p];
        ends = make_float2(fmaxf(ends.x, y.x), fminf(ends.y, y.y));
    }
    return Limits(a, t, ends.x, ends.y);
}

template <typename E> __global__ __launch_bounds__(kThreads) void sample_bins_kernel(Sample a, SampleShare x)
{
    __shared__ Shared s;
    const int64_t t = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, tid = threadIdx.x;
    Row<E> row(a, t);
    const Limits l = shared_limits(a, x, t);
    row.infinite = l.m == kLargest;
    if (l.none) return;
    if (l.greedy) {
        const int first = first_of(s, row, l.m, part);
        if (tid == 0) x.first[blockIdx.x] = first;
        return;
    }
    if (!l.cuts()) {
        const u64 sum = sum_of<kAll>(row, l, part * kWaves + (tid >> 6), 0, 0);
        if ((tid & 63) == 0) x.range[(int64_t)blockIdx.x * kWaves + (tid >> 6)] = sum;
        return;
    }
    fill_bins(s, row, l, part);
    for (int b = tid; b < kBins; b += kThreads) {
        x.count[(int64_t)blockIdx.x * kBins + b] = s.count[b];
        if (l.by_p) x.sum[(int64_t)blockIdx.x * kBins + b] = s.sum[b];
    }
}

// The row's bins from its parts', in LDS.
__device__ __forceinline__ void load_bins(Shared &s, const Sample &a, const SampleShare &x, const Limits &l, int64_t t)
{
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
        uint32_t count = 0;
        u64 sum = 0;
#pragma unroll
        for (int p = 0; p < kSampleMaxParts; ++p)
            if (p < a.parts) {
                count += x.count[(t * a.parts + p) * kBins + b];
                if (l.by_p) sum += x.sum[(t * a.parts + p) * kBins + b];
            }
        s.count[b] = count;
        s.sum[b] = sum;
    }
    __syncthreads();
}

template <typename E> __global__ __launch_bounds__(kThreads) void sample_collect_kernel(Sample a, SampleShare x)
{
    __shared__ Shared s;
    const int64_t t = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, tid = threadIdx.x;
    Row<E> row(a, t);
    const Limits l = shared_limits(a, x, t);
    row.infinite = l.m == kLargest;
    if (!l.cuts()) return;
    load_bins(s, a, x, l, t);
    const Decision d = decide(s, l, Scan(s));
    if (part == 0 && tid == 0) ((Decision *)x.decision)[t] = d;
    u64 sum = 0;
    if (d.mode == kFew) collect<true>(s, row, l, part, d.bin);
    else if (d.mode == kInBin) sum = collect<false>(s, row, l, part, d.bin);
    else if (d.mode == kWhole) sum = sum_of<kBefore>(row, l, part * kWaves + (tid >> 6), 0, d.bin);
    if ((tid & 63) == 0) x.range[(int64_t)blockIdx.x * kWaves + (tid >> 6)] = sum;
    if (d.mode == kFew || d.mode == kInBin) {
        // in LDS first: an addition to the row's cursors returns after microseconds
        __syncthreads();
        if (tid < 2) s.at[tid] = atomicAdd(&x.cursor[2 * t + tid], s.cursor[tid]);
        __syncthreads();
        u64 *list = (u64 *)x.list + t * kList;
        const uint32_t n = min(s.cursor[0], (uint32_t)kList), m = min(s.cursor[1], (uint32_t)kList - n);
        for (uint32_t e = tid; e < n; e += kThreads)
            if (s.at[0] + e < kList) list[s.at[0] + e] = s.list[e];
        for (uint32_t e = tid; e < m; e += kThreads)
            if (s.at[1] + e < kList) list[kList - 1 - s.at[1] - e] = s.list[kList - 1 - e];
    }
}

template <typename E> __global__ __launch_bounds__(kThreads) void sample_draw_kernel(Sample a, SampleShare x)
{
    __shared__ Shared s;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, ranges = a.parts * kWaves;
    Row<E> row(a, t);
    const Limits l = shared_limits(a, x, t);
    row.infinite = l.m == kLargest;
    if (l.none || l.greedy) {
        if (tid == 0) {
            int first = INT32_MAX;
            for (int p = 0; p < a.parts; ++p) first = min(first, l.none ? -1 : x.first[t * a.parts + p]);
            a.token[t] = first;
            if (a.logprob) a.logprob[t] = l.none ? -INFINITY : 0.f;
        }
        return;
    }
    if (tid < ranges) s.range[tid] = x.range[t * ranges + tid];
    if (!l.cuts()) {
        __syncthreads();
        draw_ranges(s, a, row, l, t, 0);
        return;
    }
    const Decision d = ((const Decision *)x.decision)[t];
    if (tid < 2) s.cursor[tid] = x.cursor[2 * t + tid];
    __syncthreads();
    const int n = (int)min(s.cursor[0], (uint32_t)kList), m = (int)min(s.cursor[1], (uint32_t)(kList - n));
    for (int e = tid; e < kList; e += kThreads)
        if (e < n || e >= kList - m) s.list[e] = ((const u64 *)x.list)[t * kList + e];
    __syncthreads();
    finish(s, a, row, l, t, d, [&] { load_bins(s, a, x, l, t); });
}

template <typename E> hipError_t launch(const Sample &a, const SampleShare &x, hipStream_t s)
{
    const dim3 rows((unsigned)a.T), parts((unsigned)(a.T * a.parts)), block(kThreads);
    if (!x.ends) {
        hipLaunchKernelGGL((sample_kernel<E>), rows, block, 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((sample_ends_kernel<E>), parts, block, 0, s, a, x);
    hipLaunchKernelGGL((sample_bins_kernel<E>), parts, block, 0, s, a, x);
    if (a.top_k || a.top_p) hipLaunchKernelGGL((sample_collect_kernel<E>), parts, block, 0, s, a, x);
    hipLaunchKernelGGL((sample_draw_kernel<E>), rows, block, 0, s, a, x);
    return hipGetLastError();
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// One launch takes 8-17 us where four take 12-25 (up to 16,000 logits), but a workgroup goes over 128,000 in 120 us with
// top_p (four of them 58, eight 55; 32 rows), 43 without limits (21, 18). Rows are shared out while that
// leaves every part 8,000 logits and a CU: top_p of 32,000 logits, one row 32.3 us in one launch, 29.6 in four
// parts, 64 rows 38.9 and 40.3; 128 rows of 32,000 and 64,000 39.4 and 68.7, in two parts 42.9 and 58.2; 250 rows
// of 128,000 130, in two parts 143.
int sample_parts(int64_t T, int64_t V, int num_cus)
{
    const int64_t parts = std::min<int64_t>(std::min<int64_t>(num_cus / T, kSampleMaxParts), V / 8000);
    return parts < 2 || (parts == 2 && V < 48000) ? 0 : (int)parts;
}

size_t sample_workspace(int64_t T, int parts, bool cuts, char *base, SampleShare *x)
{
    size_t at = 0;
    auto take = [&](size_t n) {
        char *p = base ? base + at : nullptr;
        at += align256(n);
        return (void *)p;
    };
    SampleShare y = {};
    if (parts) {
        const size_t P = (size_t)T * parts;
        y.ends = (float2 *)take(P * 8);
        y.first = (int *)take(P * 4);
        y.range = (unsigned long long *)take(P * kWaves * 8);
        y.cursor = (uint32_t *)take((size_t)T * 8);
        if (cuts) {
            y.decision = take((size_t)T * sizeof(Decision));
            y.list = (unsigned long long *)take((size_t)T * kList * 8);
            y.count = (uint32_t *)take(P * kBins * 4);
            y.sum = (unsigned long long *)take(P * kBins * 8);
        }
    }
    if (x) *x = y;
    return at;
}

hipError_t launch_sample(Sample a, int parts, const SampleShare &x, hipStream_t s)
{
    const int groups = (a.V + 7 + 7) / 8;
    a.parts = std::max(parts, 1);
    const int waves = kWaves * a.parts;
    a.per = (groups + waves * 64 - 1) / (waves * 64) * 64;
    return a.dt == IVF_F32   ? launch<float>(a, x, s)
           : a.dt == IVF_F16 ? launch<_Float16>(a, x, s)
                             : launch<__bf16>(a, x, s);
}

}  // namespace ivf
