// How an attention call over the 4-bit cache is carried out: which kernel takes which
// rows in how many parts, and the joining of split key ranges. The single-token kernel
// is in kv_attend_kernel.h.
#include "kv_attend_kernel.h"

namespace ivf {
namespace {

// Joins the parts of a row: WAVES waves per row take the parts in turn, lanes over
// channels; the last sum, over waves, is in their order.
enum CombineRows { kByUnit, kBySplit, kByPrompt };
template <typename TT, int ROWS, int WAVES>
__device__ __forceinline__ void combine_rows(const KvAttend &a, int64_t rows, uint32_t block)
{
    typedef typename TT::elem elem;
    __shared__ float4 sums[kWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int turn = wave % WAVES;
    const int64_t row = (int64_t)block * (kWaves / WAVES) + wave / WAVES;
    if (row >= rows) return;
    int64_t orow = row, at = row * a.splits;  // the first part, in rows of part[]
    int n = a.splits, stride = 1;
    if (ROWS == kByUnit) {
        const uint32_t x = (uint32_t)row / (uint32_t)a.c.heads, unit = x / (uint32_t)a.unit_rows;
        const uint32_t b = unit / (uint32_t)a.per_unit;
        const int head = (int)((uint32_t)row - x * (uint32_t)a.c.heads), col = (int)(x - unit * (uint32_t)a.unit_rows);
        const uint32_t r = (unit - b * (uint32_t)a.per_unit) * (uint32_t)a.unit_size + col;
        const int64_t t0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
        const int64_t m = (min(max((int64_t)a.start[b + 1], t0), a.T) - t0) * a.group;
        if (r >= m || m > a.small_rows) return;
        const int2 parts = a.unit_parts[unit];
        n = parts.y;
        if (n <= 1) return;  // written already
        at = ((int64_t)head * a.slots + parts.x) * a.unit_rows + col;
        stride = a.unit_rows;
        orow = ((t0 + r / (uint32_t)a.group) * a.c.heads + head) * a.group + r % (uint32_t)a.group;
    } else if (ROWS == kByPrompt) {
        const int64_t t = (uint32_t)row / (uint32_t)(a.c.heads * a.group);
        int64_t b = 0, hi = a.B;
        while (hi - b > 1) {
            const int64_t mid = (b + hi) >> 1;
            if (a.start[mid] <= t) b = mid;
            else hi = mid;
        }
        const int64_t t0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
        const int64_t t1 = min(max((int64_t)a.start[b + 1], t0), a.T);
        if (t < t0 || t >= t1 || (t1 - t0) * a.group <= a.small_rows) return;
    }
    const float2 *ml = a.part_ml + at;
    float top = -INFINITY;
    for (int s = lane; s < n; s += 64) top = fmaxf(top, ml[(int64_t)s * stride].x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    float total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const float *p = a.part + at * a.c.dim + 2 * lane;
    const int64_t part_stride = (int64_t)stride * a.c.dim;
    const bool in0 = 2 * lane < a.c.dim, in1 = 128 + 2 * lane < a.c.dim;
    for (int s0 = 0; s0 < n; s0 += 64) {
        float f = 0.f;
        if (s0 + lane < n) {
            const float2 x = ml[(int64_t)(s0 + lane) * stride];
            f = x.y == 0.f ? 0.f : x.x > -INFINITY ? exp2_fast(x.x - top) : x.y;
            total += x.y * f;
        }
        const int end = min(64, n - s0);
#pragma unroll 8
        for (int s = turn; s < end; s += WAVES) {
            const float fs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s));
            const float *ps = p + (s0 + s) * part_stride;
            const float2 y0 = in0 ? *(const float2 *)ps : make_float2(0.f, 0.f);
            const float2 y1 = in1 ? *(const float2 *)(ps + 128) : make_float2(0.f, 0.f);
            o.x += y0.x * fs;
            o.y += y0.y * fs;
            o.z += y1.x * fs;
            o.w += y1.y * fs;
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    if (WAVES > 1) {
        sums[wave][lane] = o;
        __syncthreads();
        if (turn != 0) return;
        for (int w = 1; w < WAVES; ++w) {
            const float4 y = sums[wave + w][lane];
            o.x += y.x;
            o.y += y.y;
            o.z += y.z;
            o.w += y.w;
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    elem *out = (elem *)a.out + orow * a.c.dim + 2 * lane;
    if (in0) *(uint32_t *)out = TT::pack(o.x * inv, o.y * inv);
    if (in1) *(uint32_t *)(out + 128) = TT::pack(o.z * inv, o.w * inv);
    if (a.lse && lane == 0) a.lse[orow] = log_of(top, total);
}

template <typename TT, int ROWS, int WAVES>
__global__ __launch_bounds__(kThreads) void kv_combine_kernel(KvAttend a, int64_t rows)
{
    combine_rows<TT, ROWS, WAVES>(a, rows, blockIdx.x);
}

// Parts of prompts (the first `blocks` workgroups) and of other requests' units in one launch (a prompt of
// 500 tokens among seven single ones, 2 heads x 128, 5,000 keys: 66 us, with a launch each 71).
template <typename TT>
__global__ __launch_bounds__(kThreads) void kv_combine_both_kernel(KvAttend prompts, int64_t rows, uint32_t blocks, KvAttend units,
                                                                   int64_t unit_rows)
{
    if (blockIdx.x < blocks) combine_rows<TT, kByPrompt, 1>(prompts, rows, blockIdx.x);
    else combine_rows<TT, kByUnit, 4>(units, unit_rows, blockIdx.x - blocks);
}

// prompts, units: calls whose parts are to be joined, or null.
template <typename TT> hipError_t launch_combine(const KvAttend *prompts, const KvAttend *units, hipStream_t s)
{
    const dim3 block(kThreads);
    const int64_t prompt_rows = prompts ? prompts->T * prompts->group * prompts->c.heads : 0;
    const int64_t rows = !units ? 0 : units->blocks ? units->T * units->group * units->c.heads
                                                    : (int64_t)units->units * units->unit_rows * units->c.heads;
    const unsigned prompt_blocks = (unsigned)((prompt_rows + kWaves - 1) / kWaves);
    if (prompts && units)  // then without selected blocks
        hipLaunchKernelGGL((kv_combine_both_kernel<TT>), dim3(prompt_blocks + (unsigned)rows), block, 0, s, *prompts, prompt_rows,
                           prompt_blocks, *units, rows);
    else if (prompts)
        hipLaunchKernelGGL((kv_combine_kernel<TT, kByPrompt, 1>), dim3(prompt_blocks), block, 0, s, *prompts, prompt_rows);
    else if (units->blocks)
        hipLaunchKernelGGL((kv_combine_kernel<TT, kBySplit, 4>), dim3((unsigned)rows), block, 0, s, *units, rows);
    else
        hipLaunchKernelGGL((kv_combine_kernel<TT, kByUnit, 4>), dim3((unsigned)rows), block, 0, s, *units, rows);
    return hipGetLastError();
}

// Requests with at most this many rows go through the single-token kernel, 16 rows a
// workgroup, others through the prompt kernel. After 4,000 tokens, 8 heads x 128, caches cold, here and there, for 64,
// 128, 256 and 512 rows: one request 28.0 and 30.8, 30.0 and 35.4, 35.9 and 47.1, 47.1 and 44.5 us; 8 requests 51.8
// and 72.4, 75.6 and 69.5, 117 and 80.0, 202 and 151; 32 requests 134 and 157, 222 and 237, 357 and 175, 679 and 323. So
// the two cross between 64 and 256 rows, later for one request, of which the limit takes no note.
constexpr int64_t kSmallRows = 64;

// Tables of at most this many keys are not shared out: joining parts costs a launch and the prefix
// sums. Measured at 128 channels, and taken for every width. `all` units of one token, 8 heads x 128, lengths drawn up to the limit, shared out and not: 8 units,
// 2,048 keys 12.2 and 15.1 us; 32 units, 2,048 keys 16.6 and 14.2, 4,096 keys 17.0 and 20.0; 128 units, 4,096
// keys 26.4 and 22.5; 1,024 units, 4,096 keys 82 and 79.
constexpr int64_t whole_keys(int64_t all) { return all < 32 ? 1024 : all < 128 ? 2048 : 4096; }

}  // namespace

KvAttendPlan kv_attend_plan(const KvCache &c, int group, int64_t T, int64_t B, int64_t cols, int64_t count,
                            int64_t longest, int num_cus)
{
    KvAttendPlan p = {};
    const int64_t keys = (count ? count : cols) << c.shift;
    auto align = [](size_t n) { return (n + 255) / 256 * 256; };
    int64_t rows;  // of one request or token, at most
    if (count) {
        p.tokens = true;
        rows = group;
        p.small_rows = INT64_MAX;
    } else {
        rows = longest * group;
        p.tokens = rows <= kSmallRows || B > 1;
        p.prompt = rows > kSmallRows;
        p.small_rows = !p.prompt ? INT64_MAX : p.tokens ? kSmallRows : 0;
        rows = std::min(rows, kSmallRows);
    }
    p.token_splits = p.prompt_splits = 1;
    p.team = kWaves;
    if (p.tokens) {
        p.unit_size = count && rows <= 8 ? 8 : 16;
        p.per_unit = (int)((rows + p.unit_size - 1) / p.unit_size);
        p.unit_rows = (int)std::min<int64_t>(rows, p.unit_size);
        p.units = (count ? T : B) * p.per_unit;
        // Waves that share a unit, where units are not cut into parts:
        // * eight where there are at most as many units as CUs, but not for 512 keys or fewer (256 units of 4,096
        //   selected keys 32 us, with four waves 34; single tokens after 777 tokens, 256 units 11.3 and 11.8,
        //   after 300 tokens, 128 units 8.8 and 7.9), nor beyond 128 channels (over 256 registers a wave);
        // * one where there is a unit for every wave that the device holds: alone it joins nothing
        //   (2,048 units of 1,536 selected keys x 128 channels 51 us, with four 55; 1,536 units 49 and 42; 256
        //   channels, 1,024 units 61 and 83, 512 units 59 and 43);
        // * four otherwise.
        const int64_t all = p.units * c.heads;
        const bool shared = !count && keys > whole_keys(all) && p.units <= kKvMaxUnits && all < 16 * (int64_t)num_cus;
        if (count && all >= (c.dim <= 128 ? 8 : 4) * (int64_t)num_cus) p.team = 1;
        else if (c.dim <= 128 && !shared && all <= num_cus && keys > 512) p.team = 8;
        // as many workgroups as are resident at once: a further round would only begin and join again
        // (16 tokens, 8 heads, 4,096 selected keys: 18.6 us, two rounds 24.5)
        if (count) {
            const int64_t most = std::max<int64_t>(1, keys / (32 * kMinSteps));
            p.token_splits = (int)std::max<int64_t>(1, std::min(num_cus / all, most));
        } else if (shared) {
            const int64_t resident = (int64_t)num_cus * (c.dim <= 128 ? 2 : 1);
            p.token_splits = (int)std::max<int64_t>(1, resident / c.heads);
        }
        if (p.token_splits > 1) {
            p.slots = p.token_splits + p.units;
            const size_t n = count ? (size_t)T * group * c.heads * p.token_splits : (size_t)p.slots * p.unit_rows * c.heads;
            p.token_ml = align(n * c.dim * 4);
            p.token_parts = p.token_ml + align(n * 8);
            p.token_bytes = p.token_parts + align(count ? 0 : (size_t)p.units * 8);
        }
        p.token_groups = count || p.token_splits == 1 ? p.units * p.token_splits : p.token_splits;
    }
    if (p.prompt) {
        const int64_t units = (T * group + kv_prompt_rows(c.dim) - 1) / kv_prompt_rows(c.dim) * c.heads;
        // parts of a tile of keys or more until every CU has work (64 tokens after 1,000: 23.8 us, parts of at
        // least two tiles 25.5, of four 32)
        if (units < kv_prompt_resident(c.dim) * (int64_t)num_cus / 2) {
            const int64_t most = std::max<int64_t>(1, keys / 128);
            p.prompt_splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(kv_prompt_resident(c.dim) * (int64_t)num_cus / units, most), 32));
        }
        if (p.prompt_splits > 1) {
            const size_t n = (size_t)T * group * c.heads * p.prompt_splits;
            p.prompt_ml = align(n * c.dim * 4);
            p.prompt_bytes = p.prompt_ml + align(n * 8);
        }
    }
    return p;
}

hipError_t launch_kv_tokens(const KvAttend &a, int64_t groups, hipStream_t s)
{
    return a.c.bf16 ? launch_tokens_dim<KvBf16>(a, KvNoTerms(), groups, s) : launch_tokens_dim<KvF16>(a, KvNoTerms(), groups, s);
}

hipError_t launch_kv_combine(const KvAttend *prompts, const KvAttend *units, hipStream_t s)
{
    const KvAttend &any = prompts ? *prompts : *units;
    return any.c.bf16 ? launch_combine<KvBf16>(prompts, units, s) : launch_combine<KvF16>(prompts, units, s);
}

}  // namespace ivf
