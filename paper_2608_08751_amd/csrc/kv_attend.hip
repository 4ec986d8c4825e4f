// Attention of up to 16 query rows of one key/value head over the 4-bit cache,
// and the joining of split key ranges.
//
// A row's output is sum_j p_j v_j / sum_j p_j with p_j = exp2(t_j - r), t_j = scale
// log2(e) q.k_j and a reference r that follows the running maximum of t. Keys and
// values go from 4 bits straight to MFMA operands in registers:
//   * scores: S^T = K Q^T, v_mfma_f32_16x16x32 with 16 keys (a strip) as A. Lane (r =
//     lane % 16, h = lane / 16) holds key 4 (r % 4) + r / 4 of the strip, so that its
//     four results are keys 4 i + h of query row r; the channels of a key are taken in
//     the order in which its row of codes lies in memory (any order serves, the query's
//     fragments use the same), 16 bytes a lane and strip at 128 channels.
//   * values: O^T = V^T P^T. The results above are the B operand as they are: lane h's
//     eight probabilities of two strips are keys 4 i + h. A lane reads the codes of
//     neighbouring channels of those keys (four loads of 256 consecutive bytes a wave),
//     v_cvt_scalef32 makes pairs of channels with the key's scale, v_perm_b32 pairs of keys.
//   * the reference is raised only when a score passes it by 2^6, for all rows of the
//     wave at once, so the common step has no exchange between lanes. Probabilities
//     carry 2^8, which keeps small ones normal in f16 (at most 2^14).
// Masked scores are replaced, not added to; values of keys that no row sees get scale
// 1, so that nothing left in unused slots reaches a sum.
//
// A workgroup of four waves takes a range of steps of 32 keys, each wave every fourth
// step with its own reference, sums and output, joined in LDS. What bounds single
// tokens is the read of the cache, 17 / 16 bytes per channel of key and value.
#include "kv.h"
#include "kv_strip.h"

#include <algorithm>
#include <type_traits>

namespace ivf {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kMinSteps = 8;   // steps of 32 keys that a part is worth

// The rows of one workgroup: rows r0 ... r0 + n of a request's (or token's) rows,
// row = token * group + head of the group.
struct RowSet {
    int64_t t0;  // token of row 0
    int r0, n;
    int b;
};

template <typename TT, int D, bool SPARSE>
__global__ __launch_bounds__(kThreads) void kv_attend_kernel(KvAttend a)
{
    typedef Pieces<D> P;
    typedef typename TT::elem elem;
    constexpr int kTiles = D / 16;
    __shared__ float merge[2][kTiles * 4 * 64];
    __shared__ float2 ml[kWaves][16];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, h = lane >> 4;
    const int head = blockIdx.x % a.c.heads;
    const int split = (blockIdx.x / a.c.heads) % a.splits;
    const int64_t unit = blockIdx.x / a.c.heads / a.splits;

    RowSet rs;
    if (SPARSE) {
        rs.t0 = unit / a.per_unit;
        rs.r0 = (int)(unit % a.per_unit) * 16;
        rs.n = min(16, a.group - rs.r0);
        rs.b = a.request[rs.t0];
    } else {
        rs.b = (int)(unit / a.per_unit);
        rs.r0 = (int)(unit % a.per_unit) * 16;
        const int64_t t0 = min(max((int64_t)a.start[rs.b], (int64_t)0), a.T);
        const int64_t t1 = min(max((int64_t)a.start[rs.b + 1], t0), a.T);
        rs.t0 = t0;
        const int64_t rows = (t1 - t0) * a.group;
        if (rs.r0 >= rows || rows > a.small_rows) return;
        rs.n = (int)min((int64_t)16, rows - rs.r0);
    }
    const bool live = rs.b >= 0 && rs.b < a.B;

    // this lane's row
    const bool have = col < rs.n;
    const int row = rs.r0 + (have ? col : 0);
    const int64_t tok = rs.t0 + row / a.group;
    const int qhead = head * a.group + row % a.group;
    const int last_key = (int)min((int64_t)a.cols << a.c.shift, (int64_t)INT32_MAX) - 1;
    const int lim = live ? min(a.position[tok], last_key) : -1;
    int lim_max = have ? lim : -1, lim_min = have ? lim : INT32_MAX;
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        lim_max = max(lim_max, __shfl_xor(lim_max, d));
        lim_min = min(lim_min, __shfl_xor(lim_min, d));
    }
    lim_max = __builtin_amdgcn_readfirstlane(lim_max);
    lim_min = __builtin_amdgcn_readfirstlane(lim_min);

    u32x4 qf[D / 32];
    {
        const elem *q = (const elem *)a.q.p + tok * a.q.ts + (int64_t)qhead * a.q.hs;
#pragma unroll
        for (int c = 0; c < P::n; ++c)
#pragma unroll
            for (int d = 0; d < P::size(c) / 32; ++d) {
                u32x4 x = {0, 0, 0, 0};
                if (have) x = *(const u32x4 *)(q + P::off(c) + P::size(c) / 4 * h + 8 * d);
                qf[P::off(c) / 32 + d] = x ^ a.q_flip;
            }
    }

    // the steps of 32 keys of this part, wave by wave
    const int strip_shift = a.c.shift - 4, strip_mask = (1 << strip_shift) - 1;
    int strips;
    if (SPARSE) strips = lim_max < 0 ? 0 : a.count << strip_shift;
    else strips = (lim_max + 16) >> 4;
    const int steps = (strips + 1) >> 1;
    const int per = max((steps + a.splits - 1) / a.splits, a.splits > 1 ? kMinSteps : 1);
    const int s_end = min((int64_t)steps, (int64_t)(split + 1) * per);
    int step = min((int64_t)steps, (int64_t)split * per) + wave;

    const int32_t *table = a.table + (int64_t)(live ? rs.b : 0) * a.cols;
    const int32_t *list = SPARSE ? a.blocks + (rs.t0 * a.c.heads + head) * a.count : nullptr;
    const size_t rec_bytes = a.c.rec_bytes();

    f32x4 acc[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float ref = -INFINITY, sub = 0.f, sum = 0.f;

    // lane 2 i + s keeps the block and the first key of strip s of the wave's i-th next step
    int pages = -1, bases = 0, ahead = 0;
    auto look = [&](int first_step) {
        const int64_t st = (int64_t)first_step + (lane >> 1) * kWaves;
        const int64_t v = 2 * st + (lane & 1);
        pages = -1;
        bases = 0;
        if (st < s_end && v < strips) {
            int64_t j;
            int base;
            if (SPARSE) {
                j = list[v >> strip_shift];
                base = (int)(j << a.c.shift) + ((int)v & strip_mask) * 16;
            } else {
                base = (int)v * 16;
                j = base >> a.c.shift;
            }
            if (j >= 0 && j < a.cols && base <= lim_max) {
                const int id = table[j];
                if (id >= 0 && id < a.c.blocks) {
                    pages = id;
                    bases = base;
                }
            }
        }
    };
    const LaneOffsets<D> offs(lane, a.c.bs);
    struct Pair {
        Strip<D> s[2];
        int page[2], base[2];
    };
    auto fetch = [&](Pair &x, int at_step) {
        if (ahead == 32) {
            look(at_step);
            ahead = 0;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            x.page[e] = __builtin_amdgcn_readlane(pages, 2 * ahead + e);
            x.base[e] = __builtin_amdgcn_readlane(bases, 2 * ahead + e);
        }
        ++ahead;
        if ((x.page[0] & x.page[1]) >= 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint8_t *rec = a.c.rec + ((int64_t)max(x.page[e], 0) * a.c.heads + head) * rec_bytes;
                load_strip<D>(x.s[e], rec, a.c.bs, (x.base[e] >> 4) & strip_mask, offs);
            }
        }
    };
    auto work = [&](const Pair &x) {
        if ((x.page[0] & x.page[1]) < 0) return;  // neither strip is there
        float t[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < P::n; ++c) {
                const float ks = kv_scale(x.s[e].ks[c]);
#pragma unroll
                for (int d = 0; d < P::size(c) / 32; ++d) {
                    const int w = P::off(c) / 32 + d;
                    y = TT::mfma(decode8<TT>(x.s[e].k[w], ks), qf[w], y);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) t[4 * e + i] = y[i] * a.scale;
        }
        float vs[P::n][2][4];
#pragma unroll
        for (int c = 0; c < P::n; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) vs[c][i / 4][i % 4] = kv_scale((x.s[i / 4].vs[c][i % 4] >> (8 * h)) & 255u);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (x.page[e] < 0 || x.base[e] + 15 > lim_min) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = x.page[e] < 0 ? INT32_MAX : x.base[e] + 4 * i + h;
                    if (key > lim) t[4 * e + i] = -INFINITY;
#pragma unroll
                    for (int c = 0; c < P::n; ++c)
                        if (key > lim_max) vs[c][e][i] = 1.f;
                }
            }
        }
        const float mx = max3(max3(t[0], t[1], t[2]), max3(t[3], t[4], t[5]), max3(t[6], t[7], t[7]));
        if (__ballot(mx > ref + kRaise)) {
            const float top = fmaxf(ref, max_over_h(mx));
            const float f = ref == top ? 1.f : exp2_fast(ref - top);
            ref = top;
            sub = top == -INFINITY ? 0.f : top - kCarry;
            sum *= f;
#pragma unroll
            for (int i = 0; i < kTiles; ++i) acc[i] *= f;
        }
        u32x4 pf;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float p0 = exp2_fast(t[i] - sub), p1 = exp2_fast(t[i + 1] - sub);
            sum += p0 + p1;
            pf[i / 2] = TT::pack(p0, p1);
        }
        auto piece = [&](auto piece_c) {
            constexpr int c = decltype(piece_c)::value, S = P::size(c);
            u32x2 v0[S / 16], v1[S / 16];
            value_operands<TT, S>(x.s[0].v[c], vs[c][0], v0);
            value_operands<TT, S>(x.s[1].v[c], vs[c][1], v1);
#pragma unroll
            for (int j = 0; j < S / 16; ++j) {
                const u32x4 v = {v0[j][0], v0[j][1], v1[j][0], v1[j][1]};
                acc[P::off(c) / 16 + j] = TT::mfma(v, pf, acc[P::off(c) / 16 + j]);
            }
        };
        piece(std::integral_constant<int, 0>());
        if constexpr (P::n > 1) piece(std::integral_constant<int, 1>());
    };
    if (step < s_end) {
        look(step);
        Pair x, y;
        fetch(x, step);
        while (true) {
            step += kWaves;
            if (step < s_end) fetch(y, step);
            work(x);
            if (step >= s_end) break;
            step += kWaves;
            if (step < s_end) fetch(x, step);
            work(y);
            if (step >= s_end) break;
        }
    }

    // join the waves: wave w's sums times exp2(ref_w - max)
    sum = sum_over_h(sum);
    if (h == 0) ml[wave][col] = make_float2(ref, sum);
    __syncthreads();
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][col].x);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float2 x = ml[w][col];
        if (x.x > -INFINITY || x.y != 0.f) total += x.y * exp2_fast(x.x - top);
    }
    const float f = ref > -INFINITY ? exp2_fast(ref - top) : sum != 0.f ? sum : 0.f;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) acc[i] *= f;
    float *buf = merge[wave & 1];
    if (wave >= 2) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) buf[(4 * i + r) * 64 + lane] = acc[i][r];
    }
    __syncthreads();
    if (wave < 2) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][r] += buf[(4 * i + r) * 64 + lane];
    }
    __syncthreads();
    if (wave == 1) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) merge[1][(4 * i + r) * 64 + lane] = acc[i][r];
    }
    __syncthreads();
    if (wave != 0 || !have) return;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][r] += merge[1][(4 * i + r) * 64 + lane];

    const int64_t orow = tok * ((int64_t)a.c.heads * a.group) + qhead;
    if (a.splits == 1) {
        write_rows<TT, D>(acc, (elem *)a.out + orow * D, total == 0.f ? 0.f : 1.f / total, h);
        if (a.lse && h == 0) a.lse[orow] = log_of(top, total);
    } else {
        const int64_t prow = SPARSE ? orow : (unit * a.unit_rows + col) * a.c.heads + head;
        const int64_t at = prow * a.splits + split;
        if (h == 0) a.part_ml[at] = make_float2(top, total);
        write_part<D>(acc, a.part + at * D, h);
    }
}

// Joins the parts of a row: a wave per row, lanes over channels. Parts without
// keys lie behind the others (or hold zeros), so the loop ends at the last that has some.
template <typename TT, bool UNITS>
__global__ __launch_bounds__(kThreads) void kv_combine_kernel(KvAttend a, int64_t rows)
{
    typedef typename TT::elem elem;
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= rows) return;
    int64_t orow = row;
    if (UNITS) {
        const int head = (int)(row % a.c.heads);
        const int64_t x = row / a.c.heads, unit = x / a.unit_rows, b = unit / a.per_unit;
        const int64_t r = unit % a.per_unit * 16 + x % a.unit_rows;
        const int64_t t0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
        const int64_t n = (min(max((int64_t)a.start[b + 1], t0), a.T) - t0) * a.group;
        if (r >= n || n > a.small_rows) return;
        orow = ((t0 + r / a.group) * a.c.heads + head) * a.group + r % a.group;
    } else if (!a.blocks) {
        const int64_t t = row / ((int64_t)a.c.heads * a.group);
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
    const float2 *ml = a.part_ml + row * a.splits;
    const float2 none = make_float2(-INFINITY, 0.f);
    const float2 x0 = lane < a.splits ? ml[lane] : none, x1 = lane + 64 < a.splits ? ml[lane + 64] : none;
    float top = fmaxf(x0.x, x1.x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    auto factor = [&](float2 x) { return x.y == 0.f ? 0.f : x.x > -INFINITY ? exp2_fast(x.x - top) : x.y; };
    const float f0 = factor(x0), f1 = factor(x1);
    float total = x0.y * f0 + x1.y * f1;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    const uint64_t m1 = __ballot(f1 != 0.f), m0 = __ballot(f0 != 0.f);
    const int parts = m1 ? 128 - __clzll((long long)m1) : m0 ? 64 - __clzll((long long)m0) : 0;
    float2 o[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    const float *p = a.part + row * a.splits * a.c.dim + 2 * lane;
    const bool in0 = 2 * lane < a.c.dim, in1 = 128 + 2 * lane < a.c.dim;
#pragma unroll 8
    for (int s = 0; s < parts; ++s) {
        const float f = __uint_as_float(s < 64 ? __builtin_amdgcn_readlane(__float_as_uint(f0), s & 63)
                                               : __builtin_amdgcn_readlane(__float_as_uint(f1), s & 63));
        const float2 y0 = in0 ? *(const float2 *)(p + (int64_t)s * a.c.dim) : make_float2(0.f, 0.f);
        const float2 y1 = in1 ? *(const float2 *)(p + (int64_t)s * a.c.dim + 128) : make_float2(0.f, 0.f);
        o[0].x += y0.x * f;
        o[0].y += y0.y * f;
        o[1].x += y1.x * f;
        o[1].y += y1.y * f;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    elem *out = (elem *)a.out + orow * a.c.dim + 2 * lane;
    if (in0) *(uint32_t *)out = TT::pack(o[0].x * inv, o[0].y * inv);
    if (in1) *(uint32_t *)(out + 128) = TT::pack(o[1].x * inv, o[1].y * inv);
    if (a.lse && lane == 0) a.lse[orow] = log_of(top, total);
}

template <typename TT, int D> hipError_t launch_tokens(const KvAttend &a, int64_t units, hipStream_t s)
{
    const unsigned grid = (unsigned)(units * a.splits * a.c.heads);
    if (a.blocks)
        hipLaunchKernelGGL((kv_attend_kernel<TT, D, true>), dim3(grid), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((kv_attend_kernel<TT, D, false>), dim3(grid), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <typename TT> hipError_t launch_tokens_dim(const KvAttend &a, int64_t units, hipStream_t s)
{
    switch (a.c.dim) {
    case 64: return launch_tokens<TT, 64>(a, units, s);
    case 96: return launch_tokens<TT, 96>(a, units, s);
    case 128: return launch_tokens<TT, 128>(a, units, s);
    case 192: return launch_tokens<TT, 192>(a, units, s);
    default: return launch_tokens<TT, 256>(a, units, s);
    }
}

// Requests with at most this many rows go through the single-token kernel,
// 16 rows a workgroup, where others take the prompt kernel.
constexpr int64_t kSmallRows = 64;

}  // namespace

KvAttendPlan kv_attend_plan(const KvCache &c, int group, int64_t T, int64_t B, int64_t cols, int64_t count,
                            int64_t longest, int num_cus)
{
    KvAttendPlan p = {};
    const int64_t keys = (count ? count : cols) << c.shift;
    const int64_t most = std::max<int64_t>(1, keys / (32 * kMinSteps));
    auto align = [](size_t n) { return (n + 255) / 256 * 256; };
    int64_t rows;  // of one unit at most, of one request or token
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
    if (p.tokens) {
        p.per_unit = (int)((rows + 15) / 16);
        p.unit_rows = (int)std::min<int64_t>(rows, 16);
        p.token_units = (count ? T : B) * p.per_unit;
        // beside a prompt most of a request's units are empty
        const int64_t busy = (p.prompt ? B * ((group + 15) / 16) : p.token_units) * c.heads;
        const int64_t want = ((int64_t)num_cus * 8 + busy - 1) / busy;
        p.token_splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, most), 128));
        if (p.token_splits > 1) {
            const size_t n = (size_t)(count ? T * group : p.token_units * p.unit_rows) * c.heads * p.token_splits;
            p.token_ml = align(n * c.dim * 4);
            p.token_bytes = p.token_ml + align(n * 8);
        }
    }
    if (p.prompt) {
        const int64_t units = (T * group + kv_prompt_rows(c.dim) - 1) / kv_prompt_rows(c.dim) * c.heads;
        if (units < num_cus) {
            const int64_t want = (2 * (int64_t)num_cus + units - 1) / units;
            p.prompt_splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, most), 32));
        }
        if (p.prompt_splits > 1) {
            const size_t n = (size_t)T * group * c.heads * p.prompt_splits;
            p.prompt_ml = align(n * c.dim * 4);
            p.prompt_bytes = p.prompt_ml + align(n * 8);
        }
    }
    return p;
}

hipError_t launch_kv_tokens(const KvAttend &a, int64_t units, hipStream_t s)
{
    return a.c.bf16 ? launch_tokens_dim<KvBf16>(a, units, s) : launch_tokens_dim<KvF16>(a, units, s);
}

hipError_t launch_kv_combine(const KvAttend &a, bool units, int64_t rows, hipStream_t s)
{
    const dim3 grid((unsigned)((rows + kWaves - 1) / kWaves)), block(kThreads);
    if (a.c.bf16 && units) hipLaunchKernelGGL((kv_combine_kernel<KvBf16, true>), grid, block, 0, s, a, rows);
    else if (a.c.bf16) hipLaunchKernelGGL((kv_combine_kernel<KvBf16, false>), grid, block, 0, s, a, rows);
    else if (units) hipLaunchKernelGGL((kv_combine_kernel<KvF16, true>), grid, block, 0, s, a, rows);
    else hipLaunchKernelGGL((kv_combine_kernel<KvF16, false>), grid, block, 0, s, a, rows);
    return hipGetLastError();
}

}  // namespace ivf
