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

// Units. A unit is up to 16 rows that share their keys: of the rows (token, head of
// the group) of a request, or of a token with selected blocks. Without them the
// number of keys differs from unit to unit and only the device knows it, so every
// workgroup forms the units' prefix sums of steps and takes an equal share of the
// whole, which may begin and end inside units: chunk = steps / workgroups, part w
// covers steps [w chunk, (w + 1) chunk). The results of part w of unit u lie at slot
// w + u (distinct, and one after the other for the parts of a unit).

// Steps of 32 keys that unit u's rows see; 0 for a unit without rows, else at
// least 1, so that somebody writes its rows.
__device__ int64_t unit_steps(const KvAttend &a, uint32_t u, int last_key)
{
    const uint32_t b = u / (uint32_t)a.per_unit;
    const int64_t r0 = (int64_t)(u - b * (uint32_t)a.per_unit) * 16;
    const int64_t t0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
    const int64_t rows = (min(max((int64_t)a.start[b + 1], t0), a.T) - t0) * a.group;
    if (r0 >= rows || rows > a.small_rows) return 0;
    const int64_t r1 = min(r0 + 16, rows) - 1;
    int lim = -1;
    for (int64_t t = t0 + (uint32_t)r0 / (uint32_t)a.group; t <= t0 + (uint32_t)r1 / (uint32_t)a.group; ++t)
        lim = max(lim, min(a.position[t], last_key));
    return max(1, (lim + 32) >> 5);
}

template <typename TT, int D, bool SPARSE>
__global__ __launch_bounds__(kThreads, D == 64 || (SPARSE && D <= 128) ? 3 : D <= 128 ? 2 : 1) void kv_attend_kernel(KvAttend a)
{
    typedef Pieces<D> P;
    typedef typename TT::elem elem;
    constexpr int kTiles = D / 16;
    __shared__ float merge[2][kTiles * 4 * 64];
    __shared__ float2 ml[kWaves][16];
    __shared__ int64_t before[SPARSE ? 1 : kKvMaxUnits + 1];  // steps of the units before
    __shared__ int64_t wave_steps[kWaves];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, h = lane >> 4;
    const uint32_t heads = a.c.heads, bid = blockIdx.x, part = bid / heads;
    const int head = (int)(bid - part * heads);
    const int last_key = (int)min((int64_t)a.cols << a.c.shift, (int64_t)INT32_MAX) - 1;
    const int strip_shift = a.c.shift - 4, strip_mask = (1 << strip_shift) - 1;
    const size_t rec_bytes = a.c.rec_bytes();
    const LaneOffsets<D> offs(lane, a.c.bs);

    uint32_t unit = part;
    int split = 0;
    int64_t from = 0, to = INT64_MAX, chunk = 0;  // this workgroup's steps, counted over all units
    if (SPARSE) {
        unit = part / (uint32_t)a.splits;
        split = (int)(part - unit * (uint32_t)a.splits);
    } else if (a.splits > 1) {
        constexpr int kPer = kKvMaxUnits / kThreads;
        int64_t mine[kPer], all = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t u = tid * kPer + i;
            mine[i] = all;
            if (u < (uint32_t)a.units) all += unit_steps(a, u, last_key);
        }
        int64_t up = all;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t x = __shfl_up(up, d);
            if (lane >= d) up += x;
        }
        if (lane == 63) wave_steps[wave] = up;
        __syncthreads();
        int64_t base = up - all, total = 0;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) base += wave_steps[w];
            total += wave_steps[w];
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) before[tid * kPer + i] = base + mine[i];
        if (tid == 0) before[kKvMaxUnits] = total;
        __syncthreads();
        chunk = max((total + a.splits - 1) / a.splits, (int64_t)kMinSteps);
        from = chunk * part;
        to = min(from + chunk, total);
        if (from >= to) return;
        int lo = 0, hi = a.units;  // the last unit with before <= from: it has steps
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (before[mid] <= from) lo = mid;
            else hi = mid;
        }
        unit = __builtin_amdgcn_readfirstlane(lo);
    }

    for (;; ++unit) {
    // the unit's rows
    int64_t t0;
    int r0, rows_here, b;
    if (SPARSE) {
        t0 = unit / (uint32_t)a.per_unit;
        r0 = (int)(unit % (uint32_t)a.per_unit) * 16;
        rows_here = min(16, a.group - r0);
        b = a.request[t0];
    } else {
        b = (int)(unit / (uint32_t)a.per_unit);
        r0 = (int)(unit % (uint32_t)a.per_unit) * 16;
        t0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
        const int64_t rows = (min(max((int64_t)a.start[b + 1], t0), a.T) - t0) * a.group;
        if (r0 >= rows || rows > a.small_rows) {
            if (a.splits == 1 || (int)unit + 1 >= a.units || before[unit + 1] >= to) return;
            continue;
        }
        rows_here = (int)min((int64_t)16, rows - r0);
    }
    const bool live = b >= 0 && b < a.B;

    // this lane's row
    const bool have = col < rows_here;
    const uint32_t row = r0 + (have ? col : 0), row_tok = row / (uint32_t)a.group;
    const int64_t tok = t0 + row_tok;
    const int qhead = head * a.group + (int)(row - row_tok * (uint32_t)a.group);
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
    int strips, s_end, step;
    bool whole;  // all of the unit's steps
    int slot = 0;
    if (SPARSE) {
        strips = lim_max < 0 ? 0 : a.count << strip_shift;
        const int steps = (strips + 1) >> 1, per = (steps + a.splits - 1) / a.splits;
        step = min((int64_t)steps, (int64_t)split * per);
        s_end = min((int64_t)steps, (int64_t)step + per);
        whole = a.splits == 1;
    } else {
        strips = (lim_max + 16) >> 4;
        const int steps = (strips + 1) >> 1;
        step = 0;
        s_end = steps;
        whole = true;
        if (a.splits > 1) {
            const int64_t u0 = before[unit], u1 = before[unit + 1];
            const int first = (int)(u0 / chunk), last = (int)((u1 - 1) / chunk);
            step = (int)(max(from, u0) - u0);
            s_end = (int)min((int64_t)steps, to - u0);
            whole = first == last;
            slot = (int)part + (int)unit;
            if (head == 0 && tid == 0 && (int)part == first)
                a.unit_parts[unit] = make_int2(first + (int)unit, last - first + 1);
        }
    }
    step += wave;

    const int32_t *table = a.table + (int64_t)(live ? b : 0) * a.cols;
    const int32_t *list = SPARSE ? a.blocks + (t0 * heads + head) * a.count : nullptr;

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
    if (wave == 0 && have) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][r] += merge[1][(4 * i + r) * 64 + lane];
        const int64_t orow = tok * ((int64_t)heads * a.group) + qhead;
        if (whole) {
            write_rows<TT, D>(acc, (elem *)a.out + orow * D, total == 0.f ? 0.f : 1.f / total, h);
            if (a.lse && h == 0) a.lse[orow] = log_of(top, total);
        } else {
            const int64_t at = SPARSE ? orow * a.splits + split
                                      : ((int64_t)head * a.slots + slot) * a.unit_rows + col;
            if (h == 0) a.part_ml[at] = make_float2(top, total);
            write_part<D>(acc, a.part + at * D, h);
        }
    }
    if (SPARSE || a.splits == 1 || (int)unit + 1 >= a.units || before[unit + 1] >= to) return;
    __syncthreads();  // the next unit writes ml and merge
    }
}

// Joins the parts of a row: WAVES waves per row take the parts in turn, lanes over
// channels; the last sum, over waves, is in their order.
enum CombineRows { kByUnit, kBySplit, kByPrompt };
template <typename TT, int ROWS, int WAVES>
__global__ __launch_bounds__(kThreads) void kv_combine_kernel(KvAttend a, int64_t rows)
{
    typedef typename TT::elem elem;
    __shared__ float4 sums[kWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int turn = wave % WAVES;
    const int64_t row = (int64_t)blockIdx.x * (kWaves / WAVES) + wave / WAVES;
    if (row >= rows) return;
    int64_t orow = row, at = row * a.splits;  // the first part, in rows of part[]
    int n = a.splits, stride = 1;
    if (ROWS == kByUnit) {
        const uint32_t x = (uint32_t)row / (uint32_t)a.c.heads, unit = x / (uint32_t)a.unit_rows;
        const uint32_t b = unit / (uint32_t)a.per_unit;
        const int head = (int)((uint32_t)row - x * (uint32_t)a.c.heads), col = (int)(x - unit * (uint32_t)a.unit_rows);
        const uint32_t r = (unit - b * (uint32_t)a.per_unit) * 16 + col;
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

template <typename TT, int D> hipError_t launch_tokens(const KvAttend &a, int64_t groups, hipStream_t s)
{
    const unsigned grid = (unsigned)(groups * a.c.heads);
    if (a.blocks)
        hipLaunchKernelGGL((kv_attend_kernel<TT, D, true>), dim3(grid), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((kv_attend_kernel<TT, D, false>), dim3(grid), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <typename TT> hipError_t launch_combine(const KvAttend &a, bool prompt, hipStream_t s)
{
    const int64_t rows = (prompt || a.blocks) ? a.T * a.group * a.c.heads : (int64_t)a.units * a.unit_rows * a.c.heads;
    const dim3 four((unsigned)rows), one((unsigned)((rows + kWaves - 1) / kWaves)), block(kThreads);
    if (prompt) hipLaunchKernelGGL((kv_combine_kernel<TT, kByPrompt, 1>), one, block, 0, s, a, rows);
    else if (a.blocks && a.splits < 16) hipLaunchKernelGGL((kv_combine_kernel<TT, kBySplit, 1>), one, block, 0, s, a, rows);
    else if (a.blocks) hipLaunchKernelGGL((kv_combine_kernel<TT, kBySplit, 4>), four, block, 0, s, a, rows);
    else hipLaunchKernelGGL((kv_combine_kernel<TT, kByUnit, 4>), four, block, 0, s, a, rows);
    return hipGetLastError();
}

template <typename TT> hipError_t launch_tokens_dim(const KvAttend &a, int64_t groups, hipStream_t s)
{
    switch (a.c.dim) {
    case 64: return launch_tokens<TT, 64>(a, groups, s);
    case 96: return launch_tokens<TT, 96>(a, groups, s);
    case 128: return launch_tokens<TT, 128>(a, groups, s);
    case 192: return launch_tokens<TT, 192>(a, groups, s);
    default: return launch_tokens<TT, 256>(a, groups, s);
    }
}

// Requests with at most this many rows go through the single-token kernel,
// 16 rows a workgroup, where others take the prompt kernel.
constexpr int64_t kSmallRows = 64;
// Tables of at most this many keys are not split: joining parts costs a launch.
constexpr int64_t kWholeKeys = 1024;

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
    if (p.tokens) {
        p.per_unit = (int)((rows + 15) / 16);
        p.unit_rows = (int)std::min<int64_t>(rows, 16);
        p.units = (count ? T : B) * p.per_unit;
        // as many workgroups as are resident at once (a further round would only begin and join again)
        const int64_t resident = (int64_t)num_cus * (c.dim <= 128 ? 2 : 1);
        if (count) {
            const int64_t most = std::max<int64_t>(1, keys / (32 * kMinSteps));
            p.token_splits = (int)std::max<int64_t>(1, std::min(resident / (p.units * c.heads), most));
        } else if (keys > kWholeKeys && p.units <= kKvMaxUnits && p.units * c.heads < 16 * (int64_t)num_cus) {
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
        if (units < num_cus) {
            const int64_t most = std::max<int64_t>(1, keys / 256);
            p.prompt_splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(2 * (int64_t)num_cus / units, most), 32));
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
    return a.c.bf16 ? launch_tokens_dim<KvBf16>(a, groups, s) : launch_tokens_dim<KvF16>(a, groups, s);
}

hipError_t launch_kv_combine(const KvAttend &a, bool prompt, hipStream_t s)
{
    return a.c.bf16 ? launch_combine<KvBf16>(a, prompt, s) : launch_combine<KvF16>(a, prompt, s);
}

}  // namespace ivf
