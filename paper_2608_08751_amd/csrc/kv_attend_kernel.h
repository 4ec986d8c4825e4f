// Attention of up to 16 query rows of one key/value head over the 4-bit cache.
//
// A row's output is sum_j p_j v_j / sum_j p_j with p_j = exp2(t_j - r), t_j = scale
// log2(e) q.k_j and a reference r that follows the running maximum of t.
//   * scores: S^T = K Q^T with 16 keys (a strip) as rows, on
//     v_mfma_scale_f32_16x16x128_f8f6f4: 32 channels of 4-bit codes with a power of two
//     are its A operand as they lie in memory, 16 bytes of codes and a scale byte a lane.
//     The query is the sum of four 6-bit numbers a channel with a power of two per
//     32 channels: digits of a fixed-point number, off by 2^-19 of the largest of the 32 at
//     most (numbers of 8 significant bits: exact down to 2^-11 of it, of 11 bits to 2^-8). A choice: keys
//     decoded to 16 bits would take the query as it is (the prompt kernel's do), at four vector
//     instructions more for 8 channels of a key; scores are off by 2e-7 of sum |q k|, far less than the
//     probabilities' rounding.
//   * values: O^T = V^T P^T on v_mfma_f32_16x16x32. The results above are the B operand as
//     they are: lane (r, h)'s eight probabilities of two strips are keys 4 h ... 4 h + 3 of each.
//     It reads the codes of neighbouring channels of those keys, v_cvt_scalef32 makes pairs of
//     channels with the key's scale, v_perm_b32 pairs of keys. Probabilities are rounded to the
//     cache's type, which is what this product takes; a second product with what the rounding leaves
//     would double the matrix work of the values and take away a sixth of the error (relative to fp64:
//     bf16 0.0020, of which the outputs' own rounding alone makes 0.0017; f16 0.00026 and 0.00021). The sum of
//     the probabilities is of the unrounded ones.
//   * with selected blocks and up to 8 rows (PACK), which leave half of the 16 columns free,
//     column r + 8 is row r again: columns below 8 take the exponentials of the first strip of a
//     step and the others those of the second, each with a reference, sum and output of its
//     own, joined at the end. 512 tokens x 8 heads over 24 blocks of 64 keys, with it and without, caches cold:
//     64, 96, 128, 192, 256 channels 81.3 and 84.9, 104 and 108, 99.7 and 102, 210 and 214, 238 and 245 us; 32 single
//     tokens over 64 blocks: 38.8 and 36.6, 52.2 and 49.0, 66.3 and 65.5, 89.1 and 92.2, 112 and 115 us. Whole contexts
//     are bound by memory, and the joining costs more than it gives: one request of 700 keys x 128 channels
//     10.6 us with it, 9.6 without.
//   * the reference is raised only when a lane's probabilities of a step sum to more than
//     2^14, for all rows of the wave at once, so the common step needs no maximum
//     and no exchange between lanes. Probabilities carry 2^8, which keeps small ones normal in f16.
// Masked scores are replaced, not added to; values of keys that no row sees get scale
// 1, so that nothing left in unused slots reaches a sum.
//
// A team of 1, 4 or 8 waves takes a range of steps of 32 keys, each wave every 1st, 4th or 8th
// step with its own reference, sums and output, joined in LDS. What bounds single tokens is
// the read of the cache, 17 / 16 bytes per channel of key and value: 64 requests of up to 32,000
// tokens, 8 heads x 128, 912 MB: 173 us with the joining, 5.3 TB/s (a plain read of 8 GB 6.0; calls one after the
// other 186 us and 8). 256 channels hold one wave a SIMD, with accumulation registers to spill into: 949 MB 222 us
// and 7. Many tokens with
// blocks of their own are bound by the decoding of values, a vector instruction a value with its
// share of scales, 1/4 of which serve a query row where a group is four rows: 2,048
// tokens x 8 heads over 24 blocks of 64 keys 286 us (calls one after the other 343), vector units 77 % and matrix
// units 29 % busy, 11 TB/s from L2. Its launch bound of three waves a SIMD costs one or two spilled registers at
// 128 channels.
//
// With terms in the scores (kv_terms.h) steps that no row of the unit sees are left out, and a step whose keys all rows
// see takes no masks. 64 single tokens of up to 32,000, variants in turn: 173 us without terms, 184 with a bias or a
// prefix, 196 with a cap, 200 with cap and bias: the cache's read does not hide the terms wholly. 32 windows of 4,096
// keys in contexts of up to 50,000, capped, 143 MB: 40 us (3.6 TB/s) and 5 to join. Selected blocks: 32 single tokens x 8 heads
// over 64 blocks of 64 keys 27 us, with a bias 27, a cap 29, all terms 29; 2,048 tokens over 24 blocks 311, with a bias 429, a
// cap 457 (two waves a SIMD, three without terms), the blocks that lie in windows of 30,000 keys alone 267, those with all terms 294.
#pragma once

#include "kv.h"
#include "kv_strip.h"
#include "kv_terms.h"

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
template <typename Terms> __device__ int64_t unit_steps(const KvAttend &a, const Terms &terms, uint32_t u, int unit, int last_key)
{
    const uint32_t b = u / (uint32_t)a.per_unit;
    const int64_t r0 = (int64_t)(u - b * (uint32_t)a.per_unit) * unit;
    const int64_t t0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
    const int64_t rows = (min(max((int64_t)a.start[b + 1], t0), a.T) - t0) * a.group;
    if (r0 >= rows || rows > a.small_rows) return 0;
    const int64_t r1 = min(r0 + unit, rows) - 1;
    if constexpr (has_terms<Terms>) {
        KvSights all;
        for (int64_t t = t0 + (uint32_t)r0 / (uint32_t)a.group; t <= t0 + (uint32_t)r1 / (uint32_t)a.group; ++t)
            all.add(KvSight::of(a, terms, t, true, last_key));
        return max(1, KvSteps::of<5>(all.prefix_max, all.first_min, all.pos_max).count);
    }
    int lim = -1;
    for (int64_t t = t0 + (uint32_t)r0 / (uint32_t)a.group; t <= t0 + (uint32_t)r1 / (uint32_t)a.group; ++t)
        lim = max(lim, min(a.position[t], last_key));
    return max(1, (lim >> 5) + 1);
}

constexpr int attend_threads(int team) { return team == 1 ? kThreads : 64 * team; }

template <typename TT, int D, bool SPARSE, bool PACK, int TEAM, typename Terms>
__global__ __launch_bounds__(attend_threads(TEAM), D > 128 ? 1 : SPARSE && TEAM < 8 && D != 96 && !has_terms<Terms> ? 3 : 2)
void kv_attend_kernel(KvAttend a, Terms terms)
{
    constexpr bool TERMS = has_terms<Terms>;
    typedef Pieces<D> P;
    typedef typename TT::elem elem;
    constexpr int kTiles = D / 16, kUnit = PACK ? 8 : 16;
    constexpr int kQueryBytes = CodedQuery<TT, D>::bytes(kUnit), kMergeBytes = TEAM / 2 * kTiles * 4 * 64 * 4;
    // TEAM waves share a unit: several join their results in LDS, one needs it for its query only
    __shared__ __align__(16) uint8_t room[TEAM == 1 ? kWaves * kQueryBytes : kQueryBytes > kMergeBytes ? kQueryBytes : kMergeBytes];
    __shared__ float2 ml[TEAM][16];
    __shared__ int64_t before[SPARSE ? 1 : kKvMaxUnits + 1];  // steps of the units before
    __shared__ int64_t wave_steps[TEAM];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, h = lane >> 4;
    const int place = PACK ? col & 7 : col;  // the lane's row of the unit
    const bool second = PACK && col >= 8;    // and the strip of a step whose scores it takes
    const uint32_t heads = a.c.heads, bid = blockIdx.x, part = bid / heads;
    const int head = (int)(bid - part * heads);
    const int last_key = (int)min((int64_t)a.cols << a.c.shift, (int64_t)INT32_MAX) - 1;
    const int strip_shift = a.c.shift - 4, strip_mask = (1 << strip_shift) - 1;
    const size_t rec_bytes = a.c.rec_bytes();
    typename CodedKeys<D>::Offsets k_offs(lane, a.c.bs);
    typename Values<D>::Offsets v_offs(lane, a.c.bs);

    uint32_t unit = part;
    int split = 0;
    int64_t from = 0, to = INT64_MAX, chunk = 0;  // this workgroup's steps, counted over all units
    if (SPARSE && TEAM == 1) {
        unit = part * kWaves + wave;
        if (unit >= (uint32_t)a.units) return;
    } else if (SPARSE) {
        unit = part / (uint32_t)a.splits;
        split = (int)(part - unit * (uint32_t)a.splits);
    } else if (a.splits > 1) {
        constexpr int kPer = kKvMaxUnits / (64 * TEAM);
        const int per = (a.units + 64 * TEAM - 1) / (64 * TEAM);  // units of a thread: one, as long as that reaches
        int64_t mine[kPer], all = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t u = tid * per + i;
            mine[i] = all;
            if (i < per && u < (uint32_t)a.units) all += unit_steps(a, terms, u, kUnit, last_key);
        }
        int64_t up = all;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t x = __shfl_up(up, d);
            if (lane >= d) up += x;
        }
        if (lane == 63) wave_steps[wave % TEAM] = up;
        __syncthreads();
        int64_t base = up - all, total = 0;
        for (int w = 0; w < TEAM; ++w) {
            if (w < wave) base += wave_steps[w];
            total += wave_steps[w];
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i < per && tid * per + i < a.units) before[tid * per + i] = base + mine[i];
        if (tid == 0) before[a.units] = total;
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
            r0 = (int)(unit % (uint32_t)a.per_unit) * kUnit;
            rows_here = min(kUnit, a.group - r0);
            b = a.request[t0];
        } else {
            b = (int)(unit / (uint32_t)a.per_unit);
            r0 = (int)(unit % (uint32_t)a.per_unit) * kUnit;
            t0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
            const int64_t rows = (min(max((int64_t)a.start[b + 1], t0), a.T) - t0) * a.group;
            if (r0 >= rows || rows > a.small_rows) {
                if (a.splits == 1 || (int)unit + 1 >= a.units || before[unit + 1] >= to) return;
                continue;
            }
            rows_here = (int)min((int64_t)a.unit_rows, rows - r0);  // never more than part[] has room for
        }
        const bool live = b >= 0 && b < a.B;

        typename CodedQuery<TT, D>::template Stage<64 * TEAM, kUnit> stage;
        const int team_tid = TEAM == 1 ? lane : tid;
        stage.load(team_tid, rows_here, [&](int r) {
            const uint32_t x = r0 + r, t = x / (uint32_t)a.group;
            return (const elem *)a.q.p + (t0 + t) * a.q.ts + (int64_t)(head * a.group + (int)(x - t * (uint32_t)a.group)) * a.q.hs;
        });

        // this lane's row
        const bool have = place < rows_here;
        const uint32_t row = r0 + (have ? place : 0), row_tok = row / (uint32_t)a.group;
        const int lim = live ? min(a.position[t0 + row_tok], last_key) : -1;
        int lim_max = have ? lim : -1, lim_min = have ? lim : INT32_MAX;
        // what this lane's row and the unit's rows see, and the row's bias by distance
        KvSight mine = {-1, 0, 0};
        KvSights seen;
        KvSteps ranges = {0, 0, 0};
        int pos = 0;
        float slope = 0.f;
        if constexpr (TERMS) {
            mine = KvSight::of(a, terms, t0 + row_tok, live, last_key);
            if (have) seen.add(mine);
            seen.join_columns();
            ranges = KvSteps::of<5>(seen.prefix_max, seen.first_min, seen.pos_max);
            lim_max = seen.last();
            if (terms.slopes) {
                pos = a.position[t0 + row_tok];
                slope = slope_of(terms, head * a.group + (int)(row - row_tok * (uint32_t)a.group));
            }
        } else {
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) {
                lim_max = max(lim_max, __shfl_xor(lim_max, d));
                lim_min = min(lim_min, __shfl_xor(lim_min, d));
            }
            lim_max = __builtin_amdgcn_readfirstlane(lim_max);
            lim_min = __builtin_amdgcn_readfirstlane(lim_min);
        }

        // the steps of 32 keys of this part, wave by wave
        int strips, s_end, step, all_steps;
        bool whole;  // all of the unit's steps
        int slot = 0;
        if (SPARSE) {
            strips = lim_max < 0 ? 0 : a.count << strip_shift;
            const int steps = (strips + 1) >> 1, per = (steps + a.splits - 1) / a.splits;
            all_steps = steps;
            step = min((int64_t)steps, (int64_t)split * per);
            s_end = min((int64_t)steps, (int64_t)step + per);
            whole = a.splits == 1;
        } else {
            strips = (lim_max + 16) >> 4;
            const int steps = TERMS ? ranges.count : (strips + 1) >> 1;
            all_steps = steps;
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
        if (TEAM > 1) step += wave;

        const int32_t *table = a.table + (int64_t)(live ? b : 0) * a.cols;
        const int32_t *list = SPARSE ? a.blocks + (t0 * heads + head) * a.count : nullptr;

        // lane 2 i + s keeps, of strip s of the wave's i-th next step, the record (bytes
        // from the first) and the first key, or -1 where there is none
        uint32_t rec_lo = 0, rec_hi = 0;
        int keys = -1, ahead = 0;
        auto look = [&](int first_step) {
            const int64_t st = (int64_t)first_step + (lane >> 1) * TEAM;
            int64_t at = st;
            if constexpr (TERMS) {
                // with a bias the nearest keys come first: scores that grow from step to step would raise the
                // reference, and rescale all sums, again and again
                if (terms.slopes) at = all_steps - 1 - st;
                if (!SPARSE && st < s_end) at = ranges.at((int)at);
            }
            const int64_t v = 2 * at + (lane & 1);
            rec_lo = rec_hi = 0;
            keys = -1;
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
                if (j >= 0 && j < a.cols && (TERMS ? seen.any(base, 16) : base <= lim_max)) {
                    const int id = table[j];
                    if (id >= 0 && id < a.c.blocks) {
                        const uint64_t off = ((uint64_t)(uint32_t)id * heads + (uint32_t)head) * rec_bytes;
                        rec_lo = (uint32_t)off;
                        rec_hi = (uint32_t)(off >> 32);
                        keys = base;
                    }
                }
            }
        };
        struct Pair {
            CodedKeys<D> k[2];
            Values<D> v[2];
            int key[2];
        };
        auto fetch = [&](Pair &x, int at_step) {
            if (ahead == 32) {
                look(at_step);
                ahead = 0;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) x.key[e] = __builtin_amdgcn_readlane(keys, 2 * ahead + e);
            if ((x.key[0] & x.key[1]) >= 0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)rec_hi, 2 * ahead + e) << 32 |
                                         (uint32_t)__builtin_amdgcn_readlane((int)rec_lo, 2 * ahead + e);
                    const StripBase base = StripBase::at<D>(a.c.rec + off, (max(x.key[e], 0) >> 4) & strip_mask);
                    x.k[e].load(base, k_offs);
                    x.v[e].load(base, v_offs);
                }
            }
            ++ahead;
        };
        Pair x, y;
        const bool any = step < s_end;
        if (any) {
            look(step);
            fetch(x, step);
        }
        uint8_t *staged = room + (TEAM == 1 ? wave * kQueryBytes : 0);
        stage.store(team_tid, rows_here, staged, a.q_flip);
        if (TEAM > 1) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        CodedQuery<TT, D> query;
        query.load(staged, kUnit, place, h);

        f32x4 acc[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        float ref = -INFINITY, sub = 0.f, sum = 0.f;
        auto work = [&](const Pair &z) {
            if ((z.key[0] & z.key[1]) < 0) return;  // neither strip is there
            f32x4 st[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) st[e] = query.scores(z.k[e]);
            float vs[P::n][2][4];
#pragma unroll
            for (int c = 0; c < P::n; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e) four_scales(z.v[e].vs[c], vs[c][e]);
            constexpr int kOwn = PACK ? 4 : 8;  // scores of this lane
            float t[kOwn];
#pragma unroll
            for (int i = 0; i < kOwn; ++i) t[i] = PACK ? (second ? st[1][i] : st[0][i]) : st[i / 4][i % 4];
            if constexpr (TERMS) {
                scale_scores(t, a.scale, terms);
                if (terms.slopes) {
#pragma unroll
                    for (int e = 0; e < kOwn / 4; ++e) {
                        const int key = (PACK ? (second ? z.key[1] : z.key[0]) : z.key[e]) + 4 * h;
                        const float apart = (float)(pos - key);  // above 2^24 rounded, as the bias is
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            t[4 * e + i] = __builtin_fmaf(-slope, fabsf(apart - (float)i), t[4 * e + i]);
                    }
                }
            }
            if (TERMS ? (z.key[0] | z.key[1]) < 0 || !seen.all(z.key[0], 16) || !seen.all(z.key[1], 16) : (z.key[0] | z.key[1]) < 0 || max(z.key[0], z.key[1]) + 15 > lim_min) {
                int key[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    key[e] = z.key[e] < 0 ? INT32_MAX - 3 : z.key[e] + 4 * h;  // a strip that is not there: past every position
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < P::n; ++c)
                            if (TERMS ? seen.nobody(key[e] + i) : key[e] + i > lim_max) vs[c][e][i] = 1.f;
                }
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const int at = (PACK ? (second ? key[1] : key[0]) : key[i / 4]) + i % 4;
                    if (TERMS ? !mine.sees(at) : at > lim) t[i] = -INFINITY;
                }
            }
            float p[kOwn], part_sum;
            auto probabilities = [&]() {
                part_sum = 0.f;
#pragma unroll
                for (int i = 0; i < kOwn; i += 2) {
                    // (terms leave scores to the base 2)
                    p[i] = exp2_fast(TERMS ? t[i] - sub : __builtin_fmaf(t[i], a.scale, -sub));
                    p[i + 1] = exp2_fast(TERMS ? t[i + 1] - sub : __builtin_fmaf(t[i + 1], a.scale, -sub));
                    part_sum += p[i] + p[i + 1];
                }
            };
            probabilities();
            if (__ballot(part_sum > kMost || ref == -INFINITY)) {
                float mx = t[0];
#pragma unroll
                for (int i = 1; i < kOwn; ++i) mx = fmaxf(mx, t[i]);
                const float top = fmaxf(ref, max_over_h(TERMS ? mx : mx * a.scale));
                const float f = ref == top ? 1.f : exp2_fast(ref - top);
                ref = top;
                sub = top == -INFINITY ? 0.f : top - kCarry;
                sum *= f;
#pragma unroll
                for (int i = 0; i < kTiles; ++i) acc[i] *= f;
                probabilities();
            }
            sum += part_sum;
            uint32_t w[kOwn / 2];
#pragma unroll
            for (int i = 0; i < kOwn; i += 2) w[i / 2] = TT::pack(p[i], p[i + 1]);
            u32x4 pf;
            if (PACK) {
                const uint32_t m1 = second ? ~0u : 0u;
                pf = (u32x4){w[0] & ~m1, w[1] & ~m1, w[0] & m1, w[1] & m1};
            } else {
                pf = (u32x4){w[0], w[1], w[kOwn / 2 - 2], w[kOwn / 2 - 1]};
            }
            auto piece = [&](auto piece_c) {
                constexpr int c = decltype(piece_c)::value, S = P::size(c);
                u32x2 v0[S / 16], v1[S / 16];
                value_operands<TT, S>(z.v[0].v[c], vs[c][0], v0);
                value_operands<TT, S>(z.v[1].v[c], vs[c][1], v1);
#pragma unroll
                for (int j = 0; j < S / 16; ++j) {
                    const u32x4 v = {v0[j][0], v0[j][1], v1[j][0], v1[j][1]};
                    acc[P::off(c) / 16 + j] = TT::mfma(v, pf, acc[P::off(c) / 16 + j]);
                }
            };
            piece(std::integral_constant<int, 0>());
            if constexpr (P::n > 1) piece(std::integral_constant<int, 1>());
        };
        while (any) {
            step += TEAM;
            if (step < s_end) fetch(y, step);
            work(x);
            if (step >= s_end) break;
            step += TEAM;
            if (step < s_end) fetch(x, step);
            work(y);
            if (step >= s_end) break;
        }

        // join the waves (and halves of the columns): sums times exp2(ref - max)
        sum = sum_over_h(sum);
        float top, total = 0.f;
        auto add = [&](float r, float s) {
            if (r > -INFINITY || s != 0.f) total += s * exp2_fast(r - top);
        };
        if (TEAM == 1) {
            const float r2 = PACK ? other_half(ref) : -INFINITY, s2 = PACK ? other_half(sum) : 0.f;
            top = fmaxf(ref, r2);
            add(second ? r2 : ref, second ? s2 : sum);
            add(second ? ref : r2, second ? sum : s2);
        } else {
            if (h == 0) ml[wave % TEAM][col] = make_float2(ref, sum);
            __syncthreads();
            top = -INFINITY;
#pragma unroll
            for (int w = 0; w < TEAM; ++w) {
                top = fmaxf(top, ml[w][col].x);
                if (PACK) top = fmaxf(top, ml[w][col ^ 8].x);
            }
#pragma unroll
            for (int w = 0; w < TEAM; ++w) {
                add(ml[w][place].x, ml[w][place].y);
                if (PACK) add(ml[w][place + 8].x, ml[w][place + 8].y);
            }
        }
        const float f = ref > -INFINITY ? exp2_fast(ref - top) : sum != 0.f ? sum : 0.f;
#pragma unroll
        for (int i = 0; i < kTiles; ++i) acc[i] *= f;
        if (TEAM > 1) {
            float(*merge)[kTiles * 4 * 64] = (float(*)[kTiles * 4 * 64])room;
            // halving: the upper half of the waves that are left hand theirs down
#pragma unroll
            for (int half = TEAM / 2; half >= 1; half /= 2) {
                if (wave >= half && wave < 2 * half) {
#pragma unroll
                    for (int i = 0; i < kTiles; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) merge[wave - half][(4 * i + r) * 64 + lane] = acc[i][r];
                }
                __syncthreads();
                if (wave < half) {
#pragma unroll
                    for (int i = 0; i < kTiles; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[i][r] += merge[wave][(4 * i + r) * 64 + lane];
                }
                if (half > 1) __syncthreads();
            }
        }
        if (TEAM == 1 || wave == 0) {
            if (PACK) {
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][r] += other_half(acc[i][r]);
            }
            if (have && !second) {
                const int64_t orow = ((t0 + row_tok) * heads + head) * a.group + (row - row_tok * (uint32_t)a.group);
                if (whole) {
                    write_rows<TT, D>(acc, (elem *)a.out + orow * D, total == 0.f ? 0.f : 1.f / total, h);
                    if (a.lse && h == 0) a.lse[orow] = log_of(top, total);
                } else {
                    const int64_t at = SPARSE ? orow * a.splits + split
                                              : ((int64_t)head * a.slots + slot) * a.unit_rows + place;
                    if (h == 0) a.part_ml[at] = make_float2(top, total);
                    write_part<D>(acc, a.part + at * D, h);
                }
            }
        }
        if (SPARSE || a.splits == 1 || (int)unit + 1 >= a.units || before[unit + 1] >= to) return;
        __syncthreads();  // the next unit writes room and ml
    }
}

template <typename TT, int D, bool SPARSE, int TEAM, typename Terms>
hipError_t launch_team(const KvAttend &a, const Terms &terms, int64_t groups, hipStream_t s)
{
    const dim3 grid((unsigned)(groups * a.c.heads)), block(attend_threads(TEAM));
    if (SPARSE && a.unit_size == 8) hipLaunchKernelGGL((kv_attend_kernel<TT, D, SPARSE, SPARSE, TEAM, Terms>), grid, block, 0, s, a, terms);
    else hipLaunchKernelGGL((kv_attend_kernel<TT, D, SPARSE, false, TEAM, Terms>), grid, block, 0, s, a, terms);
    return hipGetLastError();
}

template <typename TT, int D, typename Terms> hipError_t launch_tokens(const KvAttend &a, const Terms &terms, int64_t groups, hipStream_t s)
{
    if (a.team == 1) return launch_team<TT, D, true, 1, Terms>(a, terms, (groups + kWaves - 1) / kWaves, s);
    if constexpr (D <= 128)
        if (a.team == 8)
            return a.blocks ? launch_team<TT, D, true, 8, Terms>(a, terms, groups, s) : launch_team<TT, D, false, 8, Terms>(a, terms, groups, s);
    return a.blocks ? launch_team<TT, D, true, 4, Terms>(a, terms, groups, s) : launch_team<TT, D, false, 4, Terms>(a, terms, groups, s);
}

template <typename TT, typename Terms> hipError_t launch_tokens_dim(const KvAttend &a, const Terms &terms, int64_t groups, hipStream_t s)
{
    switch (a.c.dim) {
    case 64: return launch_tokens<TT, 64, Terms>(a, terms, groups, s);
    case 96: return launch_tokens<TT, 96, Terms>(a, terms, groups, s);
    case 128: return launch_tokens<TT, 128, Terms>(a, terms, groups, s);
    case 192: return launch_tokens<TT, 192, Terms>(a, terms, groups, s);
    default: return launch_tokens<TT, 256, Terms>(a, terms, groups, s);
    }
}

}  // namespace
}  // namespace ivf
