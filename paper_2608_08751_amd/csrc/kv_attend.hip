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
#include "kv_types.h"

#include <algorithm>

namespace ivf {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kRaise = 6.f;  // a score may pass the reference by this much
constexpr float kCarry = 8.f;  // probabilities are times 2^kCarry
constexpr int kMinSteps = 8;   // steps of 32 keys that a part is worth

// A row of channels is taken as one or two pieces of 128, 64 or 32.
template <int D> struct Pieces {
    static constexpr int first = D >= 128 ? 128 : 64, second = D - first;
    static constexpr int n = second ? 2 : 1;
    static constexpr int size(int c) { return c == 0 ? first : second; }
    static constexpr int off(int c) { return c == 0 ? 0 : first; }
};

// One strip of 16 keys and values of a head, as a lane holds it.
template <int D> struct Strip {
    uint32_t k[D / 32];
    uint32_t ks[Pieces<D>::n];
    uint32_t v[Pieces<D>::n][4];
    u32x4 vs[Pieces<D>::n];
};

// A lane's offsets into the four parts of a strip, whose first bytes are uniform
// over the wave (scalar base, 32-bit lane offset).
template <int D> struct LaneOffsets {
    uint32_t k[Pieces<D>::n], ks[Pieces<D>::n], v[Pieces<D>::n], vs[Pieces<D>::n];
    __device__ __forceinline__ LaneOffsets(int lane, int bs)
    {
        typedef Pieces<D> P;
        const int m = lane & 15, h = lane >> 4, key = 4 * (m & 3) + (m >> 2);
#pragma unroll
        for (int c = 0; c < P::n; ++c) {
            const int S = P::size(c), off = P::off(c), g = off / 32;
            k[c] = key * (D / 2) + off / 2 + S / 8 * h;
            ks[c] = key * (D / 32) + g + (S == 128 ? h : S == 64 ? h >> 1 : 0);
            v[c] = h * (D / 2) + off / 2 + m * S / 32;
            vs[c] = (g + (S == 128 ? m >> 2 : S == 64 ? m >> 3 : 0)) * bs;
        }
    }
};

template <int D>
__device__ __forceinline__ void load_strip(Strip<D> &s, const uint8_t *rec, int bs, int strip, const LaneOffsets<D> &o)
{
    typedef Pieces<D> P;
    const uint8_t *kr = rec + strip * (16 * (D / 2));
    const uint8_t *vr = kr + bs * (D / 2);
    const uint8_t *ksr = rec + bs * D + strip * (16 * (D / 32));
    const uint8_t *vsr = rec + bs * (D + D / 32) + strip * 16;
#pragma unroll
    for (int c = 0; c < P::n; ++c) {
        const int S = P::size(c), g = P::off(c) / 32;
        s.ks[c] = *(ksr + o.ks[c]);
        s.vs[c] = *(const u32x4 *)(vsr + o.vs[c]);
        if (S == 128) {
            const u32x4 x = *(const u32x4 *)(kr + o.k[c]);
#pragma unroll
            for (int i = 0; i < 4; ++i) s.k[g + i] = x[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) s.v[c][i] = *(const uint32_t *)(vr + o.v[c] + 4 * i * (D / 2));
        } else if (S == 64) {
            const u32x2 x = *(const u32x2 *)(kr + o.k[c]);
            s.k[g] = x[0];
            s.k[g + 1] = x[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) s.v[c][i] = *(const uint16_t *)(vr + o.v[c] + 4 * i * (D / 2));
        } else {
            s.k[g] = *(const uint32_t *)(kr + o.k[c]);
#pragma unroll
            for (int i = 0; i < 4; ++i) s.v[c][i] = *(vr + o.v[c] + 4 * i * (D / 2));
        }
    }
}

template <typename TT> __device__ __forceinline__ u32x4 decode8(uint32_t w, float scale)
{
    return (u32x4){TT::template decode<0>(w, scale), TT::template decode<1>(w, scale), TT::template decode<2>(w, scale),
                   TT::template decode<3>(w, scale)};
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

__device__ __forceinline__ float max_over_h(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_h(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The rows of one workgroup: rows r0 ... r0 + n of a request's (or token's) rows,
// row = token * group + head of the group.
struct RowSet {
    int64_t t0;  // token of row 0
    int r0, n;
    int b;
};

template <typename TT, int D, bool SPARSE>
__global__ __launch_bounds__(kThreads) void kv_attend_kernel(KvAttend a, int per_unit)
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
        rs.t0 = unit / per_unit;
        rs.r0 = (int)(unit % per_unit) * 16;
        rs.n = min(16, a.group - rs.r0);
        rs.b = a.request[rs.t0];
    } else {
        rs.b = (int)(unit / per_unit);
        rs.r0 = (int)(unit % per_unit) * 16;
        const int64_t t0 = min(max((int64_t)a.start[rs.b], (int64_t)0), a.T);
        const int64_t t1 = min(max((int64_t)a.start[rs.b + 1], t0), a.T);
        rs.t0 = t0;
        const int64_t rows = (t1 - t0) * a.group;
        if (rs.r0 >= rows) return;
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
                qf[P::off(c) / 32 + d] = x;
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
        float vs[P::n][8];
#pragma unroll
        for (int c = 0; c < P::n; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) vs[c][i] = kv_scale((x.s[i / 4].vs[c][i % 4] >> (8 * h)) & 255u);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (x.page[e] < 0 || x.base[e] + 15 > lim_min) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = x.page[e] < 0 ? INT32_MAX : x.base[e] + 4 * i + h;
                    if (key > lim) t[4 * e + i] = -INFINITY;
#pragma unroll
                    for (int c = 0; c < P::n; ++c)
                        if (key > lim_max) vs[c][4 * e + i] = 1.f;
                }
            }
        }
        const float mx = fmaxf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])), fmaxf(fmaxf(t[4], t[5]), fmaxf(t[6], t[7])));
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
#pragma unroll
        for (int c = 0; c < P::n; ++c) {
            const int S = P::size(c);
            uint32_t pair[8][4];  // [key][channel pair]
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t w = x.s[i / 4].v[c][i % 4];
                pair[i][0] = TT::template decode<0>(w, vs[c][i]);
                if (S >= 64) pair[i][1] = TT::template decode<1>(w, vs[c][i]);
                if (S >= 128) {
                    pair[i][2] = TT::template decode<2>(w, vs[c][i]);
                    pair[i][3] = TT::template decode<3>(w, vs[c][i]);
                }
            }
#pragma unroll
            for (int p = 0; p < S / 32; ++p) {
                u32x4 lo, hi;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lo[i] = low_halves(pair[2 * i][p], pair[2 * i + 1][p]);
                    hi[i] = high_halves(pair[2 * i][p], pair[2 * i + 1][p]);
                }
                const int tile = P::off(c) / 16 + 2 * p;
                acc[tile] = TT::mfma(lo, pf, acc[tile]);
                acc[tile + 1] = TT::mfma(hi, pf, acc[tile + 1]);
            }
        }
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
        const float inv = total == 0.f ? 0.f : 1.f / total;
        elem *o = (elem *)a.out + orow * D;
#pragma unroll
        for (int c = 0; c < P::n; ++c) {
            const int S = P::size(c), tile0 = P::off(c) / 16;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < S / 16; j += 2)
                    *(uint32_t *)(o + P::off(c) + S / 4 * h + S / 16 * r + j) =
                        TT::pack(acc[tile0 + j][r] * inv, acc[tile0 + j + 1][r] * inv);
        }
        if (a.lse && h == 0)
            a.lse[orow] = total == 0.f ? -INFINITY : (top - kCarry + __builtin_amdgcn_logf(total)) * 0.69314718056f;
    } else {
        const int64_t at = orow * a.splits + split;
        if (h == 0) a.part_ml[at] = make_float2(top, total);
        float *o = a.part + at * D;
#pragma unroll
        for (int c = 0; c < P::n; ++c) {
            const int S = P::size(c), tile0 = P::off(c) / 16;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < S / 16; j += 2)
                    *(float2 *)(o + P::off(c) + S / 4 * h + S / 16 * r + j) =
                        make_float2(acc[tile0 + j][r], acc[tile0 + j + 1][r]);
        }
    }
}

// Joins the parts of a row: a wave per row, lanes over channels.
template <typename TT>
__global__ __launch_bounds__(kThreads) void kv_combine_kernel(KvAttend a)
{
    typedef typename TT::elem elem;
    const int lane = threadIdx.x & 63;
    const int64_t heads = (int64_t)a.c.heads * a.group;
    const int64_t row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (row >= a.T * heads) return;
    if (!a.blocks) {
        const int64_t t = row / heads;
        if (t < a.start[0] || t >= a.start[a.B]) return;
    }
    const float2 *ml = a.part_ml + row * a.splits;
    float top = -INFINITY;
    for (int s = lane; s < a.splits; s += 64) top = fmaxf(top, ml[s].x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    float total = 0.f;
    float2 o[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    for (int s = 0; s < a.splits; ++s) {
        const float2 x = ml[s];
        if (x.y == 0.f) continue;  // a part without keys
        const float f = x.x > -INFINITY ? exp2_fast(x.x - top) : x.y;
        total += x.y * f;
        const float *p = a.part + (row * a.splits + s) * a.c.dim;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int d = 2 * (lane + 64 * i);
            if (d < a.c.dim) {
                const float2 y = *(const float2 *)(p + d);
                o[i].x += y.x * f;
                o[i].y += y.y * f;
            }
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int d = 2 * (lane + 64 * i);
        if (d < a.c.dim) *(uint32_t *)((elem *)a.out + row * a.c.dim + d) = TT::pack(o[i].x * inv, o[i].y * inv);
    }
    if (a.lse && lane == 0)
        a.lse[row] = total == 0.f ? -INFINITY : (top - kCarry + __builtin_amdgcn_logf(total)) * 0.69314718056f;
}

template <typename TT, int D> hipError_t launch_attend(const KvAttend &a, int64_t longest, hipStream_t s)
{
    const int per = (int)(a.blocks ? (a.group + 15) / 16 : (longest * a.group + 15) / 16);
    const int64_t units = (a.blocks ? a.T : a.B) * per;
    const unsigned grid = (unsigned)(units * a.splits * a.c.heads);
    if (a.blocks)
        hipLaunchKernelGGL((kv_attend_kernel<TT, D, true>), dim3(grid), dim3(kThreads), 0, s, a, per);
    else
        hipLaunchKernelGGL((kv_attend_kernel<TT, D, false>), dim3(grid), dim3(kThreads), 0, s, a, per);
    return hipGetLastError();
}

template <typename TT> hipError_t launch_attend_dim(const KvAttend &a, int64_t longest, hipStream_t s)
{
    switch (a.c.dim) {
    case 64: return launch_attend<TT, 64>(a, longest, s);
    case 96: return launch_attend<TT, 96>(a, longest, s);
    case 128: return launch_attend<TT, 128>(a, longest, s);
    case 192: return launch_attend<TT, 192>(a, longest, s);
    default: return launch_attend<TT, 256>(a, longest, s);
    }
}

}  // namespace

int kv_attend_splits(int heads, int group, int64_t T, int64_t B, int64_t keys, int64_t longest, bool sparse,
                     int num_cus)
{
    const int64_t units = (sparse ? T * ((group + 15) / 16) : B * ((longest * group + 15) / 16)) * heads;
    const int64_t most = std::max<int64_t>(1, keys / (32 * kMinSteps));
    const int64_t want = ((int64_t)num_cus * 8 + units - 1) / units;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, most), 128));
}

hipError_t launch_kv_attend(const KvAttend &a, int64_t longest, hipStream_t s)
{
    return a.c.bf16 ? launch_attend_dim<KvBf16>(a, longest, s) : launch_attend_dim<KvF16>(a, longest, s);
}

hipError_t launch_kv_combine(const KvAttend &a, hipStream_t s)
{
    const int64_t rows = a.T * a.c.heads * a.group;
    const unsigned grid = (unsigned)((rows + kWaves - 1) / kWaves);
    if (a.c.bf16)
        hipLaunchKernelGGL((kv_combine_kernel<KvBf16>), dim3(grid), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((kv_combine_kernel<KvF16>), dim3(grid), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace ivf
