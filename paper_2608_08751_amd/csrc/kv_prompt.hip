// Attention of many query rows per request (prompts) over the 4-bit cache.
//
// The formulas and operand layouts are those of the single-token kernel
// (kv_strip.h), with the keys decoded to 16 bits and 16 CT query rows a wave: a tile of
// keys (a strip of 16 a wave) is decoded once per workgroup, laid into LDS as the MFMA
// operands that all waves read (16 bytes a lane, no bank conflicts), and every operand
// serves CT products. The rows are the batch's rows one after the other (token, head
// of the group), so that no row of the matrix units is idle; where a workgroup's rows
// span requests it takes these in turn, the others' rows masked. Two buffers: while a
// tile is computed on, the next one's codes, loaded a tile before, are decoded into the other.
//
// Bound by the matrix products beside the vector instructions of the softmax (7 issue
// slots a score, four of them the exponential): 64 keys x 32 rows x 128 channels
// take 64 products of 16 cycles and about 340 vector issues of 4 (46 % and 48 % of the
// time, hardly at once). 2,048 tokens after
// 8,192, 32 query heads on 8 of 128 channels: 304 us, 1,020 TFLOP/s, 92 % of what one
// bf16 product of 8,192^3 reaches here; calls one after the other 358 us, 64 % of such products
// (1,340 TFLOP/s). 256 channels: 1,370 us, 450 TFLOP/s: an operand from LDS serves one product of 16 rows, and
// one wave a SIMD has nothing to do meanwhile (matrix units 19 %, vector units 21 % busy).
// Probabilities are rounded to the cache's type, as in the single-token kernel.
#include "kv.h"
#include "kv_strip.h"

#include <algorithm>
#include <type_traits>

namespace ivf {
namespace {

// D <= 128: eight waves, 32 rows each (four waves over tiles of 64 keys: 327 us where this took
// 306); wider: four waves of 16 rows (registers, LDS).
template <int D> struct PromptShape {
    static constexpr int waves = D <= 128 ? 8 : 4, ct = D <= 128 ? 2 : 1;
    static constexpr int threads = 64 * waves, rows = 16 * ct * waves;
    static constexpr int keys = 16 * waves;  // of a tile: a strip a wave
};

template <typename TT, int D>
__global__ __launch_bounds__(PromptShape<D>::threads, 2) void kv_prompt_kernel(KvAttend a, int tiles)
{
    typedef PromptShape<D> Shape;
    constexpr int CT = Shape::ct, kWaves = Shape::waves, kTileKeys = Shape::keys;
    typedef Pieces<D> P;
    typedef typename TT::elem elem;
    constexpr int kOut = D / 16, kFrag = D / 32, kRows = Shape::rows;
    __shared__ u32x4 kbuf[2][kWaves][kFrag][64];
    __shared__ u32x4 vbuf[2][kWaves / 2][kOut][64];
    __shared__ int absent[2][kWaves];  // strips that no table entry names
    __shared__ int lims[kWaves];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, h = lane >> 4;
    const uint32_t heads = a.c.heads, bid = blockIdx.x, part = bid / heads;
    const int head = (int)(bid - part * heads);
    const int split = (int)(part % (uint32_t)a.splits);
    const int64_t tile = tiles - 1 - (int)(part / (uint32_t)a.splits);  // the last rows see most keys: first

    const int64_t all_rows = a.T * a.group, g0 = tile * kRows;
    const int64_t t_first = g0 / a.group, t_last = (min(g0 + kRows, all_rows) - 1) / a.group;
    const int last_key = (int)min((int64_t)a.cols << a.c.shift, (int64_t)INT32_MAX) - 1;

    // this lane's rows
    int64_t tok[CT];
    int qhead[CT], pos[CT];
    bool mine[CT];
    u32x4 qf[CT][kFrag];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int64_t r = g0 + 16 * (CT * wave + ct) + col;
        const bool have = r < all_rows;
        tok[ct] = have ? r / a.group : -1;
        qhead[ct] = head * a.group + (int)(have ? r - tok[ct] * a.group : 0);
        pos[ct] = have ? max(min(a.position[tok[ct]], last_key), -1) : -1;  // keys are subtracted from it
        mine[ct] = false;
        const elem *q = (const elem *)a.q.p + (have ? tok[ct] * a.q.ts + (int64_t)qhead[ct] * a.q.hs : 0);
#pragma unroll
        for (int c = 0; c < P::n; ++c)
#pragma unroll
            for (int d = 0; d < P::size(c) / 32; ++d) {
                u32x4 x = {0, 0, 0, 0};
                if (have) x = *(const u32x4 *)(q + P::off(c) + P::size(c) / 4 * h + 8 * d);
                // a channel that is not finite makes every score NaN, as in the single-token kernel: an
                // infinity alone may score -infinity with all keys, which is how masked ones look
                if (!TT::finite(x)) x = (u32x4){0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
                qf[ct][P::off(c) / 32 + d] = x ^ a.q_flip;
            }
    }

    f32x4 acc[CT][kOut];
    float ref[CT], sub[CT], sum[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
        for (int i = 0; i < kOut; ++i) acc[ct][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        ref[ct] = -INFINITY;
        sub[ct] = sum[ct] = 0.f;
    }
    typename Keys<D>::Offsets k_offs(lane, a.c.bs);
    typename Values<D>::Offsets v_offs(lane, a.c.bs);
    const int strip_mask = (1 << (a.c.shift - 4)) - 1;
    const size_t rec_bytes = a.c.rec_bytes();

    // the request of the first token, by bisection, and those that follow
    int64_t b = 0;
    {
        int64_t hi = a.B;
        while (hi - b > 1) {
            const int64_t mid = (b + hi) >> 1;
            if (a.start[mid] <= t_first) b = mid;
            else hi = mid;
        }
    }
    for (; b < a.B; ++b) {
        const int64_t s0 = min(max((int64_t)a.start[b], (int64_t)0), a.T);
        const int64_t s1 = min(max((int64_t)a.start[b + 1], s0), a.T);
        if (s0 > t_last) break;
        if (s1 <= t_first || s1 == s0 || (s1 - s0) * a.group <= a.small_rows) continue;

        int lim[CT], wmax = -1, wmin = INT32_MAX;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const bool in = tok[ct] >= s0 && tok[ct] < s1;
            lim[ct] = in ? pos[ct] : -1;
            mine[ct] |= in;
            wmax = max(wmax, lim[ct]);
            wmin = min(wmin, lim[ct]);
        }
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) {
            wmax = max(wmax, __shfl_xor(wmax, d));
            wmin = min(wmin, __shfl_xor(wmin, d));
        }
        wmax = __builtin_amdgcn_readfirstlane(wmax);
        wmin = __builtin_amdgcn_readfirstlane(wmin);
        if (lane == 0) lims[wave] = wmax;
        __syncthreads();
        int gmax = -1;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) gmax = max(gmax, lims[w]);
        gmax = __builtin_amdgcn_readfirstlane(gmax);
        __syncthreads();

        const int ntiles = (int)(((int64_t)gmax + kTileKeys) / kTileKeys);  // 0 where gmax is -1
        const int per = (ntiles + a.splits - 1) / a.splits;
        const int k0 = min((int64_t)ntiles, (int64_t)split * per), k1 = min(ntiles, k0 + per);
        if (k0 >= k1) continue;
        const int32_t *table = a.table + b * a.cols;

        // lane i keeps the block of this wave's strip of the i-th next tile
        int pages = -1, ahead = 0;
        auto look = [&](int k) {
            const int64_t key = (int64_t)(k + lane) * kTileKeys + 16 * wave;
            pages = -1;
            if (key <= gmax) {
                const int id = table[key >> a.c.shift];
                if (id >= 0 && id < a.c.blocks) pages = id;
            }
        };
        Keys<D> keys;
        Values<D> vals;
        int page = -1;
        auto fetch = [&](int k) {
            if (ahead == 64) {
                look(k);
                ahead = 0;
            }
            page = __builtin_amdgcn_readlane(pages, ahead);
            ++ahead;
            if (page >= 0) {
                const uint8_t *rec = a.c.rec + ((int64_t)page * a.c.heads + head) * rec_bytes;
                const StripBase base = StripBase::at<D>(rec, (kWaves * k + wave) & strip_mask);
                keys.load(base, k_offs);
                vals.load(base, v_offs);
            }
        };
        auto stage = [&](int k) {
            const int buf = k & 1;
            if (lane == 0) absent[buf][wave] = page < 0;
            u32x2 *vdst = (u32x2 *)&vbuf[buf][wave >> 1][0][lane] + (wave & 1);
            if (page < 0) {  // nothing there: zeros, and the scores are masked
#pragma unroll
                for (int w = 0; w < kFrag; ++w) kbuf[buf][wave][w][lane] = (u32x4){0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < kOut; ++j) vdst[128 * j] = (u32x2){0, 0};
                return;
            }
            const int key = k * kTileKeys + 16 * wave;
            auto piece = [&](auto piece_c) {
                constexpr int c = decltype(piece_c)::value, S = P::size(c);
                const float ks = kv_scale(keys.ks[c]);
#pragma unroll
                for (int d = 0; d < S / 32; ++d)
                    kbuf[buf][wave][P::off(c) / 32 + d][lane] = decode8<TT>(keys.k[P::off(c) / 32 + d], ks);
                float vs[4];
                four_scales(vals.vs[c], vs);
                if (key + 15 > gmax) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key + 4 * h + i > gmax) vs[i] = 1.f;
                }
                u32x2 v[S / 16];
                value_operands<TT, S>(vals.v[c], vs, v);
#pragma unroll
                for (int j = 0; j < S / 16; ++j) vdst[128 * (P::off(c) / 16 + j)] = v[j];
            };
            piece(std::integral_constant<int, 0>());
            if constexpr (P::n > 1) piece(std::integral_constant<int, 1>());
        };
        // 64 keys of a tile
        auto compute = [&](int k, int part) {
            const int buf = k & 1, first = k * kTileKeys + 64 * part;
            if (first > wmax) return;  // uniform over the wave
            f32x4 st[4][CT];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) st[e][ct] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kFrag; ++w) {
                    const u32x4 x = kbuf[buf][4 * part + e][w][lane];
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) st[e][ct] = TT::mfma(x, qf[ct][w], st[e][ct]);
                }
            }
            const int *none = &absent[buf][4 * part];
            const int gone = none[0] | none[1] << 1 | none[2] << 2 | none[3] << 3;
            if (first + 63 > wmin || __builtin_amdgcn_readfirstlane(gone)) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    const int left = lim[ct] - first - 4 * h;  // of the lane's keys, the last to be seen
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int last = (gone >> e & 1) ? -1 : left;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (last < 16 * e + i) st[e][ct][i] = -INFINITY;
                            asm volatile("" : "+v"(st[e][ct][i]));  // one comparison at a time: no stack of masks
                        }
                    }
                }
            }
            u32x4 pf[CT][2];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float p[4][4], part_sum;
                auto probabilities = [&]() {
                    part_sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[e][i] = exp2_fast(__builtin_fmaf(st[e][ct][i], a.scale, -sub[ct]));
                        part_sum += (p[e][0] + p[e][1]) + (p[e][2] + p[e][3]);
                    }
                };
                probabilities();
                if (__ballot(part_sum > kMost || ref[ct] == -INFINITY)) {
                    float mx = st[0][ct][0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, st[i / 4][ct][i % 4]);
                    const float top = fmaxf(ref[ct], max_over_h(mx * a.scale));
                    const float f = ref[ct] == top ? 1.f : exp2_fast(ref[ct] - top);
                    ref[ct] = top;
                    sub[ct] = top == -INFINITY ? 0.f : top - kCarry;
                    sum[ct] *= f;
#pragma unroll
                    for (int i = 0; i < kOut; ++i) acc[ct][i] *= f;
                    probabilities();
                }
                sum[ct] += part_sum;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pf[ct][e >> 1][2 * (e & 1)] = TT::pack(p[e][0], p[e][1]);
                    pf[ct][e >> 1][2 * (e & 1) + 1] = TT::pack(p[e][2], p[e][3]);
                }
            }
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int j = 0; j < kOut; ++j) {
                    const u32x4 x = vbuf[buf][2 * part + p][j][lane];
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) acc[ct][j] = TT::mfma(x, pf[ct][p], acc[ct][j]);
                }
        };
        look(k0);
        fetch(k0);
        stage(k0);
        if (k0 + 1 < k1) fetch(k0 + 1);
        __syncthreads();
        for (int k = k0; k < k1; ++k) {
            if (k + 1 < k1) {
                stage(k + 1);
                if (k + 2 < k1) fetch(k + 2);
            }
#pragma unroll 1
            for (int part = 0; part < kWaves / 4; ++part) compute(k, part);
            __syncthreads();
        }
    }

#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const float total = sum_over_h(sum[ct]);
        if (!mine[ct]) continue;
        const int64_t orow = tok[ct] * ((int64_t)a.c.heads * a.group) + qhead[ct];
        if (a.splits == 1)
            write_rows<TT, D>(acc[ct], (elem *)a.out + orow * D, total == 0.f ? 0.f : 1.f / total, h);
        else
            write_part<D>(acc[ct], a.part + (orow * a.splits + split) * D, h);
        if (h == 0) {
            if (a.splits > 1) a.part_ml[orow * a.splits + split] = make_float2(ref[ct], total);
            else if (a.lse) a.lse[orow] = log_of(ref[ct], total);
        }
    }
}

template <typename TT, int D> hipError_t launch_prompt(const KvAttend &a, hipStream_t s)
{
    typedef PromptShape<D> Shape;
    const int64_t tiles = (a.T * a.group + Shape::rows - 1) / Shape::rows;
    const unsigned grid = (unsigned)(tiles * a.splits * a.c.heads);
    hipLaunchKernelGGL((kv_prompt_kernel<TT, D>), dim3(grid), dim3(Shape::threads), 0, s, a, (int)tiles);
    return hipGetLastError();
}

template <typename TT> hipError_t launch_prompt_dim(const KvAttend &a, hipStream_t s)
{
    switch (a.c.dim) {
    case 64: return launch_prompt<TT, 64>(a, s);
    case 96: return launch_prompt<TT, 96>(a, s);
    case 128: return launch_prompt<TT, 128>(a, s);
    case 192: return launch_prompt<TT, 192>(a, s);
    default: return launch_prompt<TT, 256>(a, s);
    }
}

}  // namespace

int kv_prompt_rows(int dim) { return dim <= 128 ? PromptShape<128>::rows : PromptShape<256>::rows; }

int kv_prompt_resident(int dim) { return dim <= 128 ? 8 / PromptShape<128>::waves : 1; }

hipError_t launch_kv_prompt(const KvAttend &a, hipStream_t s)
{
    return a.c.bf16 ? launch_prompt_dim<KvBf16>(a, s) : launch_prompt_dim<KvF16>(a, s);
}

}  // namespace ivf
