// A strip of 16 keys and values of the 4-bit cache in a wave's registers, as the
// attention kernels hold it, and its operands for v_mfma_f32_16x16x32.
//
// Lane (r = lane % 16, h = lane / 16). Keys: the lane holds key 4 (r % 4) + r / 4, so
// that row 4 h + i of a product with the keys as A is key 4 i + h; the channels of a
// key are taken as its row of codes lies in memory (any order serves, the query's
// fragments use the same), 16 bytes a lane at 128 channels. Values: lane (r, h)
// holds, of keys 4 i + h, the codes of neighbouring channels (dim / 16 of them).
#pragma once

#include "kv_types.h"

namespace ivf {

constexpr float kRaise = 6.f;  // a score may pass its row's reference by this much
constexpr float kCarry = 8.f;  // probabilities are times 2^kCarry

// A row of channels is taken as one or two pieces of 128, 64 or 32.
template <int D> struct Pieces {
    static constexpr int first = D >= 128 ? 128 : 64, second = D - first;
    static constexpr int n = second ? 2 : 1;
    static constexpr int size(int c) { return c == 0 ? first : second; }
    static constexpr int off(int c) { return c == 0 ? 0 : first; }
};

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

// The largest of three; a NaN among them makes the result any of the three (a
// row that holds one is NaN whatever its reference).
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The values' operand of one piece of S channels: out[j] holds channel S / 16 r + j of
// keys 4 i + h, i = 0 ... 3 (w: their codes, vs: their scales).
template <typename TT, int S>
__device__ __forceinline__ void value_operands(const uint32_t (&w)[4], const float (&vs)[4], u32x2 (&out)[S / 16])
{
#pragma unroll
    for (int p = 0; p < S / 32; ++p) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = p == 0   ? TT::template decode<0>(w[i], vs[i])
                   : p == 1 ? TT::template decode<1>(w[i], vs[i])
                   : p == 2 ? TT::template decode<2>(w[i], vs[i])
                            : TT::template decode<3>(w[i], vs[i]);
        out[2 * p] = (u32x2){low_halves(x[0], x[1]), low_halves(x[2], x[3])};
        out[2 * p + 1] = (u32x2){high_halves(x[0], x[1]), high_halves(x[2], x[3])};
    }
}


// Natural logarithm of a row's sum of exponentials.
__device__ __forceinline__ float log_of(float ref, float sum)
{
    return sum == 0.f ? -INFINITY : (ref - kCarry + __builtin_amdgcn_logf(sum)) * 0.69314718056f;
}

// A lane's share of its row: tile j, register r of a piece of S channels is channel
// S / 4 h + S / 16 r + j.
template <typename TT, int D>
__device__ __forceinline__ void write_rows(const f32x4 (&acc)[D / 16], typename TT::elem *o, float factor, int h)
{
    typedef Pieces<D> P;
#pragma unroll
    for (int c = 0; c < P::n; ++c) {
        const int S = P::size(c), tile = P::off(c) / 16;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < S / 16; j += 2)
                *(uint32_t *)(o + P::off(c) + S / 4 * h + S / 16 * r + j) =
                    TT::pack(acc[tile + j][r] * factor, acc[tile + j + 1][r] * factor);
    }
}

template <int D> __device__ __forceinline__ void write_part(const f32x4 (&acc)[D / 16], float *o, int h)
{
    typedef Pieces<D> P;
#pragma unroll
    for (int c = 0; c < P::n; ++c) {
        const int S = P::size(c), tile = P::off(c) / 16;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < S / 16; j += 2)
                *(float2 *)(o + P::off(c) + S / 4 * h + S / 16 * r + j) =
                    make_float2(acc[tile + j][r], acc[tile + j + 1][r]);
    }
}

}  // namespace ivf
