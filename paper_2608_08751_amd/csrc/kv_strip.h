// A strip of 16 keys and values of the 4-bit cache in a wave's registers, as the
// attention kernels hold it, and its operands for v_mfma_f32_16x16x32.
//
// Lane (r = lane % 16, h = lane / 16). Keys: the lane holds key r, so that its four
// results of a product with the keys as A are keys 4 h ... 4 h + 3; the channels of a
// key are taken as its row of codes lies in memory (any order serves, the query's
// fragments use the same), 16 bytes a lane at 128 channels. Values: lane (r, h)
// holds, of keys 4 h ... 4 h + 3, the codes of neighbouring channels (dim / 16 of them) and
// their four scales in one word.
#pragma once

#include "kv_types.h"

namespace ivf {

constexpr float kCarry = 8.f;      // probabilities are times 2^kCarry
constexpr float kMost = 0x1p14f;   // what a lane's probabilities of a step may sum to (f16 holds 2^16)

// A row of channels is taken as one or two pieces of 128, 64 or 32.
template <int D> struct Pieces {
    static constexpr int first = D >= 128 ? 128 : 64, second = D - first;
    static constexpr int n = second ? 2 : 1;
    static constexpr int size(int c) { return c == 0 ? first : second; }
    static constexpr int off(int c) { return c == 0 ? 0 : first; }
};

// Where a strip's four parts begin: the rows of codes (keys; the values' are
// bs D / 2 further on, which their lane offsets hold), the keys' scales and the
// values', each from the record's start. Uniform over the wave: kept in scalar registers, so that a
// load takes scalar base, 32-bit lane offset and constant.
typedef const __attribute__((address_space(1))) uint8_t *GlobalBytes;
template <typename T> __device__ __forceinline__ T load_global(GlobalBytes p)
{
    return *(const __attribute__((address_space(1))) T *)p;
}
// A lane offset as the load takes it: extended to 64 bits where it is used (taken out of the
// loop the sum would be a 64-bit vector addition a load). No instruction.
__device__ __forceinline__ uint32_t here(uint32_t &offset)
{
    asm volatile("" : "+v"(offset));
    return offset;
}
struct StripBase {
    GlobalBytes rows, k_scales, v_scales;
    template <int D> static __device__ __forceinline__ StripBase at(const uint8_t *rec, int strip)
    {
        const GlobalBytes r = (GlobalBytes)rec;
        StripBase b = {r + strip * (8 * D), r + strip * (D / 2), r + strip * 16};
        asm("" : "+s"(b.rows), "+s"(b.k_scales), "+s"(b.v_scales));  // no instruction: keeps the sums apart
        return b;
    }
};

// The values of a strip, and a lane's offsets into them.
template <int D> struct Values {
    typedef Pieces<D> P;
    uint32_t v[P::n][4];
    uint32_t vs[P::n];
    struct Offsets {
        uint32_t v[P::n], vs[P::n];
        __device__ __forceinline__ Offsets(int lane, int bs)
        {
            const int m = lane & 15, h = lane >> 4;
#pragma unroll
            for (int c = 0; c < P::n; ++c) {
                const int S = P::size(c), off = P::off(c), g = off / 32;
                v[c] = (bs + 4 * h) * (D / 2) + off / 2 + m * S / 32;
                vs[c] = bs * (D + D / 32) + (g + (S == 128 ? m >> 2 : S == 64 ? m >> 3 : 0)) * bs + 4 * h;
            }
        }
    };
    __device__ __forceinline__ void load(const StripBase &b, Offsets &o)
    {
#pragma unroll
        for (int c = 0; c < P::n; ++c) {
            const int S = P::size(c);
            vs[c] = load_global<uint32_t>(b.v_scales + here(o.vs[c]));
            const GlobalBytes row = b.rows + here(o.v[c]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const GlobalBytes p = row + i * (D / 2);
                v[c][i] = S == 128 ? load_global<uint32_t>(p) : S == 64 ? load_global<uint16_t>(p) : load_global<uint8_t>(p);
            }
        }
    }
};

// The keys of a strip as 16-bit operands are made of them: S / 32 dwords of a piece.
template <int D> struct Keys {
    typedef Pieces<D> P;
    uint32_t k[D / 32];
    uint32_t ks[P::n];
    struct Offsets {
        uint32_t k[P::n], ks[P::n];
        __device__ __forceinline__ Offsets(int lane, int bs)
        {
            const int key = lane & 15, h = lane >> 4;
#pragma unroll
            for (int c = 0; c < P::n; ++c) {
                const int S = P::size(c), off = P::off(c), g = off / 32;
                k[c] = key * (D / 2) + off / 2 + S / 8 * h;
                ks[c] = bs * D + key * (D / 32) + g + (S == 128 ? h : S == 64 ? h >> 1 : 0);
            }
        }
    };
    __device__ __forceinline__ void load(const StripBase &b, Offsets &o)
    {
#pragma unroll
        for (int c = 0; c < P::n; ++c) {
            const int S = P::size(c), g = P::off(c) / 32;
            ks[c] = load_global<uint8_t>(b.k_scales + here(o.ks[c]));
            if (S == 128) {
                const u32x4 x = load_global<u32x4>(b.rows + here(o.k[c]));
#pragma unroll
                for (int i = 0; i < 4; ++i) k[g + i] = x[i];
            } else if (S == 64) {
                const u32x2 x = load_global<u32x2>(b.rows + here(o.k[c]));
                k[g] = x[0];
                k[g + 1] = x[1];
            } else {
                k[g] = load_global<uint32_t>(b.rows + here(o.k[c]));
            }
        }
    }
};

// The keys of a strip as 4-bit operands: parts of 128 channels, a lane holds the 32
// channels of group h and their scale (a group beyond the last: the last
// once more, against zeros of the query).
template <int D> struct CodedKeys {
    static constexpr int kParts = (D + 127) / 128;
    u32x4 k[kParts];
    uint32_t ks[kParts];
    struct Offsets {
        uint32_t k[kParts], ks[kParts];
        __device__ __forceinline__ Offsets(int lane, int bs)
        {
            const int key = lane & 15, h = lane >> 4;
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                const int g = min(4 * p + h, D / 32 - 1);
                k[p] = key * (D / 2) + 16 * g;
                ks[p] = bs * D + key * (D / 32) + g;
            }
        }
    };
    __device__ __forceinline__ void load(const StripBase &b, Offsets &o)
    {
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            k[p] = load_global<u32x4>(b.rows + here(o.k[p]));
            ks[p] = load_global<uint8_t>(b.k_scales + here(o.ks[p]));
        }
    }
};

// Query rows as sums of 6-bit numbers (e2m3): a channel is a fixed-point number, the
// largest of its 32 in [8, 16), of four digits to the base 32 from -16 to 16: term t is digit t,
// beside a power of two for each 32 channels (byte t of a scale word: that of term t).
// The matrix instruction drops bits of a product that lie more than about 14 below the
// largest one it adds up: whole numbers times 4-bit codes have none there, the terms of a
// floating-point split (fp8) do (scores off by up to 2^-16 of sum |q k|, now 2^-22).
template <typename TT, int D> struct CodedQuery {
    static constexpr int kTerms = 4, kParts = CodedKeys<D>::kParts;
    static constexpr int kGroups = D / 32, kGroupBytes = 24, kRowBytes = kGroups * kGroupBytes;
    typedef int i32x6 __attribute__((ext_vector_type(6)));
    i32x6 q[kParts][kTerms];
    uint32_t scale[kParts];

    static constexpr int bytes(int rows) { return rows * (kTerms * kRowBytes + 4 * kGroups); }
    // THREADS threads stage rows r < n by row(r) (their channels; zeros up to ROWS) in
    // lds: [term][row][kRowBytes] and then the scale words [row][kGroups]. First the loads,
    // then, after what the caller has put between, the rounding.
    template <int THREADS, int ROWS> struct Stage {
        static constexpr int kLanes = D / 4, kAtOnce = THREADS / kLanes;  // a thread: 4 channels
        static constexpr int kTurns = (ROWS + kAtOnce - 1) / kAtOnce;
        u32x2 w[kTurns];
        template <typename Row> __device__ __forceinline__ void load(int tid, int n, Row row)
        {
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                const int r = tid / kLanes + i * kAtOnce;
                w[i] = (u32x2){0, 0};
                if (r < n && tid < kAtOnce * kLanes) w[i] = *(const u32x2 *)(row(r) + 4 * (tid % kLanes));
            }
        }
        __device__ __forceinline__ void store(int tid, int n, uint8_t *lds, uint32_t flip) const
        {
            const int c = tid % kLanes, at = c % 4;  // four threads: the 12 bytes of 16 channels
            uint32_t *scales = (uint32_t *)(lds + ROWS * kTerms * kRowBytes);
#pragma unroll
            for (int j = 0; j < kTurns; ++j) {
                const int r = tid / kLanes + j * kAtOnce;
                const bool mine = r < ROWS && tid < kAtOnce * kLanes;
                uint8_t *put = lds + r * kRowBytes + 12 * (c / 4) + 4 * at;
                if (j * kAtOnce >= n) {  // no rows in this turn: zeros
#pragma unroll
                    for (int t = 0; t < kTerms; ++t)
                        if (mine && at < 3) *(uint32_t *)(put + t * ROWS * kRowBytes) = 0;
                    if (mine && c % 8 == 0) scales[r * kGroups + c / 8] = 0x7f7f7f7fu;
                    continue;
                }
                const u32x2 y = w[j] ^ flip;
                float x[4] = {TT::lo(y[0]), TT::hi(y[0]), TT::lo(y[1]), TT::hi(y[1])};
                uint32_t top = 0;  // bits of the largest magnitude; of infinities and NaN: larger still
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(fabsf(x[i])));
#pragma unroll
                for (int d = 1; d < 8; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
                const int e = max((int)(top >> 23), 15);  // 255 makes the group's products NaN
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = e == 255 ? 0.f : __builtin_amdgcn_ldexpf(x[i], 130 - e);  // below 16
#pragma unroll
                for (int t = 0; t < kTerms; ++t) {
                    uint32_t four = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float whole = rintf(x[i]);  // 0 ... 16 are the 6-bit numbers 0 ... 2 in eighths
                        four |= ((uint32_t)fabsf(whole) | (__float_as_uint(x[i]) >> 31) << 5) << 6 * i;
                        x[i] = (x[i] - whole) * 32.f;
                    }
                    const uint32_t next = (uint32_t)__shfl_down((int)four, 1);
                    if (mine && at < 3)
                        *(uint32_t *)(put + t * ROWS * kRowBytes) = four >> 8 * at | next << (24 - 8 * at);
                }
                if (mine && c % 8 == 0)
                    scales[r * kGroups + c / 8] =
                        (uint32_t)e | (uint32_t)(e - 5) << 8 | (uint32_t)(e - 10) << 16 | (uint32_t)(e - 15) << 24;
            }
        }
    };
    // The operands of row r for lane (its column, h): group 4 p + h of a part.
    __device__ __forceinline__ void load(const uint8_t *lds, int rows, int r, int h)
    {
        const uint32_t *scales = (const uint32_t *)(lds + rows * kTerms * kRowBytes);
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const int g = 4 * p + h;
#pragma unroll
            for (int t = 0; t < kTerms; ++t) {
                const u32x2 *from = (const u32x2 *)(lds + (t * rows + r) * kRowBytes + kGroupBytes * g);
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    u32x2 x = {0, 0};
                    if (g < kGroups) x = from[i];
                    q[p][t][2 * i] = (int)x[0];
                    q[p][t][2 * i + 1] = (int)x[1];
                }
            }
            scale[p] = g < kGroups ? scales[r * kGroups + g] : 0x7f7f7f7fu;
        }
    }
    template <int T> __device__ __forceinline__ f32x4 term(const CodedKeys<D> &k, int p, f32x4 acc) const
    {
        const i32x8 a = {(int)k.k[p][0], (int)k.k[p][1], (int)k.k[p][2], (int)k.k[p][3], 0, 0, 0, 0};
        const i32x6 y = q[p][T];
        const i32x8 b = {y[0], y[1], y[2], y[3], y[4], y[5], 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 2, 0, (int)k.ks[p], T, (int)scale[p]);
    }
    // q.k of 16 keys (rows) and the columns' query rows, the smallest terms first
    __device__ __forceinline__ f32x4 scores(const CodedKeys<D> &k) const
    {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        acc = add<3>(k, acc);
        acc = add<2>(k, acc);
        acc = add<1>(k, acc);
        return add<0>(k, acc);
    }
    template <int T> __device__ __forceinline__ f32x4 add(const CodedKeys<D> &k, f32x4 acc) const
    {
#pragma unroll
        for (int p = 0; p < kParts; ++p) acc = term<T>(k, p, acc);
        return acc;
    }
};

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

// 2^(e - 127) of byte i of w, e in bits 23 ... 30.
template <int I> __device__ __forceinline__ float scale_byte_of(uint32_t w)
{
    return __uint_as_float(__builtin_amdgcn_perm(0u, w, (uint32_t)I << 24 | 0x0c0c0cu) >> 1);
}
__device__ __forceinline__ void four_scales(uint32_t w, float (&s)[4])
{
    s[0] = scale_byte_of<0>(w);
    s[1] = scale_byte_of<1>(w);
    s[2] = scale_byte_of<2>(w);
    s[3] = scale_byte_of<3>(w);
}

// x of the lane 8 columns further on, of 16.
__device__ __forceinline__ float other_half(float x)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x128, 0xf, 0xf, true));
}

// The values' operand of one piece of S channels: out[j] holds channel S / 16 r + j of
// keys 4 h + i, i = 0 ... 3 (w: their codes, vs: their scales).
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
