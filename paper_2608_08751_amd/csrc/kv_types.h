// The cache's 16-bit types: conversions of 4-bit codes and matrix products.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ivf {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Whether none of 8 numbers is an infinity or NaN; exponent: the bits of both halves' exponents.
__device__ __forceinline__ bool all_finite(u32x4 w, uint32_t exponent)
{
    const uint32_t lo = exponent & 0xffffu, hi = exponent & 0xffff0000u;
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) ok &= (w[i] & lo) != lo && (w[i] & hi) != hi;
    return ok;
}

struct KvF16 {
    typedef _Float16 elem;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    // two codes (byte SEL of w, the low half first) times the power of two `scale`
    template <int SEL> static __device__ __forceinline__ uint32_t decode(uint32_t w, float scale)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)  // to nearest
    {
        const f16x2 r = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, r);
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[0]; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[1]; }
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ bool finite(u32x4 w) { return all_finite(w, 0x7c007c00u); }
    static constexpr int kMinExp = -13, kMaxExp = 13;
};

struct KvBf16 {
    typedef __bf16 elem;
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    template <int SEL> static __device__ __forceinline__ uint32_t decode(uint32_t w, float scale)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const bf16x2 r = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, r);
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ bool finite(u32x4 w) { return all_finite(w, 0x7f807f80u); }
    static constexpr int kMinExp = -125, kMaxExp = 125;
};

// 2^(e - 127) of a scale byte (255 gives an infinity, which decodes to NaN)
__device__ __forceinline__ float kv_scale(uint32_t e) { return __uint_as_float(e << 23); }

}  // namespace ivf
