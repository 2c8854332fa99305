// The form in 8 bits on the device: a block of 32 values, a scale 2^k kept as the byte k + 127, codes = values / 2^k (internal device code).
#pragma once
#include "act8.h"
#include "norm_device.h"

namespace sk {

// What settles a block's scale is its largest magnitude as bits of fp32: their order is that of the magnitudes, NaN above infinity above all others.
template <int CODE> struct Code8 {
    static constexpr uint32_t top = CODE == E4M3 ? 0x600000 : 0x7e0000;     // mantissa of Q: 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
    static constexpr int down = CODE == E4M3 ? 8 : 6;                       // exponent of Q
    static constexpr uint32_t nan = CODE == E4M3 ? 0x7f : 0x80;
    // the largest magnitude that a code can stand for in a type: 61440, 65024; 1.875 * 2^127, 127 * 2^120
    __host__ __device__ static constexpr uint32_t limit(int dt)
    {
        return dt == 2 ? (CODE == E4M3 ? 0x47700000u : 0x477e0000u) : (CODE == E4M3 ? 0x7f700000u : 0x7efe0000u);
    }
    // k + 127 for a block whose largest magnitude has these bits: one more than its exponent if its mantissa is over Q's
    __device__ static __forceinline__ uint32_t scale_byte(uint32_t largest)
    {
        const int e = (int)((largest + (0x7fffffu - top)) >> 23) - down;
        return e > 10 ? e : 10;
    }
    __device__ static __forceinline__ float inverse(uint32_t byte) { return __uint_as_float((254 - byte) << 23); }
    __device__ static __forceinline__ float scale(uint32_t byte) { return __uint_as_float(byte << 23); }
    // four codes of finite values within the limit; the products with a power of two are exact
    __device__ static __forceinline__ uint32_t four(float a, float b, float c, float d, float inverse)
    {
        if constexpr (CODE == E4M3) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
            return __builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, w, true);
        } else {
            // 1.5 * 2^23 leaves no room for a fraction: the sum's low byte is the rounded value's two's complement
            const uint32_t p = __float_as_uint(fmaf(a, inverse, 12582912.f)), q = __float_as_uint(fmaf(b, inverse, 12582912.f));
            const uint32_t r = __float_as_uint(fmaf(c, inverse, 12582912.f)), s = __float_as_uint(fmaf(d, inverse, 12582912.f));
            return __builtin_amdgcn_perm(__builtin_amdgcn_perm(s, r, 0x0c0c0400), __builtin_amdgcn_perm(q, p, 0x0c0c0400), 0x05040100);
        }
    }
    __device__ static __forceinline__ uint32_t one(float v, float inverse) { return four(v, 0.f, 0.f, 0.f, inverse) & 0xff; }
    // four values, NaN left out of account
    __device__ static __forceinline__ void numbers(uint32_t w, float scale, float (&f)[4])
    {
        if constexpr (CODE == E4M3) {
            typedef float floatx2 __attribute__((ext_vector_type(2)));
            const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            f[0] = lo[0] * scale; f[1] = lo[1] * scale; f[2] = hi[0] * scale; f[3] = hi[1] * scale;
        } else {                 // unsigned bytes widen in one operation, whichever of the word's it is; 128 too much, which the sum takes off again, exactly
            const uint32_t u = w ^ 0x80808080u;
            const float below = -128.f * scale;
            f[0] = fmaf((float)(u & 0xff), scale, below);
            f[1] = fmaf((float)(u >> 8 & 0xff), scale, below);
            f[2] = fmaf((float)(u >> 16 & 0xff), scale, below);
            f[3] = fmaf((float)(u >> 24), scale, below);
        }
    }
    // is one of the four NaN, and `numbers` wrong about it?  (a byte of zero, of -128 + 128)
    __device__ static __forceinline__ uint32_t unlike(uint32_t w)
    {
        const uint32_t u = w ^ 0x80808080u;
        return CODE == E4M3 ? 0 : (u - 0x01010101u) & ~u & 0x80808080u;
    }
    __device__ static __forceinline__ void mark(uint32_t w, float (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (w >> 8 * i & 0xff) == nan ? __builtin_nanf("") : f[i];
    }
    // four values
    __device__ static __forceinline__ void values(uint32_t w, float scale, float (&f)[4])
    {
        numbers(w, scale, f);
        if (unlike(w)) mark(w, f);
    }
    __device__ static __forceinline__ float value(uint32_t byte, float scale)
    {
        float f[4];
        values(byte, scale, f);
        return f[0];
    }
};

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// what a block's scale goes by, and what is coded, of a value that may be anything: 0 for NaN and infinities, else within the limit
__device__ __forceinline__ uint32_t counted(float v, uint32_t limit)
{
    const uint32_t m = magnitude(v);
    return m >= 0x7f800000u ? 0 : m < limit ? m : limit;
}
template <int CODE> __device__ __forceinline__ uint32_t any_code(float v, float inverse, uint32_t limit)
{
    if (magnitude(v) >= 0x7f800000u) return Code8<CODE>::nan;
    const float m = __uint_as_float(counted(v, limit));
    return Code8<CODE>::one(v < 0.f ? -m : m, inverse);
}

__host__ __device__ inline long blocks_of(long length) { return (length + 31) / 32; }

template <class F> void pick_code(int code, F f)
{
    if (code == E4M3) f(std::integral_constant<int, E4M3>{});
    else f(std::integral_constant<int, I8>{});
}

}  // namespace sk
