// What the kernels of the operators on device tensors share: element types, codes of 8 bits, a softmax's weights.
#ifndef SS_OPERATOR_DEVICE_H
#define SS_OPERATOR_DEVICE_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "ss_device.h"

namespace ss {

// ------------------------------------------------------------------------------------------ element types
// T: _Float16 or __bf16.  Operands of the matrix instructions are 8 of them per lane.
template <typename T>
struct Half;
template <>
struct Half<_Float16> {
    typedef f16x8 x8;
    static __device__ __forceinline__ f32x4 mma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
template <>
struct Half<__bf16> {
    typedef bf16x8 x8;
    static __device__ __forceinline__ f32x4 mma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

constexpr float kLowest = -3.0e38f;   // running maximum of no score: finite, so that exp2(-inf - kLowest) is 0

// Eight values of 16 bits as floats, and back (half saturates at its largest finite value, NaN stays NaN).
template <typename T>
__device__ __forceinline__ void to_floats(const u32x4& r, float (&f)[8])
{
    const typename Half<T>::x8 h = __builtin_bit_cast(typename Half<T>::x8, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
}
template <typename T>
__device__ __forceinline__ u32x4 from_floats(const float (&f)[8])
{
    typename Half<T>::x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (std::is_same<T, _Float16>::value) h[i] = __builtin_bit_cast(_Float16, f2h(f[i]));
        else h[i] = (__bf16)f[i];
    }
    return __builtin_bit_cast(u32x4, h);
}

// What a weight's exponent s * sc takes off, of the maximum m that the weights are relative to.  Its rounding, up to 2^-24 of it, is a
// factor common to all of a row's slots, but where it is large no factor that a weight can hold (from 2^28 on half's range is left, from 2^31
// on the exponential's): there the differences are formed first.  A branch of the wave that ordinary scores never take.  EACH: by a row's own maximum,
// else for all rows of the wave if one needs it.
template <bool EACH = false, typename V, int N>
__device__ __forceinline__ float exponent_top(float m, float sc, V (&s)[N])
{
    float top = fmaxf(m * sc, kLowest);
    const bool large = fabsf(top) > 0x1p22f;
    if (__any(large)) {
        const float off = EACH && !large ? 0.f : m;
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] -= off;
        top = EACH && !large ? top : 0.f;
    }
    return top;
}

// score - top, where the score is a product.  Both are to be the rounded numbers: with the product inside the difference (one fma) its rounding,
// which is in the top, would remain of the largest score.
__device__ __forceinline__ float below_top(float score, float top)
{
#pragma clang fp contract(off)
    return score - top;
}

// The power of two that brings a row whose largest magnitude is `top` (in bf16) to 2^14 to 2^15, and its inverse.  2^-100 and less count as that.
__device__ __forceinline__ float half_power(float top, float* inverse)
{
    const int ex = max((int)(__float_as_uint(top) >> 23) - 127, -100);   // top is below 2^(ex + 1)
    *inverse = __uint_as_float((uint32_t)(127 - 14 + ex) << 23);
    return __uint_as_float((uint32_t)(127 + 14 - ex) << 23);
}

// R of a row over an 8-bit cache.  The largest product top = p * scale that the row has met is at least 2^6 R, and a product up to 2^15 R
// is held without a change of R: half's largest number is 2^16, and what rounds in its subnormals is off by at most 2^-25 R, 2^-31 of the
// largest.  Where the weights' maximum has moved (by `alpha`), R moves with it, as the products that it was made for no longer count.
struct WeightUnit {
    float R = 0.f;
    __device__ __forceinline__ float largest() const { return R * 0x1p15f; }
    __device__ __forceinline__ float inverse() const { return __uint_as_float(0x7f000000u - __float_as_uint(R)); }
    // `top`: of the products that come; returns what the sums so far, in the old unit, are to be multiplied by
    __device__ __forceinline__ float follow(float alpha, float top)
    {
        const float old = R * alpha;
        const uint32_t two = __float_as_uint(fmaxf(old * 64.f, top)) & 0x7f800000u;
        const uint32_t bits = min(max(two, 7u << 23) - (6u << 23), 0x7e800000u);   // 2^-126 to 2^126
        R = __uint_as_float(bits);
        return old * inverse();
    }
};

// A chunk's maximum as it is kept for the join: finite, so that differences are numbers.
__device__ __forceinline__ float part_top(float m) { return fminf(fmaxf(m, kLowest), -kLowest); }

// ------------------------------------------------------------------------------------------ vectors in 8 bits
// Largest magnitude in a vector as the bits of a float: those are ordered as the numbers, with infinities and NaN on top.
template <int HD>
__device__ __forceinline__ uint32_t vector_top(uint32_t m)
{
    auto top = [&](float o) { const uint32_t u = __float_as_uint(o); m = m > u ? m : u; };
    top(dpp<kDppXor1>(__uint_as_float(m)));
    top(dpp<kDppXor2>(__uint_as_float(m)));
    top(dpp<kDppHalfMirror>(__uint_as_float(m)));
    if (HD == 128) top(dpp<kDppMirror>(__uint_as_float(m)));
    return m;
}

// A vector in 8 bits: scale = max|x| / 127 and code = x / scale, both divisions and the step to a whole number rounded to
// nearest (even), as written.  x times the reciprocal is within 127 * 2^-23 < 1.6e-5 of that quotient, and the quotient's own rounding
// moves it by at most 2^-18, so only where a product is that near to the middle of two codes are quotients formed.  The whole
// number is the low byte of the product plus 3 * 2^22.  A vector with an infinity or NaN gets the scale NaN (it is read back as NaN
// throughout, by those who read it), one of zeros the scale 0.
template <int HD>
__device__ __forceinline__ float quantise(const float (&x)[8], uint2* codes)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = __float_as_uint(x[i]) & 0x7fffffffu;
        m = m > u ? m : u;
    }
    m = vector_top<HD>(m);
    const float scale = m < 0x7f800000u ? __uint_as_float(m) / 127.f : __uint_as_float(0x7fc00000u);
    const bool plain = scale > 0x1p-100f;   // not 0, not NaN, and its reciprocal a normal number
    const float inv = 1.f / scale;
    constexpr float kWhole = 12582912.f;
    uint32_t code[8];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = x[i] * inv, r = y + kWhole;
        off = fmaxf(off, fabsf(y - (r - kWhole)));
        code[i] = __float_as_uint(r);
    }
    if (__any(!plain || off > 0.49998f)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float r = scale > 0.f ? fminf(fmaxf(rintf(x[i] / scale), -127.f), 127.f) : 0.f;
            code[i] = (uint32_t)(int)r;
        }
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(code[4 * i + 1], code[4 * i], 0x0c0c0400u), up = __builtin_amdgcn_perm(code[4 * i + 3], code[4 * i + 2], 0x04000c0cu);
        w[i] = lo | up;
    }
    *codes = make_uint2(w[0], w[1]);
    return scale;
}

__device__ __forceinline__ void codes_to_floats(const uint2& c, float scale, float (&f)[8])
{
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)((int)(w[i >> 2] << (24 - 8 * (i & 3))) >> 24) * scale;
}

// Four bytes' codes as halves: two pairs chosen by sel_lo and sel_hi (byte numbers of b:a, zeros between them).
__device__ __forceinline__ uint32_t code_pair(uint32_t a, uint32_t b, uint32_t sel)
{
    const uint32_t u = __builtin_amdgcn_perm(b, a, sel) ^ 0x64806480u;   // 1024 + (code + 128) as halves
    const f16x2 h = __builtin_bit_cast(f16x2, u) - f16x2{(_Float16)1152.f, (_Float16)1152.f};
    return __builtin_bit_cast(uint32_t, h);
}

// ------------------------------------------------------------------------------------------ operands
template <typename C, typename T>
struct MathType { typedef T type; };           // 16-bit cache: its own type
template <typename T>
struct MathType<int8_t, T> { typedef _Float16 type; };

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// sum + a's two values, in fp32.
template <typename T>
__device__ __forceinline__ float add_pair(uint32_t a, float sum)
{
    typedef T t2 __attribute__((ext_vector_type(2)));
    const t2 one = {(T)1.f, (T)1.f};
    if constexpr (std::is_same<T, _Float16>::value) return __builtin_amdgcn_fdot2(__builtin_bit_cast(t2, a), one, sum, false);
    else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(t2, a), one, sum, false);
}

// f(head dim, tokens' type, cache's type) with values of those types and dims.
template <class F>
static void with_types(int hd, int token, int cache, F f)
{
    auto by_cache = [&](auto dim, auto t) {
        if (cache == kI8) f(dim, t, int8_t{});
        else if (cache == kF16) f(dim, t, _Float16{});
        else f(dim, t, __bf16{});
    };
    auto by_token = [&](auto dim) {
        if (token == kF16) by_cache(dim, _Float16{});
        else by_cache(dim, __bf16{});
    };
    if (hd == 128) by_token(std::integral_constant<int, 128>{});
    else by_token(std::integral_constant<int, 64>{});
}

}  // namespace ss

#endif
