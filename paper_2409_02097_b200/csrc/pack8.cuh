// The 8-bit checkpoint format of include/linfusion_layers.h on the device: 32 channels share a power of two.
//
// Why a power of two and whole numbers: x * 2^-e and code * 2^e are exact, so packing rounds once, reading not at all, and the
// same codes come out whatever computes them.  A value is off by at most half a step, max|x| / 127 of its group; against a scale of
// max|x| / 127 itself that costs half a bit on average.  (An 8-bit float of four significant bits is off by up to 1 / 16 of
// each value: for the activations of a layer several times as much in the 2-norm.)
#pragma once

#include "common.cuh"
#include "packed_math.cuh"

namespace lf {

// What a scale byte may be: e + 127 for e in -126 .. 121, or -24 .. 9 in fp16 (there the smallest step is the format's own, and
// 127 * 2^10 would pass its largest number; in bf16 127 * 2^122 would).
template <int KIND>
__device__ __forceinline__ constexpr int pack8_scale_min() { return kind_dtype(KIND) == kDtypeFp16 ? 103 : 1; }
template <int KIND>
__device__ __forceinline__ constexpr int pack8_scale_max() { return kind_dtype(KIND) == kDtypeFp16 ? 136 : 248; }

// The scale byte for the largest magnitude of a group (finite): with most = m * 2^E, 1 <= m < 2, the smallest e with
// m * 2^E <= 127 * 2^e is E - 6 for m <= 127 / 64, else E - 5; m's fraction above 0x7E0000 carries into the exponent below.
template <int KIND>
__device__ __forceinline__ int pack8_scale(float most)
{
    const int s = static_cast<int>((__float_as_uint(most) + 0x1FFFFu) >> 23) - 6;
    return min(max(s, pack8_scale_min<KIND>()), pack8_scale_max<KIND>());
}
__device__ __forceinline__ float pack8_step(int scale) { return __uint_as_float(static_cast<uint32_t>(scale) << 23); }
__device__ __forceinline__ float pack8_inverse_step(int scale) { return __uint_as_float(static_cast<uint32_t>(254 - scale) << 23); }

// |x|, or 0 where x is not finite.
__device__ __forceinline__ float finite_abs(float x)
{
    const float a = fabsf(x);
    return a < __uint_as_float(0x7f800000u) ? a : 0.0f;
}

// Four values -> four codes in a word.  Adding 1.5 * 2^23 leaves the nearest whole number (ties to even) in the low bits.
__device__ __forceinline__ uint32_t pack8_codes4(const float* x, float inverse)
{
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float r = fminf(fmaxf(x[i] * inverse, -127.0f), 127.0f);
        c[i] = __float_as_uint(r + 12582912.0f);
        if (!(fabsf(x[i]) < __uint_as_float(0x7f800000u))) c[i] = 0x80u;
    }
    return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
}

// Whether 2 * P values are all finite: 0 * x is NaN where one is not.
template <int P>
__device__ __forceinline__ bool all_finite(const f32x2 (&x)[P])
{
    f32x2 odd = both(0.0f);
#pragma unroll
    for (int i = 0; i < P; ++i) odd = fma2(x[i], both(0.0f), odd);
    return sum2(odd) == 0.0f;
}
// Four values -> four codes where all are finite and none passes 127 steps, which is nearly always: a code is the low byte of one
// fma, since x * 2^-e is exact and the sum with 1.5 * 2^23 rounds once.
__device__ __forceinline__ uint32_t pack8_codes4_plain(f32x2 x, f32x2 y, float inverse)
{
    const float2 a = unpack2(fma2(x, both(inverse), both(12582912.0f))), b = unpack2(fma2(y, both(inverse), both(12582912.0f)));
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}
// The largest magnitude of 2 * P values, of the finite ones where not all are.
template <int P>
__device__ __forceinline__ float largest(const f32x2 (&x)[P], bool plain)
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const float2 a = unpack2(x[i]);
        most = fmaxf(most, fmaxf(fabsf(a.x), fabsf(a.y)));
    }
    if (!plain) {
        most = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float2 a = unpack2(x[i]);
            most = fmaxf(most, fmaxf(finite_abs(a.x), finite_abs(a.y)));
        }
    }
    return most;
}
// 2 * P values -> codes, four in a word; plain: all finite.
template <int P>
__device__ __forceinline__ void pack8_codes(const f32x2 (&x)[P], float most, float inverse, bool plain, uint32_t (&w)[P / 2])
{
    if (plain && most * inverse <= 127.0f) {
#pragma unroll
        for (int j = 0; j < P / 2; ++j) w[j] = pack8_codes4_plain(x[2 * j], x[2 * j + 1], inverse);
    } else {
#pragma unroll
        for (int j = 0; j < P / 2; ++j) {
            const float2 a = unpack2(x[2 * j]), b = unpack2(x[2 * j + 1]);
            const float f[4] = {a.x, a.y, b.x, b.y};
            w[j] = pack8_codes4(f, inverse);
        }
    }
}

// Four codes -> four values; the code -128 -> the number of these bits (a NaN, or what a reader takes it for).  A code's byte with its top bit turned over, as the low byte of a float of 2^23, is 2^23 + 128 +
// code; the difference and the product are exact.  (One fma for both would overflow for steps above 2^104.)
__device__ __forceinline__ void unpack8_codes4(uint32_t word, float step, f32x2* x, uint32_t not_finite = 0x7fffffffu)
{
    const uint32_t w = word ^ 0x80808080u;
    const auto offset = [&](int i) { return __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 + i)); };
    x[0] = mul2(add2(pack2(offset(0), offset(1)), both(-8388736.0f)), both(step));
    x[1] = mul2(add2(pack2(offset(2), offset(3)), both(-8388736.0f)), both(step));
    // a byte of w that is zero was the code -128
    if (((w - 0x01010101u) & ~w & 0x80808080u) != 0u) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = unpack2(x[i / 2]);
            f[i] = ((word >> (8 * i)) & 0xffu) == 0x80u ? __uint_as_float(not_finite) : i % 2 == 0 ? a.x : a.y;
        }
        x[0] = pack2(f[0], f[1]);
        x[1] = pack2(f[2], f[3]);
    }
}

}  // namespace lf
