// Caches of 8-bit codes: quantisation and its inverse.
//
// A row of 64 features (K or V of a slot and head) is code * scale, int8 codes of at most 127 or fp8 (e4m3,
// at most 448), the scale the smallest power of two that keeps the row's largest value within them, at least 2^-100.
// A power of two costs int8 up to one of its bits, and e4m3 none; with it, code * scale has at most eight significant bits: it is
// a bf16 value, so the products of a bf16 cache take it without another rounding, and the quantisation's division
// is exact.  A row that holds a NaN or an infinity gets the scale NaN: whoever reads it sees that.
#pragma once

#include "rotary_device.hpp"

namespace vp {

// Scale of a row whose largest magnitude has the bits `top` (of the fp32 value), and its inverse (0 for NaN).
template <int CODE>
__device__ __forceinline__ float code_scale(uint32_t top, float* inv) {
    // 448 = 1.75 2^8, 127 = 1.984375 2^6
    const int lead = CODE == CODE_E4M3 ? 8 : 6;
    const uint32_t most = CODE == CODE_E4M3 ? 0x600000u : 0x7e0000u;
    int e = (int)(top >> 23) - 127 - lead + ((top & 0x7fffffu) > most);
    e = e < -100 ? -100 : e;
    const bool odd = top >= 0x7f800000u;
    *inv = odd ? 0.f : __uint_as_float((uint32_t)(127 - e) << 23);
    return odd ? __builtin_nanf("") : __uint_as_float((uint32_t)(e + 127) << 23);
}

// Rows whose largest code would stand for 2^128: the largest code that stands for a number (0: no such row).
template <int CODE>
__device__ __forceinline__ float code_limit(uint32_t top) {
    const bool most = CODE == CODE_E4M3 ? top > 0x7f600000u : top > 0x7f7e0000u;
    return most && top < 0x7f800000u ? (CODE == CODE_E4M3 ? 240.f : 63.f) : 0.f;
}

// Four codes of values that a scale has brought into range, the first in the lowest byte.
template <int CODE>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    if constexpr (CODE == CODE_E4M3) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    } else {
        const uint32_t x = (uint32_t)(int)__builtin_rintf(a) & 255u, y = (uint32_t)(int)__builtin_rintf(b) & 255u;
        const uint32_t z = (uint32_t)(int)__builtin_rintf(c) & 255u, w = (uint32_t)(int)__builtin_rintf(d);
        return x | y << 8 | z << 16 | w << 24;
    }
}

// A code's value (without scale) in bf16, exactly: features 0, 1 and 2, 3 of four.
template <int CODE>
__device__ __forceinline__ void decode4(uint32_t x, uint32_t* lo, uint32_t* hi) {
    if constexpr (CODE == CODE_E4M3) {
        *lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.f, false));
        *hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.f, true));
    } else {
        const bf16x2 a = {(bf16)(float)(int8_t)x, (bf16)(float)(int8_t)(x >> 8)};
        const bf16x2 b = {(bf16)(float)(int8_t)(x >> 16), (bf16)(float)(int8_t)(x >> 24)};
        *lo = __builtin_bit_cast(uint32_t, a);
        *hi = __builtin_bit_cast(uint32_t, b);
    }
}
template <int CODE>
__device__ __forceinline__ bf16x8 decode8(uint32_t x, uint32_t y) {
    u32x4 v;
    uint32_t a, b;
    decode4<CODE>(x, &a, &b);
    v[0] = a, v[1] = b;
    decode4<CODE>(y, &a, &b);
    v[2] = a, v[3] = b;
    return __builtin_bit_cast(bf16x8, v);
}
// Code times scale in fp32.
template <int CODE>
__device__ __forceinline__ void values4(uint32_t x, float s, float (&f)[4]) {
    if constexpr (CODE == CODE_E4M3) {
        uint32_t a, b;
        decode4<CODE>(x, &a, &b);
        f[0] = __uint_as_float(a << 16) * s;
        f[1] = __uint_as_float(a & 0xffff0000u) * s;
        f[2] = __uint_as_float(b << 16) * s;
        f[3] = __uint_as_float(b & 0xffff0000u) * s;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = (float)(int8_t)(x >> (8 * e)) * s;
    }
}

// Sixteen codes times their scale as bf16 values.  e4m3 with a power of two: the conversion scales by itself (by the
// exponent alone, so other scales take the product, and its rounding).
template <int CODE>
__device__ __forceinline__ void decode16(const u32x4& x, float s, u32x4 (&v)[2]) {
    if constexpr (CODE == CODE_E4M3) {
        const uint32_t b = __float_as_uint(s);
        const bool plain = (b & 0x807fffffu) == 0 && b != 0 && b < 0x7f800000u;
        if (__builtin_amdgcn_ballot_w64(!plain) == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j >> 1][2 * (j & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[j], s, false));
                v[j >> 1][2 * (j & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[j], s, true));
            }
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float f[4];
        values4<CODE>(x[j], s, f);
        const bf16x2 a = {(bf16)f[0], (bf16)f[1]}, b = {(bf16)f[2], (bf16)f[3]};
        v[j >> 1][2 * (j & 1)] = __builtin_bit_cast(uint32_t, a);
        v[j >> 1][2 * (j & 1) + 1] = __builtin_bit_cast(uint32_t, b);
    }
}

// The same in fp16, exact for code times scale within its range.  POWER: the scale is a power of two.
template <int CODE, bool POWER>
__device__ __forceinline__ void decode16_half(const u32x4& x, float s, u32x4 (&v)[2]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f16x2 a, b;
        if constexpr (CODE == CODE_E4M3 && POWER) {
            a = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x[j], s, false));
            b = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x[j], s, true));
        } else {
            float f[4];
            values4<CODE>(x[j], s, f);
            a = f16x2{(f16)f[0], (f16)f[1]}, b = f16x2{(f16)f[2], (f16)f[3]};
        }
        v[j >> 1][2 * (j & 1)] = __builtin_bit_cast(uint32_t, a);
        v[j >> 1][2 * (j & 1) + 1] = __builtin_bit_cast(uint32_t, b);
    }
}

// A slot's two scales.
__device__ __forceinline__ float key_scale(uint32_t s) { return __uint_as_float(s << 16); }
__device__ __forceinline__ float value_scale(uint32_t s) { return __uint_as_float(s & 0xffff0000u); }

}  // namespace vp
