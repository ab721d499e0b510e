// Cells of 4 bits: e2m1 (0 .5 1 1.5 2 3 4 6 and a sign), two to a byte, times a power of two that 32 features of a token share: a byte, 2^(byte - 127), 255
// for a NaN.  The power is the smallest of which the largest of the 32 is at most seven: up to there six is off by no more than one power, which is half of the step
// between four and six; with the smallest of which it is at most six the other values would have steps twice as wide for those between.
//
// gfx950 converts a byte's two cells, with the power, in one instruction.  A byte of V is two features of one token, so that both have one power, and no token
// shares a byte with another: one by itself is appended, or moved, by stores of whole bytes.
#pragma once
#include "cells.h"

namespace patch {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }     // as the conversions take it: of the exponent's bits alone, whatever the others are

// The values of byte B of w (the low four bits first) times the power, as bf16; all of them are exact there.
template <int B>
__device__ __forceinline__ uint32_t pair_e2m1(uint32_t w, float power) {
    const bf16x2_t x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)w, power, B);
    return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ u32x4_t widen8_e2m1(uint32_t w, float power) {
    return u32x4_t{pair_e2m1<0>(w, power), pair_e2m1<1>(w, power), pair_e2m1<2>(w, power), pair_e2m1<3>(w, power)};
}
// Eight bytes, each two features of a key: eight keys of the one feature, and of the other.  p0, p1: the keys' powers.
struct Two8 { u32x4_t even, odd; };
__device__ __forceinline__ Two8 turn8_e2m1(uint32_t w0, uint32_t w1, uint32_t p0, uint32_t p1) {
    const auto power = [](uint32_t p, int b) { return __uint_as_float(b == 0 ? p << 23 : b == 1 ? p << 15 : b == 2 ? p << 7 : p >> 1); };    // of bits 23 .. 30 alone
    const uint32_t x[8] = {pair_e2m1<0>(w0, power(p0, 0)), pair_e2m1<1>(w0, power(p0, 1)), pair_e2m1<2>(w0, power(p0, 2)), pair_e2m1<3>(w0, power(p0, 3)),
                           pair_e2m1<0>(w1, power(p1, 0)), pair_e2m1<1>(w1, power(p1, 1)), pair_e2m1<2>(w1, power(p1, 2)), pair_e2m1<3>(w1, power(p1, 3))};
    Two8 t;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        t.even[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x05040100u);
        t.odd[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x07060302u);
    }
    return t;
}
// One value by itself.
__device__ __forceinline__ float e2m1_value(uint32_t code, uint32_t byte) { return __uint_as_float(pair_e2m1<0>(code & 15u, power_of(byte)) << 16); }

// The byte of 32 values whose largest magnitude is `top`: from 2^-100 (what is below half of half of that is zero) to 2^125 (six of that are finite in bf16; what
// is beyond becomes that).  255 where one is a NaN or infinite: pass a NaN or an infinity.
__device__ __forceinline__ uint32_t power_byte(float top) {
    const uint32_t u = __float_as_uint(top);
    if (u >= 0x7F800000u) return 255u;
    const int byte = (int)((u + 0x1FFFFFu) >> 23) - 2;           // a mantissa above 1.75 counts as the next power's: 7 = 1.75 * 4
    return (uint32_t)(byte < 27 ? 27 : byte > 252 ? 252 : byte);
}
// Eight values over the power, nearest, ties to even, beyond six: six.
__device__ __forceinline__ uint32_t pack8_e2m1(const Four& lo, const Four& hi, float power) {
    int u = 0;
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, lo.x[0], lo.x[1], power, 0);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, lo.x[2], lo.x[3], power, 1);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, hi.x[0], hi.x[1], power, 2);
    return (uint32_t)__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, hi.x[2], hi.x[3], power, 3);
}

}  // namespace patch
