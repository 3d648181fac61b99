// ls_codes.h - numbers of 4 and 8 bits that share a power of two by 32, as a quantised cache holds them.
//
// A group of 32 elements of a row has a scale byte b, which stands for 2^(b - 127), 255 for "no numbers"; an
// element's code is sign, exponent and mantissa of a small floating number: 1, 2 and 1 bits (0, 0.5, 1, 1.5, 2, 3, 4, 6) or
// 1, 4 and 3 (up to 448).  gfx950 converts between these and 16- or 32-bit numbers two at a time, the power of two
// among the operands: it takes the exponent field of a binary32 number, which is the scale byte as it is, and
// gives NaN where that is 255.  A code times a power of two has at most 4 significant bits, so a value is exact in 16 bits
// inside the type's range (float16 ends at 65504 and at 2^-24).
#pragma once

#include "ls_device.h"
#include "ls_ops_internal.h"

namespace ls {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int kGroup = 32;  // elements that share a scale

// The scale of a group whose largest magnitude is `top` is the smallest power of two that leaves top at most half a step
// beyond the largest code: top < 7 * 2^e (6, and half of the step from 4) or 464 * 2^e (448, and half of 32).  Both
// borders are a rounding of top's bits: add so much that the mantissa of a top at the border carries into the exponent.
struct Fp4 {
    static constexpr int kBits = 4;
    static constexpr uint32_t kCarry = 0x200000;  // 7 / 4 = 1.75
    static constexpr int kBelow = 2;              // 7 = 1.75 * 2^2
    static constexpr float kMost = 6.f;
    // largest e for which 6 * 2^e is a number of float16; of bfloat16 and binary32
    static constexpr int kMostExp16 = 13, kMostExp = 125;
};
struct Fp8 {
    static constexpr int kBits = 8;
    static constexpr uint32_t kCarry = 0x180000;  // 464 / 256 = 1.8125
    static constexpr int kBelow = 8;
    static constexpr float kMost = 448.f;
    static constexpr int kMostExp16 = 7, kMostExp = 119;
};

// The scale byte as the conversions take it.
__device__ inline float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two elements of a word of codes: elements 2 SEL and 2 SEL + 1.
template <class C, int SEL>
__device__ inline f16x2 widen2(uint32_t w, float s, _Float16) {
    if constexpr (C::kBits == 4) return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, SEL);
    else return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, SEL != 0);
}
template <class C, int SEL>
__device__ inline bf16x2 widen2(uint32_t w, float s, __bf16) {
    if constexpr (C::kBits == 4) return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL);
    else return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, SEL != 0);
}
template <class C, int SEL>
__device__ inline f32x2 widen2(uint32_t w, float s, float) {
    if constexpr (C::kBits == 4) return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, SEL);
    else return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, SEL != 0);
}

// Eight elements from one word of codes (4 bits) or two.
template <class C, typename T, typename V>
__device__ inline void widen8(const uint32_t* w, float s, V* out) {
    constexpr int hi = C::kBits == 4 ? 0 : 1;
    const auto a = widen2<C, 0>(w[0], s, T{}), b = widen2<C, 1>(w[0], s, T{});
    const auto c = widen2<C, hi ? 0 : 2>(w[hi], s, T{}), d = widen2<C, hi ? 1 : 3>(w[hi], s, T{});
    out[0][0] = a[0], out[0][1] = a[1], out[0][2] = b[0], out[0][3] = b[1];
    out[0][4] = c[0], out[0][5] = c[1], out[0][6] = d[0], out[0][7] = d[1];
}

// The code word or words of eight elements in fp32, to nearest, ties to the even code; beyond the largest code: the largest.
template <class C>
__device__ inline void narrow8(const float* x, float s, uint32_t* w) {
    if constexpr (C::kBits == 4) {
        uint32_t v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], s, 0);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[2], x[3], s, 1);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[4], x[5], s, 2);
        w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[6], x[7], s, 3);
    } else {
        // the conversion makes no number of what lies beyond its largest one
        const float most = C::kMost * s;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -most, most);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s16x2 v{};
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, y[4 * h], y[4 * h + 1], s, false);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, y[4 * h + 2], y[4 * h + 3], s, true);
            w[h] = __builtin_bit_cast(uint32_t, v);
        }
    }
}

// Words of codes at an address that is only a multiple of four.
typedef uint32_t u32x2a __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32x4a __attribute__((ext_vector_type(4), aligned(4)));

}  // namespace ls
