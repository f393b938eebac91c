// Numbers in 8 bits, in blocks of 32 with one power of two: x = element * 2^(scale - 127).  Elements have a sign, 4 exponent bits (of bias 7) and 3 mantissa bits: up to 448, steps of
// 2^-9 near zero, 0x7f with either sign is no number.  The power of two is a byte: 0 .. 254, 255 is no number (and none is written).
#pragma once
#include "hag_elem.hpp"

namespace hag {

constexpr int kScaleBlock = 32;

// The scale of a block from its largest amount (finite, sign bit clear): the smallest power of two that leaves it at most 448 = 1.75 * 2^8, 1 for a block of zeros.  A power of two costs no
// precision: it moves the elements' exponents, and these reach 2^18 below the largest.
__device__ __forceinline__ uint32_t scale_byte(float most) {
    const uint32_t bits = __float_as_uint(most), e = (bits + 0x1fffffu) >> 23;     // a mantissa above 1.75 carries
    return bits == 0 ? 127u : max(e, 8u) - 8u;
}
// 2^(127 - scale) for a scale of scale_byte, which is at most 248
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// |v| where it is a number, else 0
__device__ __forceinline__ float finite_amount(float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.f; }

// Four elements, the first in the low byte, to the nearest (ties to even); at most 448 in amount, or no number.
__device__ __forceinline__ uint32_t to_fp8(float a, float b, float c, float d) {
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

// Largest of groups of W adjacent lanes (a power of two), in every lane of the group.
template <int W>
__device__ __forceinline__ float lanes_max(float v) {
    if (W > 1) v = fmaxf(v, dpp_move<0xB1>(v));
    if (W > 2) v = fmaxf(v, dpp_move<0x4E>(v));
    if (W > 4) v = fmaxf(v, dpp_move<0x141>(v));
    if (W > 8) v = fmaxf(v, dpp_move<0x140>(v));
    if (W > 16) {
        const elem_u2_t s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = fmaxf(__uint_as_float(s.x), __uint_as_float(s.y));
    }
    return v;
}

}  // namespace hag
