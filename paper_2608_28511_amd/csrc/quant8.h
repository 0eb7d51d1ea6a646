// 8-bit rows (internal to the library): the scale and the codes of a row or
// channel whose largest magnitude is a.
//   scale = a / 127,  code = 127 x / a rounded to the nearest integer, ties to even.
// Both are functions of bf16 values, so the codes are those of exact arithmetic:
// 127 x has at most 15 significant bits and a has 8, so a quotient is either half
// way between two integers or at least 2^-17 of itself away from that.  It is
// computed as x * (127 / a), within 2^-23, and rounded to a multiple of 16 of its last
// place (2^-20): that puts a tie, whose 8 bits are such a multiple, back where it is
// and moves no other quotient past one.  Adding 1.5 * 2^23 then rounds to the
// integer, which is left in the sum's low bits.
// A row of zeros has scale 0 and codes 0; a row that holds an infinity or a NaN
// has a NaN scale and codes 0, so that every product with it is NaN.
#pragma once

#include "common.h"

namespace moe {

struct Quant8 {
    float scale;      // of the row
    float pre, mul;   // x * pre * mul = 127 x / a; pre is a power of two that keeps 127 / a finite

    // top: the fp32 bits of the largest magnitude, over bits (a NaN's exceed infinity's)
    __device__ __forceinline__ void init(uint32_t top) {
        const bool fine = top < 0x7f800000u;
        const float m = __uint_as_float(top);
        scale = fine ? m / 127.f : __uint_as_float(0x7fc00000u);
        pre = m < 0x1p-100f ? 0x1p64f : 1.f;
        mul = fine && top != 0u ? 127.f / (m * pre) : 0.f;
    }
    __device__ __forceinline__ bool zero() const { return mul == 0.f; }   // every code is 0
    // The code of x in the low byte of the result, unless zero().
    __device__ __forceinline__ uint32_t code(float x) const {
        const float t = x * pre * mul;
        const float tie = __uint_as_float((__float_as_uint(t) + 8u) & ~15u);
        return __float_as_uint(tie + 0x1.8p23f);
    }
};

// The larger magnitude of a packed bf16 pair and the running maximum, as fp32 bits.
__device__ __forceinline__ uint32_t max_mag(uint32_t top, uint32_t pair) {
    return max(top, max((pair << 16) & 0x7fffffffu, pair & 0x7fff0000u));
}

// Four codes of two packed bf16 pairs, one byte each, lowest first.
__device__ __forceinline__ uint32_t codes4(const Quant8& s, uint32_t p0, uint32_t p1) {
    if (s.zero()) return 0u;
    const uint32_t lo = __builtin_amdgcn_perm(s.code(bf16_hi(p0)), s.code(bf16_lo(p0)), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(s.code(bf16_hi(p1)), s.code(bf16_lo(p1)), 0x04000c0cu);
    return lo | hi;
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

}  // namespace moe
