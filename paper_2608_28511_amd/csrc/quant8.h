// 8-bit rows (internal to the library): the scale and the codes of a row or
// channel whose largest magnitude is a.
//   scale = a / 127,  code = 127 x / a rounded to the nearest integer, ties to even.
// Both are functions of bf16 values, so the codes are those of exact arithmetic:
// 127 x has at most 15 significant bits and a has 8, so a quotient is either half
// way between two integers or at least 2^-17 of itself away from that, and only
// the ties need care when it is computed as x * (127 / a) with an error below 2^-22.
// A row of zeros has scale 0 and codes 0; a row that holds an infinity or a NaN
// has a NaN scale and codes 0, so that every product with it is NaN.
#pragma once

#include "common.h"

namespace moe {

struct Quant8 {
    float scale;      // of the row
    float pre, mul;   // x * pre * mul = 127 x / a; pre is a power of two that keeps 127 / a finite
    float a;          // a * pre

    // top: the fp32 bits of the largest magnitude, over bits (a NaN's exceed infinity's)
    __device__ __forceinline__ void init(uint32_t top) {
        const bool fine = top < 0x7f800000u;
        const float m = __uint_as_float(top);
        scale = fine ? m / 127.f : __uint_as_float(0x7fc00000u);
        pre = m < 0x1p-100f ? 0x1p64f : 1.f;
        a = m * pre;
        mul = fine && top != 0u ? 127.f / a : 0.f;
    }
    __device__ __forceinline__ int code(float x) const {
        if (mul == 0.f) return 0;   // uniform over the row: zeros, or not finite
        const float xs = x * pre;
        float q = rintf(xs * mul);
        const float e = fmaf(-q, a, 127.f * xs);   // exact: 127 xs and q a have at most 15 bits
        // half way: the even one of the two neighbours, whichever the product's error chose
        if (fabsf(e) * 2.f == a && ((int)q & 1)) q += copysignf(1.f, e);
        return (int)q;
    }
};

// The larger magnitude of a packed bf16 pair and the running maximum, as fp32 bits.
__device__ __forceinline__ uint32_t max_mag(uint32_t top, uint32_t pair) {
    return max(top, max((pair << 16) & 0x7fffffffu, pair & 0x7fff0000u));
}

// Four codes of two packed bf16 pairs, one byte each, lowest first.
__device__ __forceinline__ uint32_t codes4(const Quant8& s, uint32_t p0, uint32_t p1) {
    return (uint32_t)(s.code(bf16_lo(p0)) & 0xff) | (uint32_t)(s.code(bf16_hi(p0)) & 0xff) << 8 |
           (uint32_t)(s.code(bf16_lo(p1)) & 0xff) << 16 | (uint32_t)(s.code(bf16_hi(p1)) & 0xff) << 24;
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

}  // namespace moe
