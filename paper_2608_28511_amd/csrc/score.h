// Router scores as ordered integers, and row-wide reductions (shared by the top-K
// kernels).
#pragma once

#include "common.h"

namespace moe {

// Monotone map of an fp32 score to uint32 (larger score -> larger code).
// -0 is folded onto +0 and NaN maps to 1, below the code of -inf (0x007fffff,
// the smallest code of a number); 0 is left for experts already picked or
// past E, so that removing a pick is clearing its code.
__device__ __forceinline__ uint32_t score_code(float f) {
    if (f != f) return 1u;
    uint32_t u = __float_as_uint(f);
    if (u == 0x80000000u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float code_score(uint32_t c) {
    uint32_t u = (c & 0x80000000u) ? (c & 0x7fffffffu) : ~c;
    return __uint_as_float(u);
}

// Router score of the production variant (Section 5.2): the logistic
// sigmoid in fp32 (-inf -> 0, +inf -> 1).
__device__ __forceinline__ float sigmoid_f32(float l) { return 1.f / (1.f + expf(-l)); }

// Maximum over the lane's row of 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
    v = max(v, dpp_u32<0xB1>(v));    // quad_perm 1,0,3,2
    v = max(v, dpp_u32<0x4E>(v));    // quad_perm 2,3,0,1
    v = max(v, dpp_u32<0x141>(v));   // row_half_mirror
    return max(v, dpp_u32<0x140>(v));   // row_mirror
}

}  // namespace moe
