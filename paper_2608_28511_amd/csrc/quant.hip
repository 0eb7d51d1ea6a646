// 8-bit rows of activations and 8-bit output channels of weights (the format is in
// quant8.h).
#include <algorithm>

#include "kernels.h"
#include "quant8.h"
#include "schedule.h"

namespace moe {

// ROWS rows per wave (WAVES = 1, four waves a workgroup) or one per workgroup (WAVES =
// 16): a row is read once, CH 16-byte chunks a lane, and stays in registers between its
// maximum and its codes.  Eight chunks a lane are on their way before the first is used,
// whatever the rows' length.  With sched.tiles set, the last workgroup builds the
// grouped GEMM's tile tables instead.
template <int WAVES, int ROWS, int CH>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void quant_rows_kernel(
    const uint16_t* __restrict__ x, int64_t R, int D, int8_t* __restrict__ q, float* __restrict__ scale,
    const int32_t* __restrict__ offsets, int E, SchedPart small, SchedPart large) {
    static_assert(WAVES == 1 || ROWS == 1, "a workgroup of many waves takes one row");
    __shared__ uint32_t tops[WAVES];
    constexpr int kRowsPerWg = WAVES == 1 ? 4 * ROWS : 1;
    if (small.tiles != nullptr && blockIdx.x == gridDim.x - 1) {
        build_tile_schedule(offsets, E, (int)R, small, large);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t step = (int64_t)(gridDim.x - (small.tiles != nullptr ? 1 : 0)) * kRowsPerWg;
    const int first = WAVES == 1 ? lane : (int)threadIdx.x;
    const int n = D / 8;
    for (int64_t r0 = (int64_t)blockIdx.x * kRowsPerWg + (WAVES == 1 ? wave * ROWS : 0); r0 < R; r0 += step) {
        uint4 v[ROWS][CH];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int c = first + i * WAVES * 64;
                v[j][i] = c < n && r0 + j < R ? ld_nt((const uint4*)(x + (r0 + j) * D) + c) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const int64_t r = r0 + j;
            if (r >= R) break;
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < CH; ++i)
                top = max_mag(max_mag(max_mag(max_mag(top, v[j][i].x), v[j][i].y), v[j][i].z), v[j][i].w);
            top = wave_max_u32(top);
            if constexpr (WAVES > 1) {
                __syncthreads();   // the last row's maxima are read
                if (lane == 0) tops[wave] = top;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < WAVES; ++w) top = max(top, tops[w]);
            }
            Quant8 s;
            s.init(top);
            if (first == 0) scale[r] = s.scale;
            uint2* dst = (uint2*)(q + r * D);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int c = first + i * WAVES * 64;
                if (c < n) dst[c] = make_uint2(codes4(s, v[j][i].x, v[j][i].y), codes4(s, v[j][i].z, v[j][i].w));
            }
        }
    }
}

hipError_t launch_quant_rows(const moe_bf16* x, int64_t R, int D, int8_t* q, float* scale, hipStream_t st,
                             const int32_t* sched_offsets, int E, void* sched) {
    if (R == 0) return hipSuccess;
    SchedPart ss{}, sl{};
    unsigned extra = 0;
    if (sched != nullptr) {
        ss = sched_part(sched, E, R, false);
        sl = sched_part(sched, E, R, true);
        extra = 1;
    }
    auto go = [&](auto kernel, int rows, int threads) {   // in turns past 2^20 workgroups
        const int64_t need = (R + rows - 1) / rows;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(need, (int64_t)1 << 20) + extra), dim3(threads), 0, st, x, R, D,
                           q, scale, sched_offsets, E, ss, sl);
    };
    // Several rows a wave only where every CU has waves enough without them.
    const bool many = R >= 64 * (int64_t)cu_count();
    if (D <= 512 && many) go(quant_rows_kernel<1, 8, 1>, 32, 256);
    else if (D <= 1024 && many) go(quant_rows_kernel<1, 4, 2>, 16, 256);
    else if (D <= 2048) many ? go(quant_rows_kernel<1, 2, 4>, 8, 256) : go(quant_rows_kernel<1, 1, 4>, 4, 256);
    else if (D <= 4096) go(quant_rows_kernel<1, 1, 8>, 4, 256);
    else if (D <= 8192) go(quant_rows_kernel<1, 1, 16>, 4, 256);
    else go(quant_rows_kernel<16, 1, 8>, 1, 1024);
    return launch_check(st);
}

// One workgroup per expert and 64 output channels: a pass over the contraction for
// the channels' maxima, and one that transposes 64 x 64 codes at a time through LDS,
// so that every load is 128 bytes and every store 64 bytes of a channel.  The weights
// are laid out once; nothing on a call's path runs this.
constexpr int kQw = 64;
__global__ __launch_bounds__(256) void quant_weights_kernel(const uint16_t* __restrict__ W, int Kd, int N,
                                                            int8_t* __restrict__ Wq, float* __restrict__ scale) {
    __shared__ uint32_t top_s[32][kQw];
    // [channel][k], rows 16 bytes apart in the banks
    __shared__ __attribute__((aligned(16))) int8_t tile[kQw][kQw + 16];
    const int64_t e = blockIdx.y;
    const int n0 = blockIdx.x * kQw;
    const int c = (threadIdx.x & 7) * 8, kr = threadIdx.x >> 3;   // eight channels, one of 32 k rows
    const uint16_t* src = W + e * (int64_t)Kd * N + n0 + c;
    const bool in = n0 + c < N;   // N is a multiple of 8
    uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int k = kr; k < Kd && in; k += 32) {
        const uint4 v = *(const uint4*)(src + (int64_t)k * N);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            top[2 * u] = max(top[2 * u], (w[u] << 16) & 0x7fffffffu);
            top[2 * u + 1] = max(top[2 * u + 1], w[u] & 0x7fff0000u);
        }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) top_s[kr][c + u] = top[u];
    __syncthreads();
    Quant8 s[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        uint32_t m = 0;
        for (int j = 0; j < 32; ++j) m = max(m, top_s[j][c + u]);
        s[u].init(m);
        if (kr == 0 && in) scale[e * N + n0 + c + u] = s[u].scale;
    }
    const int ch = threadIdx.x >> 2, kc = (threadIdx.x & 3) * 16;   // a channel's 16 codes
    for (int k0 = 0; k0 < Kd; k0 += kQw) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + kr + 32 * h;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (in && k < Kd) v = *(const uint4*)(src + (int64_t)k * N);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                tile[c + 2 * u][kr + 32 * h] = s[2 * u].zero() ? 0 : (int8_t)s[2 * u].code(bf16_lo(w[u]));
                tile[c + 2 * u + 1][kr + 32 * h] =
                    s[2 * u + 1].zero() ? 0 : (int8_t)s[2 * u + 1].code(bf16_hi(w[u]));
            }
        }
        __syncthreads();
        if (n0 + ch < N && k0 + kc < Kd)   // Kd is a multiple of 16
            *(uint4*)(Wq + (e * N + n0 + ch) * (int64_t)Kd + k0 + kc) = *(const uint4*)&tile[ch][kc];
        __syncthreads();
    }
}

hipError_t launch_quant_weights(const moe_bf16* W, int E, int Kd, int N, int8_t* Wq, float* scale, hipStream_t st) {
    hipLaunchKernelGGL(quant_weights_kernel, dim3((unsigned)((N + kQw - 1) / kQw), (unsigned)E), dim3(256), 0, st, W,
                       Kd, N, Wq, scale);
    return launch_check(st);
}

}  // namespace moe
