// The 8-bit dense product of few bf16 rows in one launch (thin.h), their quantisation
// included.  Such a call is latency: of its launches, and of one pass over the rows and one
// over the weights.  So every workgroup quantises its 16 or 32 rows for itself into LDS (a
// wave a row at a time) while its 16 columns' weights are on their way, and its 16 waves share
// the contraction.  Measured, this / a launch each for the codes and the tiles of
// gemm.hip: 2,688 x 672 1 row 5.3 / 17.4 us, 16 6.9 / 17.5, 32 10.4 / 17.6, 192 11.2 / 18.0; 4,096 x
// 1,024 1 row 6.0 / 23.5, 128 13.3 / 23.8; 512 x 512 256 rows 7.6 / 8.9.
#include "kernels.h"
#include "quant8.h"
#include "thin.h"

namespace moe {

constexpr int kProjWaves = 16;
constexpr int kProjCols = 16;
constexpr int kProjChunks = kProjKd / 8 / 64;

template <int MB>
__global__ __launch_bounds__(kProjWaves * 64) void proj_few_kernel(const uint16_t* __restrict__ A, int M, ThinArgs s) {
    using T = ThinI8<1, false>;
    constexpr int P = 4;
    static_assert(T::kCols == kProjCols, "a workgroup's columns");
    __shared__ __attribute__((aligned(16))) int8_t q[16 * MB * (kProjKd + 32) + T::kStep];
    __shared__ float scale[16 * MB];
    __shared__ f32x4 red[kProjWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * T::kCols;
    A += (int64_t)blockIdx.y * 16 * MB * s.Kd;
    s.out = (uint16_t*)s.out + (int64_t)blockIdx.y * 16 * MB * s.N;
    M -= blockIdx.y * 16 * MB;   // rows from this workgroup's first on
    const int nst = (s.Kd + T::kStep - 1) / T::kStep;
    const int mine = nst > wave ? (nst - wave + kProjWaves - 1) / kProjWaves : 0;
    const __amdgpu_buffer_rsrc_t rw = thin_rsrc(s.W, s.w_bytes);
    T w[P];
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (i < mine) w[i].load(rw, s, n0, (wave + kProjWaves * i) * T::kStep, lane);

    // rows an odd number of 16-byte chunks apart: the fragment reads of 16 rows spread over the banks
    const int stride = s.Kd + ((s.Kd / 16) & 1 ? 32 : 16);
    const int n = s.Kd / 8;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int r = wave + 16 * b;
        if (r >= M) break;
        uint4 v[kProjChunks];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kProjChunks; ++i) {
            const int c = lane + 64 * i;
            v[i] = c < n ? ((const uint4*)(A + (int64_t)r * s.Kd))[c] : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < kProjChunks; ++i)
            top = max_mag(max_mag(max_mag(max_mag(top, v[i].x), v[i].y), v[i].z), v[i].w);
        Quant8 z;
        z.init(wave_max_u32(top));
        if (lane == 0) scale[r] = z.scale;
#pragma unroll
        for (int i = 0; i < kProjChunks; ++i) {
            const int c = lane + 64 * i;
            if (c < n) *(uint2*)&q[r * stride + c * 8] = make_uint2(codes4(z, v[i].x, v[i].y), codes4(z, v[i].z, v[i].w));
        }
    }
    __syncthreads();

    // Rows past M and codes past Kd read what LDS holds there: the former leave no
    // result, the latter meet zero weights.
    f32x4 acc[MB][1];
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[b][0] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < mine; i0 += P) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (i0 + i >= mine) break;
            const int k = (wave + kProjWaves * (i0 + i)) * T::kStep;
            T::A<MB> a;
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    a.v[b][h] = *(const u32x4*)&q[(16 * b + (lane & 15)) * stride + k + 64 * h + 16 * (lane >> 4)];
            w[i].template mma<MB>(acc, a, nullptr);
            if (i0 + i + P < mine) w[i].load(rw, s, n0, k + kProjWaves * P * T::kStep, lane);
        }
    }
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        if (b > 0) __syncthreads();
        red[wave][lane] = acc[b][0];
        __syncthreads();
        const int r = 16 * b + (lane & 15), col = n0 + T::piece_col(0, lane);
        if (wave != 0 || r >= M || col >= s.N) continue;   // N is a multiple of 8
        f32x4 t = red[0][lane];
#pragma unroll
        for (int j = 1; j < kProjWaves; ++j) t = thin_add<true>(t, red[j][lane]);
        const f32x4 cs = *(const f32x4*)(s.col_scale + col);
#pragma unroll
        for (int u = 0; u < 4; ++u) t[u] = (float)__float_as_int(t[u]) * scale[r] * cs[u];
        *(u32x2_thin*)((uint16_t*)s.out + (int64_t)r * s.N + col) =
            u32x2_thin{pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
    }
}

// One round of workgroups, each of which fills a CU's LDS.
bool proj_few_fits(int64_t M, int N, int Kd) {
    return Kd <= kProjKd && (M <= kProjFewRows || (M + 31) / 32 * ((N + kProjCols - 1) / kProjCols) <= cu_count());
}

hipError_t launch_proj_few(const moe_bf16* A, const int8_t* W, const float* w_scale, int64_t M, int N, int Kd,
                           moe_bf16* C, hipStream_t st) {
    if (M == 0) return hipSuccess;
    const ThinArgs s{nullptr, W, C, nullptr, w_scale, 0, (int64_t)N * Kd, 0, Kd, N, THIN_BF16};
    const unsigned nx = (unsigned)((N + kProjCols - 1) / kProjCols);
    const dim3 block(kProjWaves * 64);
    if (M <= 16) hipLaunchKernelGGL(proj_few_kernel<1>, dim3(nx), block, 0, st, A, (int)M, s);
    else hipLaunchKernelGGL(proj_few_kernel<2>, dim3(nx, (unsigned)((M + 31) / 32)), block, 0, st, A, (int)M, s);
    return launch_check(st);
}

}  // namespace moe
