// The 8-bit dense product of few bf16 rows in one launch (thin.h), their quantisation
// included.  Such a call is latency: of its launches, and of one pass over the rows and one
// over the weights.  So every workgroup quantises its 16 or 32 rows for itself into LDS (a
// wave a row at a time) while its first columns' weights are on their way, and its 16 waves share
// the contraction of one slab of columns, or of two.  Measured, this / a launch each for the codes
// and the tiles of gemm.hip: 2,688 x 672 1 row 5.2 / 17.4 us, 32 10.3 / 17.5, 192 11.3 / 18.0, 256 12.2 /
// 18.0, 700 15.1 / 18.4; 4,096 x 1,024 1 row 6.0 / 22.7, 128 13.3 / 24.0, 512 18.9 / 24.6; 512 x 512
// 256 rows 7.6 / 8.9, 1,024 8.3 / 9.0.
#include "kernels.h"
#include "quant8.h"
#include "thin.h"

namespace moe {

constexpr int kProjWaves = 16;
constexpr int kProjChunks = kProjKd / 8 / 64;

// 16 MB rows and 16 / WK slabs of 16 NB columns a workgroup; WK waves share a slab.
template <int MB, int NB, int WK>
__global__ __launch_bounds__(kProjWaves * 64) void proj_few_kernel(const uint16_t* __restrict__ A, int M, ThinArgs s) {
    using T = ThinI8<NB, false>;
    constexpr int P = 4 / NB, kPieces = MB * NB;   // steps ahead; 16 x 16 tiles of a slab
    constexpr int kCodes = 16 * MB * (kProjKd + 32) + T::kStep, kSums = kProjWaves * kPieces * 1024;
    constexpr bool kApart = kCodes + kSums < 160 * 1024 - 256;   // the waves' sums have LDS of their own
    static_assert(kSums <= kCodes, "sums take the codes' place");
    __shared__ __attribute__((aligned(16))) int8_t q[kCodes + (kApart ? kSums : 0)];
    __shared__ float scale[16 * MB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slab = wave / WK, kk = wave % WK;
    const int n0 = ((int)blockIdx.x * (kProjWaves / WK) + slab) * T::kCols;
    A += (int64_t)blockIdx.y * 16 * MB * s.Kd;
    s.out = (uint16_t*)s.out + (int64_t)blockIdx.y * 16 * MB * s.N;
    M -= blockIdx.y * 16 * MB;   // rows from this workgroup's first on
    const int nst = (s.Kd + T::kStep - 1) / T::kStep;
    const int mine = n0 < s.N && nst > kk ? (nst - kk + WK - 1) / WK : 0;
    const __amdgpu_buffer_rsrc_t rw = thin_rsrc(s.W, s.w_bytes);
    T w[P];
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (i < mine) w[i].load(rw, s, n0, (kk + WK * i) * T::kStep, lane);

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
            if (c < n)
                *(uint2*)&q[r * stride + c * 8] = make_uint2(codes4(z, v[i].x, v[i].y), codes4(z, v[i].z, v[i].w));
        }
    }
    __syncthreads();

    // Rows past M and codes past Kd read what LDS holds there: the former leave no
    // result, the latter meet zero weights.
    f32x4 acc[MB][NB];
#pragma unroll
    for (int v = 0; v < kPieces; ++v) acc[v / NB][v % NB] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < mine; i0 += P) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (i0 + i >= mine) break;
            const int k = (kk + WK * (i0 + i)) * T::kStep;
            typename T::template A<MB> a;
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    a.v[b][h] = *(const u32x4*)&q[(16 * b + (lane & 15)) * stride + k + 64 * h + 16 * (lane >> 4)];
            w[i].template mma<MB>(acc, a, nullptr);
            if (i0 + i + P < mine) w[i].load(rw, s, n0, k + WK * P * T::kStep, lane);
        }
    }
    if constexpr (!kApart) __syncthreads();   // the codes are read: the waves' sums take their place
    f32x4* const sums = (f32x4*)(q + (kApart ? kCodes : 0));
    auto sum = [&](int of, int v) -> f32x4& { return sums[(of * kPieces + v) * 64 + lane]; };
#pragma unroll
    for (int v = 0; v < kPieces; ++v) sum(wave, v) = acc[v / NB][v % NB];
    __syncthreads();
    for (int v = kk; v < kPieces; v += WK) {
        const int r = 16 * (v / NB) + (lane & 15), col = n0 + T::piece_col(v % NB, lane);
        if (r >= M || col >= s.N) continue;   // N is a multiple of 8
        f32x4 t = sum(slab * WK, v);
#pragma unroll
        for (int j = 1; j < WK; ++j) t = thin_add<true>(t, sum(slab * WK + j, v));
        const f32x4 cs = *(const f32x4*)(s.col_scale + col);
#pragma unroll
        for (int u = 0; u < 4; ++u) t[u] = (float)__float_as_int(t[u]) * scale[r] * cs[u];
        *(u32x2_thin*)((uint16_t*)s.out + (int64_t)r * s.N + col) =
            u32x2_thin{pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
    }
}

namespace {

// Columns of a workgroup that still make one round of workgroups, each of which fills a CU's LDS: 16,
// 32 or 64; 0 if those do not suffice.  The fewest (us with 16 / 32: 128 rows of 2,688 x 672 10.9 / 11.7, of
// 4,096 x 1,024 13.2 / 14.1).  More lose to the two launches (1,024 rows at 128 columns: 2,688 x 672
// 19.6 / 18.8, 4,096 x 1,024 28.2 / 26.0), and so do more than 16 of a short contraction, whose two
// launches are latency alone (256 rows of 48 x 1,000 8.5 / 7.7).
int proj_cols(int64_t M, int N, int Kd) {
    for (int cols = 16; cols <= (Kd < 256 ? 16 : 64); cols *= 2)
        if ((M + 31) / 32 * ((N + cols - 1) / cols) <= cu_count()) return cols;
    return M <= kProjFewRows ? 16 : 0;
}

}  // namespace

bool proj_few_fits(int64_t M, int N, int Kd) { return Kd <= kProjKd && proj_cols(M, N, Kd) > 0; }

hipError_t launch_proj_few(const moe_bf16* A, const int8_t* W, const float* w_scale, int64_t M, int N, int Kd,
                           moe_bf16* C, hipStream_t st) {
    if (M == 0) return hipSuccess;
    const ThinArgs s{nullptr, W, C, nullptr, w_scale, 0, (int64_t)N * Kd, 0, Kd, N, THIN_BF16};
    const int cols = M <= 16 ? 16 : proj_cols(M, N, Kd);
    const dim3 block(kProjWaves * 64), grid((unsigned)((N + cols - 1) / cols), (unsigned)((M + 31) / 32));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, A, (int)M, s); };
    if (M <= 16) go(proj_few_kernel<1, 1, 16>);
    else if (cols == 16) go(proj_few_kernel<2, 1, 16>);
    else if (cols == 32) go(proj_few_kernel<2, 2, 16>);
    else go(proj_few_kernel<2, 2, 8>);
    return launch_check(st);
}

// The grouped 8-bit product where experts have few rows: a workgroup takes one entry of the tile table, at most
// 128 rows of an expert, and one slab of 16 NB columns.  Its four waves share the contraction of up to 32 rows; of
// more rows, each takes 32 and the whole contraction, and nothing waits for another wave.
struct RowsThin {
    const int8_t* A;
    const float* a_scale;
    const int8_t* W;
    const float* w_scale;
    uint16_t* C;
    const int4* tiles;
    int Kd, N, groups, epi;
};
template <int NB, bool NT>
__global__ __launch_bounds__(kThinThreads, NB == 2 ? 4 : 3) void rows_thin_kernel(RowsThin p) {
    using T = ThinI8<NB, NT>;
    __shared__ __attribute__((aligned(16))) char lds[4 * T::kWaveLds];
    const int tile = blockIdx.x / p.groups, n0 = blockIdx.x % p.groups * T::kCols;
    const int4 t = p.tiles[tile];
    const int e = __builtin_amdgcn_readfirstlane(t.x), row0 = __builtin_amdgcn_readfirstlane(t.y);
    if (e < 0) return;
    const int nrows = __builtin_amdgcn_readfirstlane(t.z) - row0;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool few = nrows <= 32;
    const int r0 = few ? 0 : 32 * wave, n = min(nrows - r0, 32);
    if (n <= 0) return;
    const int64_t row = row0 + r0;
    const ThinArgs a{p.A + row * p.Kd, p.W + (int64_t)e * p.N * p.Kd, p.C + row * p.N, p.a_scale + row,
                     p.w_scale + (int64_t)e * p.N, (int64_t)n * p.Kd, (int64_t)p.N * p.Kd, p.Kd, p.Kd, p.N, p.epi};
    thin_rows<T, 2>(a, n0, few ? wave : 0, few ? 4 : 1, n, [](int i) { return i; }, [](int i) { return i; }, lds);
}

// Up to 20 rows an expert on average, whose loads the host does not know.  90 random expert FFNs (8 to 256 experts,
// 256 to 2,688 by 512 to 3,712, even and Zipf(0.7) loads) take of the tiles' time, by rows an expert: 4 to 8 0.65, 8 to
// 12 0.77, 12 to 16 0.81, 16 to 20 0.85 (of the drawn ones at most 0.99), 20 to 24 0.89 (1.04).  In us, tiles / this, even
// loads of 8 rows: 128 experts of 2,048 x 1,024 119 / 104, 1,024 of them 803 / 743; 24 of 2,688 x 3,520 129 / 91; 8 of 512 x
// 1,024 21.3 / 13.4.  An expert with many rows costs: its weights are read again for every 32 of them, and they for every
// slab.  16 rows an expert by Zipf(1.1): 128 experts 141 / 131, 256 226 / 240, 1,024 804 / 877; half of 20 rows an expert
// with one (two picks a token): 128 143 / 129, 1,024 892 / 913; all of them (one pick a token): 64 40 / 66, 256 58 / 108,
// 1,024 142 / 368.
bool rows_thin_pays(int E, int64_t R) { return R <= 20 * (int64_t)E; }

// Columns of a slab.  64 read the rows half as often as 32, which pays where there are more than 12 an expert, unless
// so few weights that the workgroups are few (64 MB: of the tiles' time with 32 / 64 columns, 12 to 20 rows, more
// weights 0.87 / 0.85, fewer 0.81 / 0.89; 8 to 12 rows 0.77 / 0.82).
static int rows_thin_cols(int E, int64_t R, int N, int Kd) {
    return R > 12 * (int64_t)E && (int64_t)E * N * Kd > (int64_t)64 << 20 ? 64 : 32;
}

hipError_t launch_rows_thin(const int8_t* A, const float* a_scale, const int8_t* W, const float* w_scale, void* C,
                            bool relu2, const int4* tiles, int max_tiles, int E, int64_t R, int N, int Kd,
                            hipStream_t st) {
    const int cols = rows_thin_cols(E, R, N, Kd), groups = (N + cols - 1) / cols;
    const RowsThin p{A, a_scale, W, w_scale, (uint16_t*)C, tiles, Kd, N, groups, relu2 ? THIN_RELU2 : THIN_BF16};
    const dim3 grid((unsigned)(max_tiles * groups)), block(kThinThreads);
    const bool nt = thin_nt(W, Kd, 2 * (R < E ? R : E) * N * Kd);   // the other projection's weights as many
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, p); };
    if (cols == 32) nt ? go(rows_thin_kernel<2, true>) : go(rows_thin_kernel<2, false>);
    else nt ? go(rows_thin_kernel<4, true>) : go(rows_thin_kernel<4, false>);
    return launch_check(st);
}

}  // namespace moe
