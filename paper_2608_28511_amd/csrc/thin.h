// Products of at most 64 rows with weights that are read once (internal to the
// library): what bounds them is the reading, so weights go from memory to the matrix
// cores' operands in registers, several steps ahead, and never through LDS, where the
// wide tiles of gemm.hip keep theirs to use them again.  A slab of output columns belongs
// to one wave, or to the two or four waves of a workgroup that share its contraction and join
// their sums in LDS.
#pragma once

#include <type_traits>

#include "common.h"
#include "tile_dma.h"

namespace moe {

constexpr uint32_t kThinDrop = 0x80000000u;   // beyond any descriptor's range: reads as zero
constexpr int kThinNt = 2;                   // cache policy: non-temporal
constexpr int kThinThreads = 256;
constexpr int kThinRows = 64;
typedef unsigned u32x2_thin __attribute__((ext_vector_type(2)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t thin_rsrc(const void* base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int32_t)bytes, 0x00020000);
}

// What leaves a product: fp32, or bf16 of it, or its squared ReLU, in bf16 with 8-bit weights and
// in two bf16 parts with bf16 ones.
enum { THIN_F32 = 0, THIN_BF16 = 1, THIN_RELU2 = 2 };

// One expert's product.
struct ThinArgs {
    const void* A;              // its rows start within a_bytes
    const void* W;              // bf16 [Kd, N] or int8 [N, Kd]
    void* out;                  // [rows][N]; in two parts [rows][N / 8][2][8]
    const float* row_scale;     // 8-bit: by source row
    const float* col_scale;     // 8-bit: [N]
    int64_t a_bytes, w_bytes;
    int lda;                    // bytes
    int Kd, N;
    int epi;
};

// bf16 weights, N-contiguous: slabs of 64 columns, steps of 32 k.  A lane loads 4
// columns of 8 k rows (each load of the wave four whole cache lines) and packs them into
// the fragments of columns 4 c + q, q = 0 .. 3, with one byte permutation a register.  NT:
// non-temporal loads (see thin_nt).  PARTS: bf16 parts of A's values, whose products are
// summed; a row of A holds the first parts of eight values, then their second ones.
template <bool NT, int PARTS = 1>
struct ThinBf16 {
    static constexpr bool kI8 = false;
    static constexpr int kCols = 64, kStep = 32, kAcc = 4;
    static constexpr int kWaveLds = kAcc * 1024;   // bytes: the wave's sums
    template <int MB>
    static constexpr int kAhead = MB == 4 || PARTS == 2 ? 3 : 4;
    u32x2_thin w[8];

    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& rw, const ThinArgs& s, int n0, int k, int lane) {
        const int g = lane >> 4, c = lane & 15;
        const uint32_t ld = (uint32_t)s.N * 2;
        const uint32_t o = n0 + 4 * c < s.N ? (uint32_t)(k + 8 * g) * ld + (uint32_t)(n0 + 4 * c) * 2 : kThinDrop;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = __builtin_amdgcn_raw_buffer_load_b64(rw, o + (uint32_t)j * ld, 0, NT ? kThinNt : 0);
    }
    template <int MB>
    struct A {
        u32x4 v[MB][PARTS];
        __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& ra, const uint32_t (&row)[MB], int k, int Kd,
                                             int lane) {
            const int kk = k + 8 * (lane >> 4);
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    v[m][p] = __builtin_amdgcn_raw_buffer_load_b128(
                        ra, kk < Kd ? row[m] + (uint32_t)(kk * PARTS + 8 * p) * 2 : kThinDrop, 0, 0);
        }
    };
    template <int MB>
    __device__ __forceinline__ void mma(f32x4 (&acc)[MB][kAcc], const A<MB>& a, char*) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32x4 f;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                f[u] = __builtin_amdgcn_perm(w[2 * u + 1][q >> 1], w[2 * u][q >> 1], q & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    acc[m][q] =
                        mfma16<false>(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, a.v[m][p]), acc[m][q]);
        }
    }
    // acc[q][v] of a lane is column 16 g + 4 v + q of its token: piece v is four columns
    __device__ __forceinline__ static f32x4 piece(const f32x4 (&acc)[kAcc], int v) {
        return f32x4{acc[0][v], acc[1][v], acc[2][v], acc[3][v]};
    }
    __device__ __forceinline__ static int piece_col(int v, int lane) { return 16 * (lane >> 4) + 4 * v; }
};

// 8-bit weights, K-contiguous: slabs of 16 NB columns, steps of 128 k.  A fragment is 16
// bytes of each of 16 channels and four places: loaded as such, an instruction takes half of
// 16 cache lines.  NT: it takes eight whole ones, non-temporally, which the wave turns into
// fragments in 2 NB KB of LDS of its own (row layout of tile_dma.h).  Half lines ask for each
// line twice (16 tokens top-8 of 256: 188 us as they lie in memory, 202 with the hint, 166 with
// whole lines and the hint; from memory come 0.50 GB a product in all three, 0.495 of them
// weights), and whole lines alone cost the turn (3 tokens top-22 of 512: 53 / 59).  Two steps ahead: three cost a workgroup a CU (53 / 55.5).
template <int NB, bool NT>
struct ThinI8 {
    static constexpr bool kI8 = true;
    static constexpr int kCols = 16 * NB, kStep = 128, kAcc = NB;
    static constexpr int kWaveLds = NB * 2048;
    template <int MB>
    static constexpr int kAhead = 2;
    u32x4 w[NB][2];

    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& rw, const ThinArgs& s, int n0, int k, int lane) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = n0 + 16 * b + (NT ? 8 * h + (lane >> 3) : lane & 15);
                const int kk = k + (NT ? 16 * (lane & 7) : 64 * h + 16 * (lane >> 4));
                const uint32_t o = n < s.N && kk < s.Kd ? (uint32_t)n * (uint32_t)s.Kd + (uint32_t)kk : kThinDrop;
                w[b][h] = __builtin_amdgcn_raw_buffer_load_b128(rw, o, 0, NT ? kThinNt : 0);
            }
        }
    }
    template <int MB>
    struct A {
        u32x4 v[MB][2];
        __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& ra, const uint32_t (&row)[MB], int k, int Kd,
                                             int lane) {
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int kk = k + 64 * h + 16 * (lane >> 4);
                    v[m][h] = __builtin_amdgcn_raw_buffer_load_b128(ra, kk < Kd ? row[m] + (uint32_t)kk : kThinDrop, 0, 0);
                }
        }
    };
    // stage: the wave's LDS
    template <int MB>
    __device__ __forceinline__ void mma(f32x4 (&acc)[MB][kAcc], const A<MB>& a, char* stage) const {
        const int lane = threadIdx.x & 63;
        u32x4 f[NB][2];
        if constexpr (NT) {
            // a wave's LDS operations are done in order: the fences keep the compiler to it
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = 8 * h + (lane >> 3);
                    *(u32x4*)(stage + b * 2048 + r * 128 + (((lane & 7) ^ rswz(r)) * 16)) = w[b][h];
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = lane & 15, c = 4 * h + (lane >> 4);
                    f[b][h] = *(const u32x4*)(stage + b * 2048 + r * 128 + ((c ^ rswz(r)) * 16));
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) f[b][h] = w[b][h];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int m = 0; m < MB; ++m)
                    acc[m][b] = mfma16<true>(__builtin_bit_cast(bf16x8, f[b][h]), __builtin_bit_cast(bf16x8, a.v[m][h]),
                                             acc[m][b]);
    }
    __device__ __forceinline__ static f32x4 piece(const f32x4 (&acc)[kAcc], int b) { return acc[b]; }
    __device__ __forceinline__ static int piece_col(int b, int lane) { return 16 * b + 4 * (lane >> 4); }
};

template <bool I8>
__device__ __forceinline__ f32x4 thin_add(f32x4 a, f32x4 b) {
    if constexpr (I8)
        return __builtin_bit_cast(f32x4, __builtin_bit_cast(i32x4, a) + __builtin_bit_cast(i32x4, b));
    else
        return a + b;
}

// Columns [n0, n0 + kCols) of the product for 16 MB rows, of which nrows exist: dst(i) is
// row i's row in out and src(dst) its place in A.  The wave is the kk-th of the wk that share
// the slab: it takes every wk-th step, and their sums are joined through LDS in wave
// order, each wave finishing some of the slab's pieces.  lds: T::kWaveLds bytes of every wave.
// Every wave of the workgroup calls it (n0 may lie past N: such a slab has nothing to do).
template <class T, int MB, class Src, class Dst>
__device__ __forceinline__ void thin_body(const ThinArgs& s, int n0, int kk, int wk, int nrows, Src&& src, Dst&& dst,
                                          char* lds) {
    constexpr int P = T::template kAhead<MB>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nst = (s.Kd + T::kStep - 1) / T::kStep;
    const int mine = n0 < s.N && nst > kk ? (nst - kk + wk - 1) / wk : 0;
    const __amdgpu_buffer_rsrc_t rw = thin_rsrc(s.W, s.w_bytes);
    const __amdgpu_buffer_rsrc_t ra = thin_rsrc(s.A, s.a_bytes);
    f32x4 acc[MB][T::kAcc];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int q = 0; q < T::kAcc; ++q) acc[m][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    T w[P];
    typename T::template A<MB> a[P];
    auto step_k = [&](int i) { return (kk + wk * i) * T::kStep; };
    // the weights' first steps are on their way before the rows are known
#pragma unroll
    for (int q = 0; q < P; ++q)
        if (q < mine) w[q].load(rw, s, n0, step_k(q), lane);
    int to[MB], from[MB];
    uint32_t row[MB];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        const int i = m * 16 + (lane & 15);
        to[m] = i < nrows ? dst(i) : -1;
        from[m] = i < nrows ? src(to[m]) : 0;
        row[m] = i < nrows ? (uint32_t)from[m] * (uint32_t)s.lda : kThinDrop;
    }
#pragma unroll
    for (int q = 0; q < P; ++q)
        if (q < mine) a[q].load(ra, row, step_k(q), s.Kd, lane);
    for (int i0 = 0; i0 < mine; i0 += P) {
#pragma unroll
        for (int q = 0; q < P; ++q) {
            if (i0 + q >= mine) break;
            w[q].template mma<MB>(acc, a[q], lds + wave * T::kWaveLds);
            if (i0 + q + P < mine) {
                w[q].load(rw, s, n0, step_k(i0 + q + P), lane);
                a[q].load(ra, row, step_k(i0 + q + P), s.Kd, lane);
            }
        }
    }
    auto leave = [&](int m, int v, f32x4 t) {
        const int col = n0 + T::piece_col(v, lane);
        if (to[m] < 0 || col >= s.N) return;   // N is a multiple of 8
        if constexpr (T::kI8) {
            const float rs = s.row_scale[from[m]];
            const f32x4 cs = *(const f32x4*)(s.col_scale + col);
#pragma unroll
            for (int q = 0; q < 4; ++q) t[q] = (float)__float_as_int(t[q]) * rs * cs[q];
        }
        const int64_t at = (int64_t)to[m] * s.N + col;
        if (s.epi == THIN_F32) {
            *(f32x4*)((float*)s.out + at) = t;
        } else {
            if (s.epi == THIN_RELU2) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    t[q] = relu_f32(t[q]);
                    t[q] *= t[q];
                }
            }
            uint16_t* o = (uint16_t*)s.out + at;
            if constexpr (!T::kI8) {
                // The largest bf16 below the value, and the rest rounded to eight bits: within 2^-16 of it.
                // Neither part of a positive value is zero, so an infinite weight makes no NaN of it,
                // and an infinity is the largest bf16 and an infinity.
                o += at - (col & 4);
                f32x4 rest;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t below = __builtin_elementwise_sub_sat(__float_as_uint(t[q]), 1u);
                    const float first = __uint_as_float(below & 0xffff0000u);
                    rest[q] = t[q] - first;
                    t[q] = first;
                }
                *(u32x2_thin*)(o + 8) = u32x2_thin{pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3])};
            }
            *(u32x2_thin*)o = u32x2_thin{pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
        }
    };
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        if (m > 0 && m * 16 >= nrows) break;
        if (wk == 1) {
#pragma unroll
            for (int v = 0; v < T::kAcc; ++v) leave(m, v, T::piece(acc[m], v));
        } else {
            if (m > 0) __syncthreads();
            auto sum = [&](int w, int v) -> f32x4& { return ((f32x4*)(lds + w * T::kWaveLds))[v * 64 + lane]; };
#pragma unroll
            for (int v = 0; v < T::kAcc; ++v) sum(wave, v) = T::piece(acc[m], v);
            __syncthreads();
            const int first = wave - kk;
            for (int v = kk; v < T::kAcc; v += wk) {
                f32x4 t = sum(first, v);
                for (int j = 1; j < wk; ++j) t = thin_add<T::kI8>(t, sum(first + j, v));
                leave(m, v, t);
            }
        }
    }
}

// Whether weights [rows, row_bytes] at W, of which a call reads `bytes` in all, are better
// read non-temporally: not what the last-level cache (256 MB) may still hold from the call
// before, and not where rows do not start on cache lines, more of which are then read again
// (64 tokens top-22 of 512, rows of 1,344 bytes in bf16: 1.48 GB from memory for 1.09 of weights,
// with the hint 1.60; both products in 8 bits 1.14 / 1.33 for 1.09).  us, without / with the hint, each call on other weights than the one before, bf16: 64
// tokens of 64 experts of 2,048 x 1,024, 537 MB, 124 / 112; 8 of the 192-expert layer, 2.1 GB, 318 /
// 291; 64 tokens top-22 of 512, rows of 1,344 bytes among them, 437 / 445 and, those excepted, 416;
// 8 bits: 32 tokens top-16 of 256 of 1,024 x 1,536 142 / 124; 16 tokens top-8 of 256 of 2,048 x
// 2,688, 187 / 166.  Smaller calls may gain too where no call repeats the weights of the one before, and
// may lose where it does: bf16 4 tokens of 64 experts, 200 MB at most, 58.5 / 54.0 and 45.1 / 51.6 repeated;
// 1 token, 50 MB, 27.9 / 29.8 and 27.0 / 29.4; 8 bits 64 tokens of 64 experts, 256 MiB, 80.2 / 75.2
// and 76.3 / 74.0, of 48 65.7 / 67.5 and 60.1 / 65.1.
inline bool thin_nt(const void* W, int64_t row_bytes, int64_t bytes) {
    return bytes > (int64_t)256 << 20 && row_bytes % 128 == 0 && (uintptr_t)W % 128 == 0;
}

// thin_body for as few 16-row blocks as nrows needs, of at most MBMAX.
template <class T, int MBMAX, class Src, class Dst>
__device__ __forceinline__ void thin_rows(const ThinArgs& s, int n0, int kk, int wk, int nrows, Src&& src, Dst&& dst,
                                          char* lds) {
    if (MBMAX == 1 || nrows <= 16) thin_body<T, 1>(s, n0, kk, wk, nrows, src, dst, lds);
    else if (MBMAX == 2 || nrows <= 32) thin_body<T, MBMAX == 1 ? 1 : 2>(s, n0, kk, wk, nrows, src, dst, lds);
    else thin_body<T, MBMAX>(s, n0, kk, wk, nrows, src, dst, lds);
}

}  // namespace moe
