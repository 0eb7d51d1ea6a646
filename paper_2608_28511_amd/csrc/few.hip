// A whole layer for at most 64 tokens (a decode step, a few drafted tokens).
//
// Such a call reads the picked experts' weights once and does little else, so what
// bounds it is HBM and, below some tens of megabytes, the latency of each launch.  No
// permutation is built: routed row r = t K + k keeps its place, and a workgroup of a
// product finds its expert and that expert's rows in the S K picks itself.
//
//   few_logits   partial router logits: 64 d x 64 experts x 16 tokens a workgroup, fp32 products
//   few_route    one workgroup a token: the partial sums, top-K and weights; with 8-bit
//                weights as many again quantise the token rows
//   few_gemm     up: h = bf16(max(x W1, 0)^2)
//   few_quant    8-bit weights: the rows of h
//   few_gemm     down: y_k = h W2 in fp32
//   few_combine  y = bf16(sum_k p_k y_k + shared), all sums in fp32 and fixed order
//
// few_gemm's matrix products take 16 tokens; weights go from memory to the matrix
// cores' operands in registers, several steps ahead, and never through LDS: every
// weight is used by one wave only.  The waves of a workgroup share a slab of output
// columns, each a part of its contraction.
#include <algorithm>

#include "kernels.h"
#include "quant8.h"
#include "score.h"
#include "tile_dma.h"

namespace moe {

constexpr uint32_t kFewDrop = 0x80000000u;   // beyond any descriptor's range: reads as zero
constexpr int kFewThreads = 256;
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t few_rsrc(const void* base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int32_t)bytes, 0x00020000);
}

// ---- router ---------------------------------------------------------------
// part[chunk][t][e] = sum over 64 d of x[t, d] Wr[d, e].  A lane is an expert and a
// wave 16 of the 64 d, whose weights it holds; token values are broadcast from LDS.
constexpr int kFewD = 64, kFewT = 16;
__global__ __launch_bounds__(kFewThreads) void few_logits_kernel(const uint16_t* __restrict__ x,
                                                                 const float* __restrict__ Wr, int S, int D, int E,
                                                                 float* __restrict__ part) {
    __shared__ float xs[kFewT][kFewD];
    __shared__ float red[4][kFewT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int d0 = blockIdx.x * kFewD, e = blockIdx.y * 64 + lane;
    const int t0 = blockIdx.z * kFewT, nt = S - t0 < kFewT ? S - t0 : kFewT;
    float w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int d = d0 + wave * 16 + i;
        w[i] = d < D && e < E ? Wr[(int64_t)d * E + e] : 0.f;
    }
    for (int c = threadIdx.x; c < nt * (kFewD / 8); c += kFewThreads) {
        const int t = c / (kFewD / 8), d = (c % (kFewD / 8)) * 8;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (d0 + d < D) v = *(const uint4*)(x + (int64_t)(t0 + t) * D + d0 + d);   // D is a multiple of 8
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            xs[t][d + 2 * q] = bf16_lo(u[q]);
            xs[t][d + 2 * q + 1] = bf16_hi(u[q]);
        }
    }
    __syncthreads();
    for (int t = 0; t < nt; ++t) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) a = fmaf(xs[t][wave * 16 + i], w[i], a);
        red[wave][t][lane] = a;
    }
    __syncthreads();
    if (e >= E) return;
    for (int t = wave; t < nt; t += 4)
        part[((int64_t)blockIdx.x * S + t0 + t) * E + e] =
            (red[0][t][lane] + red[1][t][lane]) + (red[2][t][lane] + red[3][t][lane]);
}

__device__ __forceinline__ uint32_t wave_max_code(uint32_t v) {
    v = row_max_u32(v);
    const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
    const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    return max(max(a, b), max(c, d));
}

// Workgroup t < S: token t's logits, its K best experts and their weights.  Its first
// wave picks: lane l holds experts l EPL .. + EPL - 1, so the lowest lane with the largest
// code holds the lowest expert.  Workgroup S + t (8-bit weights): token t's codes.
template <int EPL, bool SIG>
__global__ __launch_bounds__(kFewThreads) void few_route_kernel(
    const float* __restrict__ part, int nd, const float* __restrict__ bias, const float* __restrict__ sel_bias, int S,
    int E, int K, int32_t* __restrict__ topk_idx, float* __restrict__ topk_prob, const uint16_t* __restrict__ x, int D,
    int8_t* __restrict__ xq, float* __restrict__ xs) {
    __shared__ float lg[1024];
    __shared__ uint32_t tops[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if ((int)blockIdx.x >= S) {
        const int t = blockIdx.x - S;
        const uint4* src = (const uint4*)(x + (int64_t)t * D);
        uint32_t top = 0;
        for (int c = tid; c < D / 8; c += kFewThreads) {
            const uint4 v = src[c];
            top = max_mag(max_mag(max_mag(max_mag(top, v.x), v.y), v.z), v.w);
        }
        top = wave_max_u32(top);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        Quant8 s;
        s.init(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
        if (tid == 0) xs[t] = s.scale;
        for (int c = tid; c < D / 8; c += kFewThreads) {
            const uint4 v = src[c];
            ((uint2*)(xq + (int64_t)t * D))[c] = make_uint2(codes4(s, v.x, v.y), codes4(s, v.z, v.w));
        }
        return;
    }
    const int t = blockIdx.x;
    for (int e = tid; e < E; e += kFewThreads) {
        float a = 0.f;
#pragma unroll 8
        for (int c = 0; c < nd; ++c) a += part[((int64_t)c * S + t) * E + e];
        lg[e] = bias != nullptr ? a + bias[e] : a;
    }
    __syncthreads();
    if (wave != 0) return;

    uint32_t code[EPL], top = 0u;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        const int e = lane * EPL + i;
        code[i] = 0u;
        if (e < E) {
            float s = lg[e];
            if constexpr (SIG) s = sigmoid_f32(s) + (sel_bias != nullptr ? sel_bias[e] : 0.f);
            code[i] = score_code(s);
        }
        top = max(top, code[i]);
    }
    int my_e = 0;
    uint32_t my_c = 0u;
    for (int k = 0; k < K; ++k) {   // K <= E: the maximum is never a cleared code
        const uint32_t m = wave_max_code(top);
        const int owner = __builtin_ctzll(__ballot(top == m));
        int i_sel = 0;
#pragma unroll
        for (int i = EPL - 1; i >= 0; --i) i_sel = code[i] == m ? i : i_sel;
        const int e = __builtin_amdgcn_readlane(lane * EPL + i_sel, owner);
        if (lane == owner) {
            top = 0u;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                code[i] = i == i_sel ? 0u : code[i];
                top = max(top, code[i]);
            }
        }
        if (lane == k) {
            my_e = e;
            my_c = m;
        }
    }
    float z = 0.f;
    if constexpr (SIG) {
        if (lane < K) z = sigmoid_f32(lg[my_e]);
    } else {
        const float best = code_score(__builtin_amdgcn_readlane(my_c, 0));
        if (lane < K) z = expf(code_score(my_c) - best);
    }
    float sum = z;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) sum += __shfl_xor(sum, m);   // K <= 32: the first 32 lanes
    if (lane < K) {
        topk_idx[t * K + lane] = my_e;
        topk_prob[t * K + lane] = z / sum;
    }
}

// ---- products -------------------------------------------------------------
// One kind of expert (the E routed ones, or the shared one) of one product.
struct FewSide {
    const void* A;       // rows of lda bytes; routed row r reads row r / a_div
    const void* W;       // bf16 [Kd, N] or int8 [N, Kd] per expert
    void* out;           // [rows][N]: h in bf16 (up) or y in fp32 (down)
    const float* row_scale;     // 8-bit: of A's rows
    const float* col_scale;     // 8-bit: [experts][N]
    int64_t a_bytes, w_bytes;   // of A, of one expert's W
    int lda, a_div;
    int Kd, N;
    int groups;          // workgroups an expert takes
};
struct FewGemmArgs {
    FewSide routed, shared;
    const int32_t* idx;   // [S, K]
    int S, K, r_items;    // workgroups of the routed experts
    int wk;               // waves that share a slab's contraction; 4 / wk slabs side by side in a workgroup
    int up;
};

// The a-th expert (ascending) among the n picks and its rows, in order, in rows[];
// returns the expert, or -1 if fewer are picked.  Every thread of the workgroup calls it.
__device__ __forceinline__ int few_plan(const int32_t* __restrict__ idx, int n, int a, uint32_t* seen, int32_t* picks,
                                        int32_t* rows, int32_t* nrows) {
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < 32) seen[tid] = 0u;
    __syncthreads();
    for (int q = tid; q < n; q += kFewThreads) {
        const int e = idx[q] & 1023;   // E <= 1024
        picks[q] = e;
        atomicOr(&seen[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    const uint32_t word = lane < 32 ? seen[lane] : 0u;
    int incl = __popc(word);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    const uint64_t past = __ballot(lane < 32 && incl > a);
    if (past == 0) return -1;
    const int wi = __builtin_ctzll(past);
    uint32_t bits = __builtin_amdgcn_readlane(word, wi);
    int skip = a - (__builtin_amdgcn_readlane(incl, wi) - __popc(bits));
    while (skip-- > 0) bits &= bits - 1u;
    const int e = wi * 32 + __builtin_ctz(bits);
    if (tid < 64) {
        int at = 0;
        for (int q0 = 0; q0 < n; q0 += 64) {
            const bool hit = q0 + lane < n && picks[q0 + lane] == e;
            const uint64_t m = __ballot(hit);
            const int pos = at + __popcll(m & ((1ull << lane) - 1ull));
            if (hit && pos < kFewMaxTokens) rows[pos] = q0 + lane;   // a token picks an expert once
            at += __popcll(m);
        }
        if (lane == 0) *nrows = at < kFewMaxTokens ? at : kFewMaxTokens;
    }
    return e;
}

// bf16 weights, N-contiguous: slabs of 64 columns, steps of 32 k.  A lane loads 4
// columns of 8 k rows (each load of the wave four whole cache lines) and packs them into
// the fragments of columns 4 c + q, q = 0 .. 3, with one byte permutation a register.
struct FewBf16 {
    static constexpr bool kI8 = false;
    static constexpr int kCols = 64, kStep = 32, kAcc = 4;
    template <int MB>
    static constexpr int kAhead = MB == 4 ? 3 : 4;
    u32x2 w[8];

    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& rw, const FewSide& s, int n0, int k, int lane) {
        const int g = lane >> 4, c = lane & 15;
        const uint32_t ld = (uint32_t)s.N * 2;
        const uint32_t o = n0 + 4 * c < s.N ? (uint32_t)(k + 8 * g) * ld + (uint32_t)(n0 + 4 * c) * 2 : kFewDrop;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = __builtin_amdgcn_raw_buffer_load_b64(rw, o + (uint32_t)j * ld, 0, 0);
    }
    template <int MB>
    struct A {
        u32x4 v[MB];
        __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& ra, const uint32_t (&row)[MB], int k, int Kd,
                                             int lane) {
            const int kk = k + 8 * (lane >> 4);
#pragma unroll
            for (int m = 0; m < MB; ++m)
                v[m] = __builtin_amdgcn_raw_buffer_load_b128(ra, kk < Kd ? row[m] + (uint32_t)kk * 2 : kFewDrop, 0, 0);
        }
    };
    template <int MB>
    __device__ __forceinline__ void mma(f32x4 (&acc)[MB][kAcc], const A<MB>& a) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32x4 f;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                f[u] = __builtin_amdgcn_perm(w[2 * u + 1][q >> 1], w[2 * u][q >> 1], q & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int m = 0; m < MB; ++m)
                acc[m][q] = mfma16<false>(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, a.v[m]), acc[m][q]);
        }
    }
    // acc[q][v] of a lane is column 16 g + 4 v + q of its token: piece v is four columns
    __device__ __forceinline__ static f32x4 piece(const f32x4 (&acc)[kAcc], int v) {
        return f32x4{acc[0][v], acc[1][v], acc[2][v], acc[3][v]};
    }
    __device__ __forceinline__ static int piece_col(int v, int lane) { return 16 * (lane >> 4) + 4 * v; }
};

// 8-bit weights, K-contiguous: slabs of 32 columns, steps of 128 k, whose fragments
// are 16 bytes of a channel as they lie in memory.
struct FewI8 {
    static constexpr bool kI8 = true;
    static constexpr int kCols = 32, kStep = 128, kAcc = 2;
    template <int MB>
    static constexpr int kAhead = MB == 4 ? 2 : 3;
    u32x4 w[2][2];

    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& rw, const FewSide& s, int n0, int k, int lane) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int n = n0 + 16 * b + (lane & 15);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int kk = k + 64 * h + 16 * (lane >> 4);
                const uint32_t o = n < s.N && kk < s.Kd ? (uint32_t)n * (uint32_t)s.Kd + (uint32_t)kk : kFewDrop;
                w[b][h] = __builtin_amdgcn_raw_buffer_load_b128(rw, o, 0, 0);
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
                    v[m][h] = __builtin_amdgcn_raw_buffer_load_b128(ra, kk < Kd ? row[m] + (uint32_t)kk : kFewDrop, 0, 0);
                }
        }
    };
    template <int MB>
    __device__ __forceinline__ void mma(f32x4 (&acc)[MB][kAcc], const A<MB>& a) const {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int m = 0; m < MB; ++m)
                    acc[m][b] = mfma16<true>(__builtin_bit_cast(bf16x8, w[b][h]), __builtin_bit_cast(bf16x8, a.v[m][h]),
                                             acc[m][b]);
    }
    __device__ __forceinline__ static f32x4 piece(const f32x4 (&acc)[kAcc], int b) { return acc[b]; }
    __device__ __forceinline__ static int piece_col(int b, int lane) { return 16 * b + 4 * (lane >> 4); }
};

template <bool I8>
__device__ __forceinline__ f32x4 few_add(f32x4 a, f32x4 b) {
    if constexpr (I8)
        return __builtin_bit_cast(f32x4, __builtin_bit_cast(i32x4, a) + __builtin_bit_cast(i32x4, b));
    else
        return a + b;
}

// Columns [n0, n0 + kCols) of the product for 16 MB rows of expert e.  The wave is the
// kk-th of the wk that share the slab: it takes every wk-th step, and their sums are
// joined through LDS in wave order, each wave finishing some of the slab's pieces.
// Every wave of the workgroup calls it (n0 may lie past N: such a slab has nothing to do).
template <class T, int MB>
__device__ __forceinline__ void few_body(const FewGemmArgs& p, const FewSide& s, int e, int n0, int kk, int wk,
                                         const int32_t* rows, int nrows, f32x4 (*red)[T::kAcc][64]) {
    constexpr int P = T::template kAhead<MB>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nst = (s.Kd + T::kStep - 1) / T::kStep;
    const int mine = n0 < s.N && nst > kk ? (nst - kk + wk - 1) / wk : 0;
    const __amdgpu_buffer_rsrc_t rw = few_rsrc((const char*)s.W + e * s.w_bytes, s.w_bytes);
    const __amdgpu_buffer_rsrc_t ra = few_rsrc(s.A, s.a_bytes);
    uint32_t row[MB];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        const int i = m * 16 + (lane & 15);
        row[m] = i < nrows ? (uint32_t)(rows[i] / s.a_div) * (uint32_t)s.lda : kFewDrop;
    }
    f32x4 acc[MB][T::kAcc];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int q = 0; q < T::kAcc; ++q) acc[m][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    T w[P];
    typename T::template A<MB> a[P];
    auto load = [&](int slot, int i) {
        const int k = (kk + wk * i) * T::kStep;
        w[slot].load(rw, s, n0, k, lane);
        a[slot].load(ra, row, k, s.Kd, lane);
    };
#pragma unroll
    for (int q = 0; q < P; ++q)
        if (q < mine) load(q, q);
    for (int i0 = 0; i0 < mine; i0 += P) {
#pragma unroll
        for (int q = 0; q < P; ++q) {
            if (i0 + q >= mine) break;
            w[q].template mma<MB>(acc, a[q]);
            if (i0 + q + P < mine) load(q, i0 + q + P);
        }
    }
    auto leave = [&](int m, int v, f32x4 t) {
        const int i = m * 16 + (lane & 15), col = n0 + T::piece_col(v, lane);
        if (i >= nrows || col >= s.N) return;   // N is a multiple of 8
        const int r = rows[i];
        if constexpr (T::kI8) {
            const float rs = s.row_scale[r / s.a_div];
            const f32x4 cs = *(const f32x4*)(s.col_scale + (int64_t)e * s.N + col);
#pragma unroll
            for (int q = 0; q < 4; ++q) t[q] = (float)__float_as_int(t[q]) * rs * cs[q];
        }
        const int64_t at = (int64_t)r * s.N + col;
        if (p.up) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                t[q] = relu_f32(t[q]);
                t[q] *= t[q];
            }
            *(u32x2*)((uint16_t*)s.out + at) = u32x2{pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
        } else {
            *(f32x4*)((float*)s.out + at) = t;
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
#pragma unroll
            for (int v = 0; v < T::kAcc; ++v) red[wave][v][lane] = T::piece(acc[m], v);
            __syncthreads();
            const int first = wave - kk;
            for (int v = kk; v < T::kAcc; v += wk) {
                f32x4 t = red[first][v][lane];
                for (int j = 1; j < wk; ++j) t = few_add<T::kI8>(t, red[first + j][v][lane]);
                leave(m, v, t);
            }
        }
    }
}

// MBMAX = 1: at most 16 tokens, so at most 16 rows an expert; four waves a SIMD.
template <class T, int MBMAX>
__global__ __launch_bounds__(kFewThreads, MBMAX == 1 ? 4 : 2) void few_gemm_kernel(FewGemmArgs p) {
    __shared__ uint32_t seen[32];
    __shared__ int32_t picks[(MBMAX == 1 ? 16 : kFewMaxTokens) * 32], rows[kFewMaxTokens], nrows_s;
    __shared__ f32x4 red[4][T::kAcc][64];   // wk > 1: every wave's sums
    const bool shared = (int)blockIdx.x >= p.r_items;
    const int b = (int)blockIdx.x - (shared ? p.r_items : 0);
    const FewSide s = shared ? p.shared : p.routed;
    const int a = b / s.groups, in = b - a * s.groups;
    int e = 0;
    if (shared) {
        if ((int)threadIdx.x < p.S) rows[threadIdx.x] = threadIdx.x;
        if (threadIdx.x == 0) nrows_s = p.S;
    } else {
        e = few_plan(p.idx, p.S * p.K, a, seen, picks, rows, &nrows_s);
        if (e < 0) return;
    }
    __syncthreads();
    const int nrows = __builtin_amdgcn_readfirstlane(nrows_s);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = p.wk;
    const int kk = wave & (wk - 1), wn = wave / wk;
    const int n0 = (in * (4 / wk) + wn) * T::kCols;
    if (MBMAX == 1 || nrows <= 16) few_body<T, 1>(p, s, e, n0, kk, wk, rows, nrows, red);
    else if (nrows <= 32) few_body<T, MBMAX == 1 ? 1 : 2>(p, s, e, n0, kk, wk, rows, nrows, red);
    else few_body<T, MBMAX == 1 ? 1 : 4>(p, s, e, n0, kk, wk, rows, nrows, red);
}

// ---- between the products and after them ------------------------------------
struct FewRows {
    const uint16_t* h;   // [rows][F]
    int8_t* q;
    float* scale;
    int F, rows;
};

// 8-bit rows of the activations, one workgroup a row: the routed experts', then the
// shared one's.
__global__ __launch_bounds__(kFewThreads) void few_quant_kernel(FewRows routed, FewRows shared) {
    __shared__ uint32_t tops[4];
    const bool sh = (int)blockIdx.x >= routed.rows;
    const FewRows p = sh ? shared : routed;
    const int64_t row = (int)blockIdx.x - (sh ? routed.rows : 0);
    const int tid = threadIdx.x;
    const uint4* src = (const uint4*)(p.h + row * p.F);
    uint2* dst = (uint2*)(p.q + row * p.F);
    const int n = p.F / 8;
    uint4 v[2];   // the row's first 4,096 elements stay in registers
    uint32_t top = 0;
    for (int i = 0; i * kFewThreads < n; ++i) {
        const int c = tid + i * kFewThreads;
        const uint4 u = c < n ? src[c] : make_uint4(0u, 0u, 0u, 0u);
        if (i == 0) v[0] = u;
        if (i == 1) v[1] = u;
        top = max_mag(max_mag(max_mag(max_mag(top, u.x), u.y), u.z), u.w);
    }
    top = wave_max_u32(top);
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    Quant8 s;
    s.init(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
    if (tid == 0) p.scale[row] = s.scale;
    for (int i = 0; i * kFewThreads < n; ++i) {
        const int c = tid + i * kFewThreads;
        if (c >= n) break;
        const uint4 u = i == 0 ? v[0] : i == 1 ? v[1] : src[c];
        dst[c] = make_uint2(codes4(s, u.x, u.y), codes4(s, u.z, u.w));
    }
}

// Sixty-four groups of four columns a workgroup; a wave takes every fourth expert of
// the token's K, so that at most eight loads follow each other, and the waves' sums are
// added in order.
__global__ __launch_bounds__(kFewThreads) void few_combine_kernel(const float* __restrict__ yk,
                                                                  const float* __restrict__ ys,
                                                                  const float* __restrict__ prob, int K, int D,
                                                                  uint16_t* __restrict__ y) {
    __shared__ f32x4 sum[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.y, d = (blockIdx.x * 64 + lane) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (d < D) {
        f32x4 u[8];
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = wave + 4 * i;
            w[i] = 0.f;
            if (k < K) {
                w[i] = prob[t * K + k];
                u[i] = *(const f32x4*)(yk + (int64_t)(t * K + k) * D + d);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (wave + 4 * i < K) {
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = fmaf(w[i], u[i][q], v[q]);
            }
        if (wave == 3 && ys != nullptr) v += *(const f32x4*)(ys + (int64_t)t * D + d);
    }
    sum[wave][lane] = v;
    __syncthreads();
    if (wave != 0 || d >= D) return;
    v = ((sum[0][lane] + sum[1][lane]) + sum[2][lane]) + sum[3][lane];
    *(u32x2*)(y + (int64_t)t * D + d) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// ---- host -------------------------------------------------------------------
namespace {

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

int cdiv(int a, int b) { return (a + b - 1) / b; }

struct FewPlan {
    int nd, r_experts;
    int wk1, wk2;          // waves that share a slab of the up and of the down product
    size_t part, idx, prob, xq, xs, h, hs, hq, hqs, sc, scs, y, ys, bytes;   // offsets
};

// Waves of a workgroup's four that share a slab's contraction, each keeping a step.  Four
// give the most workgroups, which the CUs then share evenly (us with 1 / 2 / 4, one product's
// choice varied: 8 tokens of 192 experts 382 / 354 / 347; 1 token of 64 40 / 31 / 26.5); with many
// picks two, since every workgroup searches them all (64 tokens of 64 experts: 116 / 119 / 121
// and 119 / 120 / 127; 32 of 256: 302 / 290 / 283 and 303 / 300 / 314).
int few_share(int picks, int steps) {
    const int most = picks > 256 ? 2 : 4;
    return std::min(most, steps >= 4 ? 4 : steps >= 2 ? 2 : 1);
}

FewPlan few_plan_of(const moe_layer_few_args* a) {
    FewPlan p{};
    const int S = (int)a->S, D = a->D, E = a->E, K = a->K, F = a->F, Fs = a->Fs;
    const bool i8 = a->weights == MOE_WEIGHTS_I8;
    const size_t R = (size_t)S * K;
    const int step = i8 ? FewI8::kStep : FewBf16::kStep;
    p.nd = cdiv(D, kFewD);
    p.r_experts = (int)std::min<size_t>((size_t)E, R);
    p.wk1 = few_share((int)R, cdiv(D, step));
    p.wk2 = few_share((int)R, cdiv(F, step));
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += up256(bytes);
        return o;
    };
    p.part = take((size_t)p.nd * S * E * 4);
    p.idx = take(R * 4);
    p.prob = take(R * 4);
    p.xq = take(i8 ? (size_t)S * D : 0);
    p.xs = take((size_t)S * 4);
    p.h = take(R * F * 2);
    p.hs = take((size_t)S * Fs * 2);
    p.hq = take(i8 ? R * F : 0);
    p.hqs = take(i8 ? (size_t)S * Fs : 0);
    p.sc = take(R * 4);
    p.scs = take((size_t)S * 4);
    p.y = take(R * D * 4);
    p.ys = take(Fs ? (size_t)S * D * 4 : 0);
    p.bytes = at;
    return p;
}

template <int EPL>
void launch_route_few(bool sig, dim3 g, hipStream_t st, const float* part, int nd, const moe_layer_few_args* a,
                      int32_t* idx, float* prob, int8_t* xq, float* xs) {
    if (sig)
        hipLaunchKernelGGL((few_route_kernel<EPL, true>), g, dim3(kFewThreads), 0, st, part, nd, a->router_bias,
                           a->sel_bias, (int)a->S, a->E, a->K, idx, prob, a->x, a->D, xq, xs);
    else
        hipLaunchKernelGGL((few_route_kernel<EPL, false>), g, dim3(kFewThreads), 0, st, part, nd, a->router_bias,
                           a->sel_bias, (int)a->S, a->E, a->K, idx, prob, a->x, a->D, xq, xs);
}

}  // namespace

size_t layer_few_ws_bytes(const moe_layer_few_args* a) { return few_plan_of(a).bytes; }

hipError_t launch_layer_few(const moe_layer_few_args* a, hipStream_t st) {
    const FewPlan p = few_plan_of(a);
    const int S = (int)a->S, D = a->D, E = a->E, K = a->K, F = a->F, Fs = a->Fs, R = S * K;
    const bool i8 = a->weights == MOE_WEIGHTS_I8;
    const int wb = i8 ? 1 : 2, cols = i8 ? FewI8::kCols : FewBf16::kCols;
    char* ws = (char*)a->ws;
    float* part = (float*)(ws + p.part);
    int32_t* idx = a->topk_idx != nullptr ? a->topk_idx : (int32_t*)(ws + p.idx);
    float* prob = a->topk_prob != nullptr ? a->topk_prob : (float*)(ws + p.prob);
    int8_t *xq = (int8_t*)(ws + p.xq), *hq = (int8_t*)(ws + p.hq), *hqs = (int8_t*)(ws + p.hqs);
    float *xs = (float*)(ws + p.xs), *sc = (float*)(ws + p.sc), *scs = (float*)(ws + p.scs);
    uint16_t *h = (uint16_t*)(ws + p.h), *hs = (uint16_t*)(ws + p.hs);
    float *y = (float*)(ws + p.y), *ys = (float*)(ws + p.ys);

    hipLaunchKernelGGL(few_logits_kernel, dim3((unsigned)p.nd, (unsigned)cdiv(E, 64), (unsigned)cdiv(S, kFewT)),
                       dim3(kFewThreads), 0, st, a->x, a->Wr, S, D, E, part);
    const dim3 gr((unsigned)(i8 ? 2 * S : S));
    const bool sig = a->score_fn == MOE_SCORE_SIGMOID;
    if (E <= 64) launch_route_few<1>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else if (E <= 128) launch_route_few<2>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else if (E <= 256) launch_route_few<4>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else if (E <= 512) launch_route_few<8>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else launch_route_few<16>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);

    auto gemm = [&](FewSide r, FewSide s, int wk, bool up) {
        for (FewSide* q : {&r, &s}) {
            q->lda = q->Kd * wb;
            q->a_bytes *= q->lda;                       // given as rows
            q->w_bytes = (int64_t)q->Kd * q->N * wb;
            q->groups = cdiv(cdiv(q->N, cols), 4 / wk);
        }
        const FewGemmArgs g{r, s, idx, S, K, p.r_experts * r.groups, wk, up ? 1 : 0};
        const dim3 grid((unsigned)(g.r_items + (Fs ? s.groups : 0))), block(kFewThreads);
        if (S <= 16) {
            if (i8) hipLaunchKernelGGL((few_gemm_kernel<FewI8, 1>), grid, block, 0, st, g);
            else hipLaunchKernelGGL((few_gemm_kernel<FewBf16, 1>), grid, block, 0, st, g);
        } else {
            if (i8) hipLaunchKernelGGL((few_gemm_kernel<FewI8, 4>), grid, block, 0, st, g);
            else hipLaunchKernelGGL((few_gemm_kernel<FewBf16, 4>), grid, block, 0, st, g);
        }
    };
    // A, W, out, row and column scales, rows of A, (set above), lda, a_div, Kd, N, groups
    const void* x = i8 ? (const void*)xq : (const void*)a->x;
    gemm(FewSide{x, a->W1, h, xs, a->s1, S, 0, 0, K, D, F, 0}, FewSide{x, a->Ws1, hs, xs, a->ss1, S, 0, 0, 1, D, Fs, 0},
         p.wk1, true);
    const void *hr = h, *hsr = hs;
    if (i8) {
        const FewRows qr{h, hq, sc, F, R}, qs{hs, hqs, scs, Fs, Fs ? S : 0};
        hipLaunchKernelGGL(few_quant_kernel, dim3((unsigned)(qr.rows + qs.rows)), dim3(kFewThreads), 0, st, qr, qs);
        hr = hq;
        hsr = hqs;
    }
    gemm(FewSide{hr, a->W2, y, sc, a->s2, R, 0, 0, 1, F, D, 0}, FewSide{hsr, a->Ws2, ys, scs, a->ss2, S, 0, 0, 1, Fs, D, 0},
         p.wk2, false);
    hipLaunchKernelGGL(few_combine_kernel, dim3((unsigned)cdiv(D, 256), (unsigned)S), dim3(kFewThreads), 0, st, y,
                       Fs ? ys : nullptr, prob, K, D, a->y);
    return launch_check(st);
}

}  // namespace moe
