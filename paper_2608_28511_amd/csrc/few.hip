// A whole layer for at most 64 tokens (a decode step, a few drafted tokens).
//
// Such a call reads the picked experts' weights once and does little else, so what
// bounds it is HBM and, below some tens of megabytes, the latency of each launch.  No
// permutation is built: routed row r = t K + k keeps its place, and a workgroup of a
// product finds its expert and that expert's rows in the S K picks itself.
//
//   few_logits   partial router logits: 64 d x 64 experts a workgroup, fp32 products
//   few_route    one workgroup a token: the partial sums, top-K and weights; with 8-bit
//                weights as many again quantise the token rows
//   few_gemm     up: partial u = x W1 over a share of the contraction
//   few_act      h = bf16(max(u, 0)^2) (8-bit weights: and its rows' codes)
//   few_gemm     down: partial y = h W2
//   few_combine  y = bf16(sum_k p_k y_k + shared), all sums in fp32 and fixed order
//
// few_gemm's matrix products take 16 tokens; weights go from memory to the matrix
// cores' operands in registers, each wave a share of the contraction, several
// steps ahead, and never through LDS: every weight is used by one wave only.
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
constexpr int kFewD = 64;
__global__ __launch_bounds__(kFewThreads) void few_logits_kernel(const uint16_t* __restrict__ x,
                                                                 const float* __restrict__ Wr, int S, int D, int E,
                                                                 float* __restrict__ part) {
    __shared__ float xs[kFewMaxTokens][kFewD];
    __shared__ float red[4][kFewMaxTokens][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int d0 = blockIdx.x * kFewD, e = blockIdx.y * 64 + lane;
    float w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int d = d0 + wave * 16 + i;
        w[i] = d < D && e < E ? Wr[(int64_t)d * E + e] : 0.f;
    }
    for (int c = threadIdx.x; c < S * (kFewD / 8); c += kFewThreads) {
        const int t = c / (kFewD / 8), d = (c % (kFewD / 8)) * 8;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (d0 + d < D) v = *(const uint4*)(x + (int64_t)t * D + d0 + d);   // D is a multiple of 8
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            xs[t][d + 2 * q] = bf16_lo(u[q]);
            xs[t][d + 2 * q + 1] = bf16_hi(u[q]);
        }
    }
    __syncthreads();
    for (int t = 0; t < S; ++t) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) a = fmaf(xs[t][wave * 16 + i], w[i], a);
        red[wave][t][lane] = a;
    }
    __syncthreads();
    if (e >= E) return;
    for (int t = wave; t < S; t += 4)
        part[((int64_t)blockIdx.x * S + t) * E + e] =
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
    uint32_t* out;       // [splits][rows][N] fp32 or int32
    int64_t a_bytes, w_bytes;   // of A, of one expert's W
    int lda, a_div;
    int Kd, N, rows;
    int slabs, splits;   // output columns and contraction in this many workgroups
};
struct FewGemmArgs {
    FewSide routed, shared;
    const int32_t* idx;   // [S, K]
    int S, K, r_items;    // workgroups of the routed experts
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

// bf16 weights, N-contiguous: a workgroup's 64 columns, a wave's every fourth step of
// 32 k.  A lane loads 4 columns of 8 k rows (each load of the wave four whole cache
// lines) and packs them into the fragments of columns 4 c + q, q = 0 .. 3, with one byte
// permutation a register.
struct FewBf16 {
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
    // acc[q][v] of a lane is column 16 g + 4 v + q of its token: four stores of four columns
    template <class T>
    __device__ __forceinline__ static void leave(const f32x4 (&acc)[kAcc], T&& put, int lane) {
#pragma unroll
        for (int v = 0; v < 4; ++v)
            put(16 * (lane >> 4) + 4 * v, f32x4{acc[0][v], acc[1][v], acc[2][v], acc[3][v]});
    }
};

// 8-bit weights, K-contiguous: a workgroup's 32 columns, a wave's every fourth step of
// 128 k, whose fragments are 16 bytes of a channel as they lie in memory.
struct FewI8 {
    static constexpr int kCols = 32, kStep = 128, kAcc = 2;
    template <int MB>
    static constexpr int kAhead = MB == 4 ? 2 : 4;
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
    template <class T>
    __device__ __forceinline__ static void leave(const f32x4 (&acc)[kAcc], T&& put, int lane) {
#pragma unroll
        for (int b = 0; b < 2; ++b) put(16 * b + 4 * (lane >> 4), acc[b]);
    }
};

// The workgroup's partial product for 16 MB rows: steps [st0, st1), the waves' sums
// joined in LDS in wave order.
template <class T, int MB>
__device__ __forceinline__ void few_body(const FewSide& s, int e, int n0, int split, const int32_t* rows, int nrows,
                                         uint32_t (*red)[16][T::kCols + 4]) {
    constexpr bool I8 = std::is_same<T, FewI8>::value;
    constexpr int P = T::template kAhead<MB>;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nst = (s.Kd + T::kStep - 1) / T::kStep;
    const int st0 = (int)((int64_t)nst * split / s.splits), st1 = (int)((int64_t)nst * (split + 1) / s.splits);
    const int mine = st1 - st0 > wave ? (st1 - st0 - wave + 3) / 4 : 0;
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
        const int k = (st0 + wave + 4 * i) * T::kStep;
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
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        if (m > 0) __syncthreads();
        T::leave(acc[m], [&](int col, f32x4 v) { *(f32x4*)&red[wave][lane & 15][col] = v; }, lane);
        __syncthreads();
        for (int c = tid; c < 16 * (T::kCols / 4); c += kFewThreads) {
            const int i = c / (T::kCols / 4), col = (c % (T::kCols / 4)) * 4;
            if (m * 16 + i >= nrows || n0 + col >= s.N) continue;   // N is a multiple of 8
            u32x4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *(const u32x4*)&red[u][i][col];
            u32x4 t;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (I8)
                    t[q] = (v[0][q] + v[1][q]) + (v[2][q] + v[3][q]);
                else
                    t[q] = __float_as_uint((__uint_as_float(v[0][q]) + __uint_as_float(v[1][q])) +
                                           (__uint_as_float(v[2][q]) + __uint_as_float(v[3][q])));
            }
            *(u32x4*)(s.out + ((int64_t)split * s.rows + rows[m * 16 + i]) * s.N + n0 + col) = t;
        }
    }
}

template <class T>
__global__ __launch_bounds__(kFewThreads, 2) void few_gemm_kernel(FewGemmArgs p) {
    __shared__ uint32_t seen[32];
    __shared__ int32_t picks[kFewMaxTokens * 32], rows[kFewMaxTokens], nrows_s;
    __shared__ __attribute__((aligned(16))) uint32_t red[4][16][T::kCols + 4];
    const bool shared = (int)blockIdx.x >= p.r_items;
    const int b = (int)blockIdx.x - (shared ? p.r_items : 0);
    const FewSide s = shared ? p.shared : p.routed;
    const int a = b / (s.slabs * s.splits), in = b - a * (s.slabs * s.splits);
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
    const int split = in / s.slabs, n0 = (in - split * s.slabs) * T::kCols;
    if (nrows <= 16) few_body<T, 1>(s, e, n0, split, rows, nrows, red);
    else if (nrows <= 32) few_body<T, 2>(s, e, n0, split, rows, nrows, red);
    else few_body<T, 4>(s, e, n0, split, rows, nrows, red);
}

// ---- between the products and after them ------------------------------------
struct FewAct {
    const uint32_t* u;       // [splits][rows][F]
    void* h;                 // [rows][F] bf16 or int8
    float* hs;               // [rows] scales (8-bit)
    const float* scale;      // [experts][F] channel scales (8-bit)
    int F, rows, splits;
};

// Four elements of the row's activation from the partial sums.
template <bool I8>
__device__ __forceinline__ void few_act4(const FewAct& p, int row, int f, float xs, const float* cs, uint32_t& h01,
                                         uint32_t& h23) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    int n[4] = {0, 0, 0, 0};
    for (int s = 0; s < p.splits; ++s) {
        const u32x4 w = *(const u32x4*)(p.u + ((int64_t)s * p.rows + row) * p.F + f);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (I8) n[q] += (int)w[q];
            else v[q] += __uint_as_float(w[q]);
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (I8) v[q] = (float)n[q] * xs * cs[f + q];
        v[q] = relu_f32(v[q]);
        v[q] *= v[q];
    }
    h01 = pack_bf16x2(v[0], v[1]);
    h23 = pack_bf16x2(v[2], v[3]);
}

// One workgroup a row: routed rows first, then the shared expert's.
template <bool I8>
__global__ __launch_bounds__(kFewThreads) void few_act_kernel(FewAct routed, FewAct shared,
                                                              const int32_t* __restrict__ idx,
                                                              const float* __restrict__ xs, int K) {
    __shared__ uint32_t tops[4];
    const bool sh = (int)blockIdx.x >= routed.rows;
    const FewAct p = sh ? shared : routed;
    const int row = (int)blockIdx.x - (sh ? routed.rows : 0);
    const int tid = threadIdx.x;
    float x = 1.f;
    const float* cs = nullptr;
    if constexpr (I8) {
        x = xs[sh ? row : row / K];
        cs = p.scale + (sh ? 0 : (int64_t)idx[row] * p.F);
    }
    uint32_t top = 0;
    for (int f = tid * 4; f < p.F; f += kFewThreads * 4) {
        uint32_t a, b;
        few_act4<I8>(p, row, f, x, cs, a, b);
        if constexpr (I8) top = max_mag(max_mag(top, a), b);
        else *(uint2*)((uint16_t*)p.h + (int64_t)row * p.F + f) = make_uint2(a, b);
    }
    if constexpr (I8) {
        top = wave_max_u32(top);
        if ((tid & 63) == 0) tops[tid >> 6] = top;
        __syncthreads();
        Quant8 s;
        s.init(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
        if (tid == 0) p.hs[row] = s.scale;
        for (int f = tid * 4; f < p.F; f += kFewThreads * 4) {
            uint32_t a, b;
            few_act4<I8>(p, row, f, x, cs, a, b);
            *(uint32_t*)((int8_t*)p.h + (int64_t)row * p.F + f) = codes4(s, a, b);
        }
    }
}

struct FewOut {
    const uint32_t* y;     // [splits][rows][D] partial products
    const float* hs;       // [rows] (8-bit)
    const float* scale;    // [experts][D] (8-bit)
    int rows, splits;
};

template <bool I8>
__device__ __forceinline__ void few_out4(const FewOut& p, int row, int64_t e, int D, int d, float w, float (&y)[4]) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    int n[4] = {0, 0, 0, 0};
    for (int s = 0; s < p.splits; ++s) {
        const u32x4 q4 = *(const u32x4*)(p.y + ((int64_t)s * p.rows + row) * D + d);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (I8) n[q] += (int)q4[q];
            else v[q] += __uint_as_float(q4[q]);
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (I8) v[q] = (float)n[q] * p.hs[row] * p.scale[e * D + d + q];
        y[q] = fmaf(w, v[q], y[q]);
    }
}

template <bool I8>
__global__ __launch_bounds__(64) void few_combine_kernel(FewOut routed, FewOut shared, const int32_t* __restrict__ idx,
                                                         const float* __restrict__ prob, int K, int D,
                                                         uint16_t* __restrict__ y) {
    const int t = blockIdx.y, d = (blockIdx.x * 64 + threadIdx.x) * 4;
    if (d >= D) return;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < K; ++k)
        few_out4<I8>(routed, t * K + k, I8 ? idx[t * K + k] : 0, D, d, prob[t * K + k], v);
    if (shared.rows > 0) few_out4<I8>(shared, t, 0, D, d, 1.f, v);
    *(uint2*)(y + (int64_t)t * D + d) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// ---- host -------------------------------------------------------------------
namespace {

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

struct FewPlan {
    int nd, r_experts;
    int cols, step;
    int slabs1, slabs2, slabs1s;           // 64- or 32-column slabs of F, D, Fs
    int split1, split2, split2s;           // shares of D (both up products), F, Fs
    size_t part, idx, prob, xq, xs, u, us, h, hs, hsc, hssc, y, ys, bytes;   // offsets
};

int cdiv(int a, int b) { return (a + b - 1) / b; }

// Shares of a contraction of `steps` steps: enough workgroups for two a compute unit,
// while every wave keeps two steps.
int few_splits(int items, int steps) {
    const int want = cdiv(2 * cu_count(), items > 0 ? items : 1);
    const int most = std::max(1, steps / 8);
    return std::max(1, std::min(want, most));
}

FewPlan few_plan_of(const moe_layer_few_args* a) {
    FewPlan p{};
    const int S = (int)a->S, D = a->D, E = a->E, K = a->K, F = a->F, Fs = a->Fs;
    const bool i8 = a->weights == MOE_WEIGHTS_I8;
    const size_t R = (size_t)S * K;
    p.nd = cdiv(D, kFewD);
    p.r_experts = (int)std::min<size_t>((size_t)E, R);
    p.cols = i8 ? FewI8::kCols : FewBf16::kCols;
    p.step = i8 ? FewI8::kStep : FewBf16::kStep;
    p.slabs1 = cdiv(F, p.cols);
    p.slabs2 = cdiv(D, p.cols);
    p.slabs1s = cdiv(Fs, p.cols);
    p.split1 = few_splits(p.r_experts * p.slabs1 + p.slabs1s, cdiv(D, p.step));
    const int items2 = (p.r_experts + (Fs ? 1 : 0)) * p.slabs2;
    p.split2 = few_splits(items2, cdiv(F, p.step));
    p.split2s = Fs ? few_splits(items2, cdiv(Fs, p.step)) : 1;
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
    p.u = take((size_t)p.split1 * R * F * 4);
    p.us = take((size_t)p.split1 * S * Fs * 4);
    p.h = take(R * F * (i8 ? 1 : 2));
    p.hs = take((size_t)S * Fs * (i8 ? 1 : 2));
    p.hsc = take(R * 4);
    p.hssc = take((size_t)S * 4);
    p.y = take((size_t)p.split2 * R * D * 4);
    p.ys = take(Fs ? (size_t)p.split2s * S * D * 4 : 0);
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
    const int wb = i8 ? 1 : 2;
    char* ws = (char*)a->ws;
    float* part = (float*)(ws + p.part);
    int32_t* idx = a->topk_idx != nullptr ? a->topk_idx : (int32_t*)(ws + p.idx);
    float* prob = a->topk_prob != nullptr ? a->topk_prob : (float*)(ws + p.prob);
    int8_t* xq = (int8_t*)(ws + p.xq);
    float *xs = (float*)(ws + p.xs), *hsc = (float*)(ws + p.hsc), *hssc = (float*)(ws + p.hssc);
    uint32_t *u = (uint32_t*)(ws + p.u), *us = (uint32_t*)(ws + p.us);
    uint32_t *y = (uint32_t*)(ws + p.y), *ys = (uint32_t*)(ws + p.ys);
    void *h = ws + p.h, *hs = ws + p.hs;

    hipLaunchKernelGGL(few_logits_kernel, dim3((unsigned)p.nd, (unsigned)cdiv(E, 64)), dim3(kFewThreads), 0, st, a->x,
                       a->Wr, S, D, E, part);
    const dim3 gr((unsigned)(i8 ? 2 * S : S));
    const bool sig = a->score_fn == MOE_SCORE_SIGMOID;
    if (E <= 64) launch_route_few<1>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else if (E <= 128) launch_route_few<2>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else if (E <= 256) launch_route_few<4>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else if (E <= 512) launch_route_few<8>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    else launch_route_few<16>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);

    auto side = [&](const void* A, int64_t a_rows, int a_div, const void* W, int Kd, int N, int rows, int slabs,
                    int splits, uint32_t* out) {
        FewSide s{};
        s.A = A; s.W = W; s.out = out;
        s.lda = Kd * wb;
        s.a_bytes = a_rows * s.lda;
        s.w_bytes = (int64_t)Kd * N * wb;
        s.a_div = a_div; s.Kd = Kd; s.N = N; s.rows = rows; s.slabs = slabs; s.splits = splits;
        return s;
    };
    auto gemm = [&](const FewSide& r, const FewSide& s) {
        FewGemmArgs g{r, s, idx, S, K, p.r_experts * r.slabs * r.splits};
        const dim3 grid((unsigned)(g.r_items + s.slabs * s.splits));
        if (i8) hipLaunchKernelGGL(few_gemm_kernel<FewI8>, grid, dim3(kFewThreads), 0, st, g);
        else hipLaunchKernelGGL(few_gemm_kernel<FewBf16>, grid, dim3(kFewThreads), 0, st, g);
    };
    const void* x = i8 ? (const void*)xq : (const void*)a->x;
    gemm(side(x, S, K, a->W1, D, F, R, p.slabs1, p.split1, u),
         side(x, S, 1, a->Ws1, D, Fs, S, p.slabs1s, p.split1, us));
    const FewAct ar{u, h, hsc, a->s1, F, R, p.split1}, as{us, hs, hssc, a->ss1, Fs, Fs ? S : 0, p.split1};
    const dim3 ga((unsigned)(ar.rows + as.rows));
    if (i8) hipLaunchKernelGGL(few_act_kernel<true>, ga, dim3(kFewThreads), 0, st, ar, as, idx, xs, K);
    else hipLaunchKernelGGL(few_act_kernel<false>, ga, dim3(kFewThreads), 0, st, ar, as, idx, xs, K);
    gemm(side(h, R, 1, a->W2, F, D, R, p.slabs2, p.split2, y),
         side(hs, S, 1, a->Ws2, Fs, D, S, Fs ? p.slabs2 : 0, p.split2s, ys));
    const FewOut orr{y, hsc, a->s2, R, p.split2}, os{ys, hssc, a->ss2, Fs ? S : 0, p.split2s};
    const dim3 gc((unsigned)cdiv(D, 256), (unsigned)S);
    if (i8) hipLaunchKernelGGL(few_combine_kernel<true>, gc, dim3(64), 0, st, orr, os, idx, prob, K, D, a->y);
    else hipLaunchKernelGGL(few_combine_kernel<false>, gc, dim3(64), 0, st, orr, os, idx, prob, K, D, a->y);
    return launch_check(st);
}

}  // namespace moe
