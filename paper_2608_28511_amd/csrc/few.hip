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
//   few_table    many picks: the picked experts' rows, else found by each workgroup below
//   few_gemm     up: h = max(x W1, 0)^2, rounded to bf16 with 8-bit weights (then to codes); with bf16
//                weights in two bf16 parts, within 2^-16, so that the only rounding to bf16 is y's: a
//                second matrix instruction a fragment in the down product, 0 to 4% of a call that
//                reads its weights (64 tokens of 64 experts 107 / 111 us, 8 of the production layer
//                286 / 290; 64 tokens on two experts of 2,048 x 4,096 58 / 73)
//   few_quant    8-bit weights: the rows of h
//   few_gemm     down: y_k = h W2 in fp32
//   few_combine  y = bf16(sum_k p_k y_k + shared), all sums in fp32 and fixed order
//
// us of a call, and the time of its weights at the 6.16 TB/s of a large read: 1 token top-6 of 64
// experts of 2,048 x 1,024 25-28 (8; launches 2.4 each), 64 tokens 106-112 (87), 8 tokens of the
// production layer 265-298 (310), in 8 bits 16 tokens top-8 of 256 of 2,048 x 2,688 164-179 (183), 3 tokens
// top-22 of 512 of 672 x 1,856 53-61 (26).
#include <algorithm>

#include "kernels.h"
#include "quant8.h"
#include "score.h"
#include "thin.h"

namespace moe {

constexpr int kFewThreads = kThinThreads;
constexpr int kSlabBf16 = ThinBf16<false>::kCols, kSlabI8 = ThinI8<2, false>::kCols;
static_assert(kFewMaxTokens <= kThinRows, "an expert's rows are at most the tokens");

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

// What the lanes of a wave wrote to LDS before is what they read after.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ uint32_t wave_max_code(uint32_t v) {
    v = row_max_u32(v);
    const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
    const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    return max(max(a, b), max(c, d));
}

// The K largest codes of a wave, in order, ties to the lower expert: pick k goes to lane k.
// Lane l holds experts l EPL .. + EPL - 1 and top, the largest of their codes.  The K-th
// largest of the lanes' tops bounds the K-th largest code from below, so only codes from
// there on can be picked (at least K of them, since at least K lanes hold an expert: EPL
// is the least power of two with 64 EPL >= E, and K <= 32).  They are gathered in LDS, one
// a lane, and each counts those before it: no chain of K rounds, which took half as long
// again (3 tokens, 512 experts top-22: 7.6 us the launch, the sums of the logits included).
template <int EPL>
__device__ __forceinline__ void few_pick(const uint32_t (&code)[EPL], uint32_t top, int K, uint32_t* codes, uint2* cand,
                                         int& my_e, uint32_t& my_c) {
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll 16
    for (int j = 0; j < 64; ++j) {
        const uint32_t o = __builtin_amdgcn_readlane(top, j);
        before += o > top || (o == top && j < lane) ? 1 : 0;
    }
    if constexpr (EPL == 1) {   // the lanes' ranks themselves
        if (before < K) cand[before] = make_uint2(top, (uint32_t)lane);
        wave_sync();
        if (lane < K) {
            const uint2 mine = cand[lane];
            my_c = mine.x;
            my_e = (int)mine.y;
        }
        return;
    }
    const uint32_t bound = __builtin_amdgcn_readlane(top, __builtin_ctzll(__ballot(before == K - 1)));
    int n = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        const bool in = code[i] >= bound && code[i] != 0u;
        const uint64_t m = __ballot(in);
        const int at = n + __popcll(m & ((1ull << lane) - 1ull));
        if (in && at < 64) cand[at] = make_uint2(code[i], (uint32_t)(lane * EPL + i));
        n += __popcll(m);
    }
    if (n > 64) {   // many equal scores: K rounds of the wave's maximum, its lowest holder, and clearing it
#pragma unroll
        for (int i = 0; i < EPL; ++i) codes[lane * EPL + i] = code[i];
        for (int k = 0; k < K; ++k) {   // K <= E: the maximum is never a cleared code
            uint32_t t = 0u;
            int at = 0;
            for (int i = EPL - 1; i >= 0; --i) {
                const uint32_t c = codes[lane * EPL + i];
                at = c >= t ? i : at;
                t = max(t, c);
            }
            const uint32_t m = wave_max_code(t);
            const int owner = __builtin_ctzll(__ballot(t == m));
            if (lane == owner) codes[lane * EPL + at] = 0u;
            const int e = __builtin_amdgcn_readlane(lane * EPL + at, owner);
            if (lane == k) {
                my_e = e;
                my_c = m;
            }
        }
        return;
    }
    // larger code first, then the lower expert
    wave_sync();
    const uint2 c = lane < n ? cand[lane] : make_uint2(0u, 1023u);
    int rank = 0;
    for (int j = 0; j < n; ++j) {
        const uint32_t oc = __builtin_amdgcn_readlane(c.x, j), oe = __builtin_amdgcn_readlane(c.y, j);
        rank += oc > c.x || (oc == c.x && oe < c.y) ? 1 : 0;
    }
    wave_sync();   // every lane has its candidate
    if (lane < n && rank < K) cand[rank] = c;
    wave_sync();
    if (lane < K) {
        const uint2 mine = cand[lane];
        my_c = mine.x;
        my_e = (int)mine.y;
    }
}

// Workgroup t < S: token t's logits, its K best experts (picked by its first wave) and
// their weights.  Workgroup S + t (8-bit weights): token t's codes.
constexpr int kRouteThreads = 1024;
template <int EPL, bool SIG>
__global__ __launch_bounds__(kRouteThreads) void few_route_kernel(
    const float* __restrict__ part, int nd, const float* __restrict__ bias, const float* __restrict__ sel_bias, int S,
    int E, int K, int32_t* __restrict__ topk_idx, float* __restrict__ topk_prob, const uint16_t* __restrict__ x, int D,
    int8_t* __restrict__ xq, float* __restrict__ xs) {
    __shared__ float lg[1024];
    __shared__ uint32_t tops[kRouteThreads / 64];
    __shared__ uint32_t codes[64 * EPL];
    __shared__ uint2 cand[64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if ((int)blockIdx.x >= S) {
        const int t = blockIdx.x - S;
        const uint4* src = (const uint4*)(x + (int64_t)t * D);
        uint32_t top = 0;
        for (int c = tid; c < D / 8; c += kRouteThreads) {
            const uint4 v = src[c];
            top = max_mag(max_mag(max_mag(max_mag(top, v.x), v.y), v.z), v.w);
        }
        top = wave_max_u32(top);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        for (int w = 0; w < kRouteThreads / 64; ++w) top = max(top, tops[w]);
        Quant8 s;
        s.init(top);
        if (tid == 0) xs[t] = s.scale;
        for (int c = tid; c < D / 8; c += kRouteThreads) {
            const uint4 v = src[c];
            ((uint2*)(xq + (int64_t)t * D))[c] = make_uint2(codes4(s, v.x, v.y), codes4(s, v.z, v.w));
        }
        return;
    }
    // 64 EPL experts side by side, the chunks of d dealt to the threads that are left
    const int t = blockIdx.x;
    constexpr int kSide = 64 * EPL, kParts = kRouteThreads / kSide;
    const int e = tid % kSide, p = tid / kSide;
    float a = 0.f;
    if (e < E) {
#pragma unroll 8
        for (int c = p; c < nd; c += kParts) a += part[((int64_t)c * S + t) * E + e];
    }
    lg[tid] = a;
    __syncthreads();
    if (p == 0 && e < E) {
        for (int q = 1; q < kParts; ++q) a += lg[q * kSide + e];
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
    few_pick<EPL>(code, top, K, codes, cand, my_e, my_c);
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
    int groups;          // workgroups an expert takes (0: there is no such expert)
};
struct FewGemmArgs {
    FewSide routed, shared;
    const int32_t* idx;   // [S, K]
    const int4* table;    // the picked experts {expert, first in rows, rows, 0}, from few_table; null: each workgroup
    const int32_t* rows;  // searches the picks itself
    int S, K, r_items;    // workgroups of the routed experts
    int wk;               // waves that share a slab's contraction; 4 / wk slabs side by side in a workgroup
    int epi;
};

// The a-th expert (ascending) among at most kFewSearch picks and its rows, in order, in rows[];
// returns the expert, or -1 if fewer are picked.  A single token's picks are distinct and
// need no order.  Every thread of the workgroup calls it.
constexpr int kFewSearch = 256;   // most picks that a workgroup searches
struct FewPicks {
    uint32_t seen[32];
    int32_t picks[kFewSearch], rows[kFewMaxTokens], nrows;
};
__device__ __forceinline__ int few_plan(const int32_t* __restrict__ idx, int S, int K, int a, FewPicks& sh) {
    const int tid = threadIdx.x, lane = tid & 63, n = S * K;
    if (S == 1) {
        if (tid == 0) {
            sh.rows[0] = a;
            sh.nrows = 1;
        }
        return a < K ? __builtin_amdgcn_readfirstlane(idx[a]) & 1023 : -1;
    }
    if (tid < 32) sh.seen[tid] = 0u;
    __syncthreads();
    for (int q = tid; q < n; q += kFewThreads) {
        const int e = idx[q] & 1023;   // E <= 1024
        sh.picks[q] = e;
        atomicOr(&sh.seen[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    const uint32_t word = lane < 32 ? sh.seen[lane] : 0u;
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
            const bool hit = q0 + lane < n && sh.picks[q0 + lane] == e;
            const uint64_t m = __ballot(hit);
            const int pos = at + __popcll(m & ((1ull << lane) - 1ull));
            if (hit && pos < kFewMaxTokens) sh.rows[pos] = q0 + lane;   // a token picks an expert once
            at += __popcll(m);
        }
        if (lane == 0) sh.nrows = at < kFewMaxTokens ? at : kFewMaxTokens;
    }
    return e;
}

// The picked experts, ascending, and their rows, by one workgroup: entries of table past
// them hold no rows.  An expert's rows come in any order: a row's result depends on the
// row alone.
constexpr int kTableThreads = 1024;
__global__ __launch_bounds__(kTableThreads) void few_table_kernel(const int32_t* __restrict__ idx, int n, int entries,
                                                                  int4* __restrict__ table, int32_t* __restrict__ rows) {
    __shared__ int32_t count[kMaxExperts], first[kMaxExperts];
    __shared__ int2 wsum[kTableThreads / 64];
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    count[e] = 0;
    __syncthreads();
    int pick[2], rank[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {   // n <= 64 x 32
        const int q = e + u * kTableThreads;
        if (q < n) {
            pick[u] = idx[q] & (kMaxExperts - 1);
            rank[u] = atomicAdd(&count[pick[u]], 1);
        }
    }
    __syncthreads();
    const int c = min(count[e], kFewMaxTokens);   // a token picks an expert once
    int2 incl = make_int2(c, c > 0 ? 1 : 0);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int ox = __shfl_up(incl.x, d), oy = __shfl_up(incl.y, d);
        if (lane >= d) {
            incl.x += ox;
            incl.y += oy;
        }
    }
    if (lane == 63) wsum[wave] = incl;
    __syncthreads();
    int2 base = make_int2(0, 0);
    int active = 0;
    for (int w = 0; w < kTableThreads / 64; ++w) {
        if (w < wave) {
            base.x += wsum[w].x;
            base.y += wsum[w].y;
        }
        active += wsum[w].y;
    }
    const int f = base.x + incl.x - c;
    first[e] = f;
    if (c > 0) table[base.y + incl.y - 1] = make_int4(e, f, c, 0);
    if (e >= active && e < entries) table[e] = make_int4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int q = e + u * kTableThreads;
        if (q < n && rank[u] < kFewMaxTokens) rows[first[pick[u]] + rank[u]] = q;
    }
}

// At most 16 MBMAX tokens, and so rows an expert.  The fewer, the more waves a SIMD has registers for: 32
// tokens of 8-bit weights top-16 of 256 experts of 1,024 x 1,536 122 us at four, 143 at the two that 64 leave,
// top-6 of 64 of 2,048 x 1,024 71.0 / 77.2.
constexpr int few_waves(int mb_max, int wave_lds) { return mb_max == 4 ? 2 : wave_lds * mb_max <= 8192 ? 4 : 3; }
template <class T, int MBMAX>
__global__ __launch_bounds__(kFewThreads, few_waves(MBMAX, T::kWaveLds)) void few_gemm_kernel(FewGemmArgs p) {
    __shared__ FewPicks sh;
    __shared__ __attribute__((aligned(16))) char lds[4 * T::kWaveLds];
    const bool shared = (int)blockIdx.x >= p.r_items;
    const int b = (int)blockIdx.x - (shared ? p.r_items : 0);
    const FewSide s = shared ? p.shared : p.routed;
    const int a = b / s.groups, in = b - a * s.groups;
    int e = 0, nrows = p.S;
    const int32_t* rows = nullptr;   // the shared expert's are the tokens
    if (!shared && p.table != nullptr) {
        const int4 t = p.table[a];
        e = __builtin_amdgcn_readfirstlane(t.x);
        nrows = __builtin_amdgcn_readfirstlane(t.z);
        if (nrows == 0) return;
        rows = p.rows + __builtin_amdgcn_readfirstlane(t.y);
    } else if (!shared) {
        e = few_plan(p.idx, p.S, p.K, a, sh);
        if (e < 0) return;
        __syncthreads();
        nrows = __builtin_amdgcn_readfirstlane(sh.nrows);
        rows = sh.rows;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = p.wk;
    const int kk = wave & (wk - 1), n0 = (in * (4 / wk) + wave / wk) * T::kCols;
    const ThinArgs t{s.A, (const char*)s.W + e * s.w_bytes, s.out, s.row_scale, s.col_scale + (int64_t)e * s.N,
                     s.a_bytes, s.w_bytes, s.lda, s.Kd, s.N, p.epi};
    thin_rows<T, MBMAX>(t, n0, kk, wk, nrows, [&](int r) { return r / s.a_div; },
                        [&](int i) { return rows != nullptr ? rows[i] : i; }, lds);
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

// The only launch that writes y, and no later one reads x: callers may let them overlap.
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
    *(u32x2_thin*)(y + (int64_t)t * D + d) = u32x2_thin{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// ---- host -------------------------------------------------------------------
namespace {

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

int cdiv(int a, int b) { return (a + b - 1) / b; }

struct FewPlan {
    int nd, r_experts;
    int wk1, wk2;          // waves that share a slab of the up and of the down product
    bool table;
    size_t part, idx, prob, tab, rows, xq, xs, h, hs, hq, hqs, sc, scs, y, ys, bytes;   // offsets
};

// Waves of a workgroup's four that share a slab's contraction, each keeping a step.  Four
// give the most workgroups, which the CUs then share evenly, two the fewer that have to find
// their rows and join their sums: two where they still make two workgroups a CU of more than
// 16 tokens (us with 2 / 4: 64 tokens top-6 of 64 experts of 2,048 x 1,024 112 / 123 and in 8 bits
// 79.8 / 85.3, top-22 of 512 of 672 x 1,856 416 / 440 and 255 / 276, but top-2 of 8 of 2,048 x 1,024
// 47.2 / 37.2 and 35.0 / 32.4), and with up to 16 tokens and bf16 weights eight a CU (16 tokens
// top-8 of 256 of 2,048 x 2,688 316 / 325; 8 tokens of the 192-expert layer 293 / 291; 1 token of 64
// 34.2 / 27.2, 16 of them 89.1 / 91.4; in 8 bits 16 tokens top-8 of 256 170 / 166, 8 of 192 175 / 168).
int few_share(bool i8, bool many, int slabs, int steps) {
    const int groups = many ? 2 : i8 ? 1 << 20 : 8;   // a CU's
    int wk = slabs / 2 >= (int64_t)groups * cu_count() ? 2 : 4;
    while (wk > steps) wk /= 2;
    return wk;
}

// Whether a launch of its own (2.5 us) finds the picked experts' rows, instead of every
// workgroup of both products.  64 tokens top-22 of 512 of 672 x 1,856 416 us against 452 and, in 8
// bits, 255 against 339; 40 tokens top-22 of 64 of them 101 / 108 and 71.7 / 78.6; 64 tokens top-6 of 64
// of 2,048 x 1,024 (384 picks) 112 / 112 and 80.2 / 85.4; 16 tokens top-8 of 256 (128 picks) 318 / 316 and
// 167 / 166; 1 token of 64 30.2 / 27.1.
bool few_table_pays(int picks) { return picks > kFewSearch; }

// Columns of a slab.  8-bit weights take 32, or, where more than 16 tokens give an expert
// twelve rows or more on average, 64, which halves how often the rows are read, if that still
// makes a workgroup a CU.  Of 53 calls of 17 to 64 tokens (4 to 512 experts, 512 to 2,816 by 512 to
// 3,456) the 7 that take 64 take 0.91 to 1.02 of their time with 32, and of the others 36 of
// 46 would lose up to a fifth (us with 32 / 64: 54 tokens top-10 of 22 of 2,560 x 1,408 81.3 /
// 74.3, 30 top-22 of 39 of 2,176 x 2,688 115.5 / 110.4, 40 top-22 of 64 of 672 x 1,856 70.2 /
// 71.7; 64 top-6 of 48 of 2,048 x 1,024 65.5 / 73.9, 33 top-4 of 4 of 1,664 x 1,920 34.5 / 40.8,
// 64 top-22 of 512 of 672 x 1,856 254 / 267).
int few_cols(const moe_layer_few_args* a) {
    if (a->weights != MOE_WEIGHTS_I8) return kSlabBf16;
    const int64_t slabs = (int64_t)a->E * cdiv(std::min(a->D, a->F), 2 * kSlabI8);   // all experts have rows
    return a->S > 16 && a->S * a->K >= 12 * (int64_t)a->E && slabs >= cu_count() ? 2 * kSlabI8 : kSlabI8;
}

FewPlan few_plan_of(const moe_layer_few_args* a) {
    FewPlan p{};
    const int S = (int)a->S, D = a->D, E = a->E, K = a->K, F = a->F, Fs = a->Fs;
    const bool i8 = a->weights == MOE_WEIGHTS_I8;
    const size_t R = (size_t)S * K;
    const int step = i8 ? ThinI8<2, false>::kStep : ThinBf16<false>::kStep;
    p.nd = cdiv(D, kFewD);
    p.r_experts = (int)std::min<size_t>((size_t)E, R);
    const int cols = few_cols(a), ns = Fs ? 1 : 0;
    p.wk1 = few_share(i8, S > 16, p.r_experts * cdiv(F, cols) + ns * cdiv(Fs, cols), cdiv(D, step));
    p.wk2 = few_share(i8, S > 16, (p.r_experts + ns) * cdiv(D, cols), cdiv(F, step));
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += up256(bytes);
        return o;
    };
    p.part = take((size_t)p.nd * S * E * 4);
    p.idx = take(R * 4);
    p.prob = take(R * 4);
    p.table = few_table_pays((int)R);
    p.tab = take(p.table ? (size_t)p.r_experts * 16 : 0);
    p.rows = take(p.table ? R * 4 : 0);
    p.xq = take(i8 ? (size_t)S * D : 0);
    p.xs = take((size_t)S * 4);
    p.h = take(R * F * (i8 ? 2 : 4));   // bf16 weights: two parts
    p.hs = take((size_t)S * Fs * (i8 ? 2 : 4));
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
hipError_t launch_route_few(bool sig, dim3 g, hipStream_t st, const float* part, int nd, const moe_layer_few_args* a,
                      int32_t* idx, float* prob, int8_t* xq, float* xs) {
    if (sig)
        hipLaunchKernelGGL((few_route_kernel<EPL, true>), g, dim3(kRouteThreads), 0, st, part, nd, a->router_bias,
                           a->sel_bias, (int)a->S, a->E, a->K, idx, prob, a->x, a->D, xq, xs);
    else
        hipLaunchKernelGGL((few_route_kernel<EPL, false>), g, dim3(kRouteThreads), 0, st, part, nd, a->router_bias,
                           a->sel_bias, (int)a->S, a->E, a->K, idx, prob, a->x, a->D, xq, xs);
    return launch_check(st);
}

#define FEW_TRY(expr)                    \
    do {                                 \
        const hipError_t e_ = (expr);    \
        if (e_ != hipSuccess) return e_; \
    } while (0)

}  // namespace

size_t layer_few_ws_bytes(const moe_layer_few_args* a) { return few_plan_of(a).bytes; }

hipError_t launch_layer_few(const moe_layer_few_args* a, hipStream_t st) {
    const FewPlan p = few_plan_of(a);
    const int S = (int)a->S, D = a->D, E = a->E, K = a->K, F = a->F, Fs = a->Fs, R = S * K;
    const bool i8 = a->weights == MOE_WEIGHTS_I8;
    const int wb = i8 ? 1 : 2, cols = few_cols(a);
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
    FEW_TRY(launch_check(st));
    const dim3 gr((unsigned)(i8 ? 2 * S : S));
    const bool sig = a->score_fn == MOE_SCORE_SIGMOID;
    auto route = [&](auto epl) {
        return launch_route_few<decltype(epl)::value>(sig, gr, st, part, p.nd, a, idx, prob, xq, xs);
    };
    FEW_TRY(E <= 64    ? route(std::integral_constant<int, 1>{})
            : E <= 128 ? route(std::integral_constant<int, 2>{})
            : E <= 256 ? route(std::integral_constant<int, 4>{})
            : E <= 512 ? route(std::integral_constant<int, 8>{})
                       : route(std::integral_constant<int, 16>{}));

    const int4* table = p.table ? (const int4*)(ws + p.tab) : nullptr;
    if (p.table) {
        hipLaunchKernelGGL(few_table_kernel, dim3(1), dim3(kTableThreads), 0, st, idx, R, p.r_experts,
                           (int4*)(ws + p.tab), (int32_t*)(ws + p.rows));
        FEW_TRY(launch_check(st));
    }
    // parts: of the values of A, where weights are bf16
    auto gemm = [&](auto parts, FewSide r, FewSide s, int wk, int epi) {
        constexpr int PARTS = decltype(parts)::value;
        for (FewSide* q : {&r, &s}) {
            q->lda = q->Kd * (i8 ? 1 : 2 * PARTS);
            q->a_bytes *= q->lda;                       // given as rows
            q->w_bytes = (int64_t)q->Kd * q->N * wb;
            q->groups = cdiv(cdiv(q->N, cols), 4 / wk);
        }
        if (Fs == 0) s.groups = 0;
        const FewGemmArgs g{r, s, idx, table, (const int32_t*)(ws + p.rows), S, K, p.r_experts * r.groups, wk, epi};
        const dim3 grid((unsigned)(g.r_items + s.groups)), block(kFewThreads);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, g); };
        auto pick = [&](auto nt) {
            constexpr bool NT = decltype(nt)::value;
            if (S <= 16) i8 ? go(few_gemm_kernel<ThinI8<2, NT>, 1>) : go(few_gemm_kernel<ThinBf16<NT, PARTS>, 1>);
            else if (!i8) go(few_gemm_kernel<ThinBf16<NT, PARTS>, 4>);
            else if (S <= 32)
                cols == kSlabI8 ? go(few_gemm_kernel<ThinI8<2, NT>, 2>) : go(few_gemm_kernel<ThinI8<4, NT>, 2>);
            else cols == kSlabI8 ? go(few_gemm_kernel<ThinI8<2, NT>, 4>) : go(few_gemm_kernel<ThinI8<4, NT>, 4>);
        };
        // the routed experts' weights decide for the shared one's, a small part of the call
        if (thin_nt(r.W, (int64_t)(i8 ? r.Kd : r.N) * wb, 2 * (int64_t)p.r_experts * r.w_bytes)) pick(std::true_type{});
        else pick(std::false_type{});
        return launch_check(st);
    };
    // A, W, out, row and column scales, rows of A, .., .., a_div, Kd, N (the rest is set above)
    const void* x = i8 ? (const void*)xq : (const void*)a->x;
    FEW_TRY(gemm(std::integral_constant<int, 1>{}, FewSide{x, a->W1, h, xs, a->s1, S, 0, 0, K, D, F, 0},
                 FewSide{x, a->Ws1, hs, xs, a->ss1, S, 0, 0, 1, D, Fs, 0}, p.wk1, THIN_RELU2));
    const void *hr = h, *hsr = hs;
    if (i8) {
        const FewRows qr{h, hq, sc, F, R}, qs{hs, hqs, scs, Fs, Fs ? S : 0};
        hipLaunchKernelGGL(few_quant_kernel, dim3((unsigned)(qr.rows + qs.rows)), dim3(kFewThreads), 0, st, qr, qs);
        FEW_TRY(launch_check(st));
        hr = hq;
        hsr = hqs;
    }
    FEW_TRY(gemm(std::integral_constant<int, 2>{}, FewSide{hr, a->W2, y, sc, a->s2, R, 0, 0, 1, F, D, 0},
                 FewSide{hsr, a->Ws2, ys, scs, a->ss2, S, 0, 0, 1, Fs, D, 0}, p.wk2, THIN_F32));
    hipLaunchKernelGGL(few_combine_kernel, dim3((unsigned)cdiv(D, 256), (unsigned)S), dim3(kFewThreads), 0, st, y,
                       Fs ? ys : nullptr, prob, K, D, a->y);
    return launch_check(st);
}

}  // namespace moe
