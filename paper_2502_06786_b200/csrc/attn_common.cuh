// What the kernels of matq_attn_paged share: parameters, page lookup, the score function, the join of key splits.
#pragma once

#include "tc.cuh"

namespace matq {
namespace attn {

constexpr float kLog2e = 1.4426950408889634f;
// The running maximum of a row is only a reference for the exponents: weights, sums and outputs are floating-point numbers whose relative precision does
// not depend on it.  It moves when a score lies more than kFar (in exponents of two) above it: weights stay below 2^32, sums over 2^31 keys below 2^63, and
// what is flushed to zero below 2^-126 is nothing beside a largest weight of 2^-32 or more.  (With 8 in place of 32 rows of a long prompt moved theirs now and
// then, and a step done again for one row costs its whole warp: 8192 tokens over 8192 at 32/8 x 128 heads took 1.98 ms.)
constexpr float kFar = 32.f;

// The weights 2^x are rounded to bf16 for the product with v, as v and the outputs are: that is what the tensor cores take beside bf16 values, and half the
// registers and tensor memory of fp32.  Each is off by 2^-8 of itself at most, so an output by 2^-8 of sum_j p_j |v_j|; their sum is taken before the rounding.
// Against 64 bits the outputs of 64 ragged tokens (500 over 6511) are off by 2.1e-3 (2.3e-3) of their norm, of which rounding the outputs is 1.7e-3.

struct Params {
    const __nv_bfloat16 *q, *v;
    __nv_bfloat16* out;
    const int32_t *table, *cu_q, *kv_len;
    int64_t ldq, ldo, table_stride, table_width, n_pages, T;
    int64_t window;              // 0 = none
    int batch, q_heads, kv_heads, group, page_size, page_shift;
    int tiles_per_seq;           // row tiles that the grid holds per sequence (a sequence with more is walked in steps)
    int splits;                  // parts of the key range
    int64_t split_keys;          // keys per part, a multiple of the key tile; the last part takes what is left
    float scale, softcap;
    float* part_o;               // [splits][T * q_heads][D], not normalised; only with splits > 1
    float2* part_ml;             // [splits][T * q_heads]: running maximum (of base-2 exponents) and sum
    int32_t* dev_status;
    long long wait_cycles;
    int hold;
};

// Scores as exponents of two: p = 2^(value - maximum).  Without a cap that is one product.  The cap's tanh is a polynomial for arguments up to
// kTanhMax and 1 - 2 / (1 + e^2x) above, which saturates without overflow; near zero that difference would keep an absolute accuracy only, and a cap far
// above the scores multiplies it (1e-7 of the cap: at 1e5 weights were off by more than one percent).
// Odd polynomial t (1 + c1 t^2 + ... + c4 t^8), relative error at most 9e-8 (least maximum, fitted on Chebyshev points with the first coefficient held at 1).
constexpr float kTanhMax = 0.6f, kTanh1 = -0.333325975f, kTanh2 = 0.133131167f, kTanh3 = -0.0522118075f, kTanh4 = 0.015612634f;
struct Score {
    float mul, cap2, tmul;       // cap2 = softcap * log2(e), 0 without a cap; tmul: the tanh's argument per score
    __device__ __forceinline__ Score(float scale, float softcap) {
        tmul = softcap > 0.f ? scale / softcap : 0.f;
        mul = softcap > 0.f ? tmul * (2.f * kLog2e) : scale * kLog2e;
        cap2 = softcap > 0.f ? softcap * kLog2e : 0.f;
    }
};
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float capped_near(float t, float cap2) {
    const float u = t * t;
    return __fmul_rn(t * cap2, fmaf(fmaf(fmaf(fmaf(kTanh4, u, kTanh3), u, kTanh2), u, kTanh1), u, 1.f));       // rounded: see kLarge
}
__device__ __forceinline__ float capped_far(float s, const Score& sc) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2(s * sc.mul)));
    return fmaf(-2.f * r, sc.cap2, sc.cap2);
}
// A value is rounded before a reference is taken off it, here and without a cap: a product fused with that difference would keep what the rounding of the
// reference, itself such a value, left out.  From kLarge on (in exponents of two) that passes many exponents, above 2^30 more than kFar, and weights
// would be Inf or all zero.
constexpr float kLarge = 16777216.f;
// (equal to capped_near() where that applies: callers may take either)
__device__ __forceinline__ float capped(float s, const Score& sc) {
    const float t = s * sc.tmul;
    return fabsf(t) <= kTanhMax ? capped_near(t, sc.cap2) : capped_far(s, sc);
}

// two fp32 lanes per instruction
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ bool nonfinite_bf16(uint32_t bits) { return (bits & 0x7f80u) == 0x7f80u; }

// A sequence's bounds; n_new = 0 when it has no new token or when they contradict the token arrays or the page table (reported).
struct Sequence {
    int64_t q0, n_new;
    int kv_len;
};
__device__ __forceinline__ Sequence sequence(const Params& P, int b) {
    Sequence s;
    s.q0 = P.cu_q[b];
    s.n_new = P.cu_q[b + 1] - s.q0;
    s.kv_len = max(P.kv_len[b], 0);                                     // below zero no query sees a key either, and positions keep within 32 bits
    if (s.n_new > 0 && (s.q0 < 0 || s.q0 + s.n_new > P.T || s.kv_len > P.table_width * P.page_size)) {
        report(P.dev_status, MATQ_ERR_PAGE);
        s.n_new = 0;
    }
    return s;
}

// First row, in the cache seen as rows of D elements, of the slots that hold keys key .. key + count - 1 of sequence b, head h (all in one page).
// Slots of which no query sees a key (below `first`, where a sliding window may have given its pages back, or past the sequence) are not looked up: the
// row past the end reads as zeros.  So does a page number that is out of range, which is reported.
__device__ __forceinline__ int page_row(const Params& P, int h, int64_t key, int64_t page) {
    if (page < 0 || page >= P.n_pages) {
        report(P.dev_status, MATQ_ERR_PAGE);
        return (int)(P.n_pages * P.kv_heads * P.page_size);
    }
    return (int)((page * P.kv_heads + h) * P.page_size + (key & (P.page_size - 1)));
}
__device__ __forceinline__ int cache_row(const Params& P, int b, int h, int64_t key, int count, int first, int kv_len) {
    const int64_t last = P.n_pages * P.kv_heads * P.page_size;
    if (key >= kv_len || key + count <= first) return (int)last;
    const int64_t pg = key >> P.page_shift;
    int64_t page = -1;
    if (pg < P.table_width) page = P.table[(int64_t)b * P.table_stride + pg];
    return page_row(P, h, key, page);
}

// Joins the parts of the key range: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  A CTA per (token, head): the weights of the
// parts are made side by side, then eight warps take every eighth part each, and their sums are added in a fixed order.
constexpr int kMaxSplits = 256, kJoinThreads = 256;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const Params P) {
    __shared__ float s_w[kMaxSplits], s_red[2][8];
    __shared__ __align__(16) float s_o[8][D];
    after_previous_kernel();
    let_next_kernel_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t rows = P.T * P.q_heads, row = blockIdx.x, t = row / P.q_heads;
    if (t >= P.cu_q[P.batch]) return;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (tid < P.splits) ml = P.part_ml[(int64_t)tid * rows + row];
    float mx = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (lane == 0) s_red[0][warp] = mx;
    __syncthreads();
    mx = s_red[0][0];
#pragma unroll
    for (int w = 1; w < 8; ++w) mx = fmaxf(mx, s_red[0][w]);
    const bool any = !(ml.x == -INFINITY && ml.y == 0.f);               // the part holds keys of this row
    const float w = any && mx != -INFINITY ? ex2(ml.x - mx) : 0.f;
    s_w[tid] = any ? w : -1.f;                                          // negative: the part's sums were not written
    float sum = any ? ml.y * w : 0.f;
    if (any && mx == -INFINITY) sum = ml.y;                              // NaN
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_red[1][warp] = sum;
    const bool seen = __syncthreads_or(any);
    sum = 0.f;
#pragma unroll
    for (int v = 0; v < 8; ++v) sum += s_red[1][v];
    constexpr int kV = D / 64;                                          // float2 pieces per lane
    float2 acc[kV];
#pragma unroll
    for (int j = 0; j < kV; ++j) acc[j] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int s = warp; s < P.splits; s += 8) {
        const float ws = s_w[s];
        const float2* o = reinterpret_cast<const float2*>(P.part_o + ((int64_t)s * rows + row) * D);
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const float2 v = ws >= 0.f ? o[lane + 32 * j] : make_float2(0.f, 0.f);
            acc[j].x = fmaf(v.x, ws, acc[j].x);
            acc[j].y = fmaf(v.y, ws, acc[j].y);
        }
    }
#pragma unroll
    for (int j = 0; j < kV; ++j) *reinterpret_cast<float2*>(&s_o[warp][2 * (lane + 32 * j)]) = acc[j];
    __syncthreads();
    if (tid < D / 2) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int v = 0; v < 8; ++v) { a += s_o[v][2 * tid]; b += s_o[v][2 * tid + 1]; }
        const float inv = 1.f / sum;
        reinterpret_cast<uint32_t*>(P.out + t * P.ldo + (row - t * P.q_heads) * D)[tid] = seen ? pack_bf16(a * inv, b * inv) : 0u;
    }
}

// The same for up to kFewSplits parts (chunks: many rows, few parts): one warp per (token, head), all parts requested at once.
constexpr int kFewSplits = 8;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attn_join_few_kernel(const Params P) {
    after_previous_kernel();
    let_next_kernel_start();
    const int lane = threadIdx.x & 31;
    const int64_t rows = P.T * P.q_heads, row = (int64_t)blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5);
    if (row >= rows) return;
    const int64_t t = row / P.q_heads;
    if (t >= P.cu_q[P.batch]) return;
    constexpr int kV = D / 64;
    float2 ml[kFewSplits], acc[kV];
    float mx = -INFINITY, sum = 0.f;
    bool seen = false;
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
        ml[s] = s < P.splits ? P.part_ml[(int64_t)s * rows + row] : make_float2(-INFINITY, 0.f);
        mx = fmaxf(mx, ml[s].x);
    }
#pragma unroll
    for (int j = 0; j < kV; ++j) acc[j] = make_float2(0.f, 0.f);
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
        if (ml[s].x == -INFINITY && ml[s].y == 0.f) continue;           // no keys of this row: the part's sums were not written
        seen = true;
        const float w = mx == -INFINITY ? 1.f : ex2(ml[s].x - mx);
        sum = fmaf(ml[s].y, w, sum);
        const float2* o = reinterpret_cast<const float2*>(P.part_o + ((int64_t)s * rows + row) * D);
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const float2 v = o[lane + 32 * j];
            acc[j].x = fmaf(v.x, w, acc[j].x);
            acc[j].y = fmaf(v.y, w, acc[j].y);
        }
    }
    const float inv = 1.f / sum;
    uint32_t* dst = reinterpret_cast<uint32_t*>(P.out + t * P.ldo + (row - t * P.q_heads) * D);
#pragma unroll
    for (int j = 0; j < kV; ++j) dst[lane + 32 * j] = seen ? pack_bf16(acc[j].x * inv, acc[j].y * inv) : 0u;
}

}  // namespace attn
}  // namespace matq
