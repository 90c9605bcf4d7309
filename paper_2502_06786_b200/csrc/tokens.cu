// matq_quantize_tokens: activations to 8 bits with one symmetric scale per token,
//   s_m = max(max_k |X[m,k]| / 127, 2^-126),  xq = clamp(rne(X / s_m), -127, 127),  sum_m = sum_k xq.
//
// One CTA per token; up to K = 16384 the row stays in registers between the two passes (one 16-byte load per thread and 2048
// elements), longer rows are read a second time, from the L2.  Two bytes in and one out per element: HBM-bound for many tokens,
// a launch and two trips to memory for few.  4096 x 14336: 36 us = 4.9 TB/s; one token of 2304: 1.9 us.
#include "common.cuh"

namespace matq {
namespace tok {


// largest of the eight magnitudes, as bf16 bit patterns (their order is that of the magnitudes, NaN above Inf above all)
__device__ __forceinline__ uint32_t abs_max8(uint4 v, uint32_t m) {
    m = __vmaxu2(m, v.x & 0x7fff7fffu);
    m = __vmaxu2(m, v.y & 0x7fff7fffu);
    m = __vmaxu2(m, v.z & 0x7fff7fffu);
    return __vmaxu2(m, v.w & 0x7fff7fffu);
}

// Codes of eight elements.  k = rne(x * (1 / s)) by adding and taking off 1.5 * 2^23, whose low byte is then k's; no result passes 127, since |x| <= 127 s up to
// a rounding.  x * (1 / s) is within 1.5 * 2^-23 of x / s relatively, so below 2^-15 absolutely: it rounds like the correctly rounded quotient unless it lies
// that close to a half, and only then is the division done.
__device__ __forceinline__ uint32_t bits_of(float x, float inv, float& worst) {
    constexpr float kMagic = 12582912.f;
    const float r = x * inv, t = r + kMagic;
    worst = fmaxf(worst, fabsf(r - (t - kMagic)));
    return __float_as_uint(t);
}
__device__ __noinline__ uint2 codes8_divided(uint4 v, float s) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        o[e >> 2] |= ((uint32_t)(int)rintf(__fdiv_rn(x, s)) & 0xffu) << (8 * (e & 3));
    }
    return make_uint2(o[0], o[1]);
}
__device__ __forceinline__ uint2 codes8(uint4 v, float s, float inv, int& sum) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t b[8];
    float worst = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        b[2 * e] = bits_of(__uint_as_float(w[e] << 16), inv, worst);
        b[2 * e + 1] = bits_of(__uint_as_float(w[e] & 0xffff0000u), inv, worst);
    }
    uint2 o = make_uint2(__byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410),
                         __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410));
    if (worst > 0.5f - 6.1035e-5f) o = codes8_divided(v, s);
    sum = __dp4a((int)o.x, 0x01010101, __dp4a((int)o.y, 0x01010101, sum));
    return o;
}
__device__ __forceinline__ float scale_of(uint32_t mx) { return fmaxf(__fdiv_rn(__uint_as_float(mx << 16), 127.f), 1.17549435e-38f); }

// V > 0: the row fits V 16-byte pieces per thread and stays in registers; V == 0: any length, read twice
template <int V, int kThreads>
__global__ void __launch_bounds__(kThreads)
quantize_tokens_kernel(const __nv_bfloat16* __restrict__ X, int64_t K, int64_t ldx, int8_t* __restrict__ xq, int64_t ldq,
                       float* __restrict__ scale, int32_t* __restrict__ rowsum, int32_t* dev_status) {
    __shared__ uint32_t s_max[kThreads / 32];
    __shared__ int s_sum[kThreads / 32];
    after_previous_kernel();
    let_next_kernel_start();
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n8 = (int)(K / 8);
    const uint4* row = reinterpret_cast<const uint4*>(X + m * ldx);
    uint4 v[V > 0 ? V : 1];
    uint32_t mx = 0;
    if (V > 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int i = tid + j * kThreads;
            v[j] = i < n8 ? __ldg(row + i) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) mx = abs_max8(v[j], mx);
    } else {
        for (int i = tid; i < n8; i += kThreads) mx = abs_max8(__ldg(row + i), mx);
    }
    mx = max(mx & 0xffffu, mx >> 16);
    mx = __reduce_max_sync(0xffffffffu, mx);
    if (lane == 0) s_max[warp] = mx;
    __syncthreads();
    mx = s_max[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) mx = max(mx, s_max[w]);
    const bool finite = mx < 0x7f80u;
    const float s = scale_of(mx), inv = __fdiv_rn(1.f, s);
    int sum = 0;
    uint2* out = reinterpret_cast<uint2*>(xq + m * ldq);
    if (V > 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int i = tid + j * kThreads;
            if (i < n8) out[i] = finite ? codes8(v[j], s, inv, sum) : make_uint2(0, 0);
        }
    } else {
        for (int i = tid; i < n8; i += kThreads) out[i] = finite ? codes8(__ldg(row + i), s, inv, sum) : make_uint2(0, 0);
    }
    sum = __reduce_add_sync(0xffffffffu, sum);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        int total = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) total += s_sum[w];
        scale[m] = finite ? s : __uint_as_float(0x7fffffffu);
        rowsum[m] = total;
        if (!finite) report(dev_status, MATQ_ERR_NONFINITE);
    }
}

}  // namespace tok
}  // namespace matq

extern "C" int matq_quantize_tokens(const void* X, int64_t M, int64_t K, int64_t ldx, int8_t* xq, int64_t ldq, float* scale,
                                    int32_t* rowsum, int32_t* dev_status, void* stream) {
    using namespace matq;
    using namespace matq::tok;
    if (M < 0 || K <= 0) return MATQ_ERR_INVALID_ARG;
    if (M >= (1ll << 31) || K % 16 != 0 || K > 65536 || ldx < K || ldx % 8 != 0 || ldq < K || ldq % 16 != 0) return MATQ_ERR_SHAPE;
    if (M == 0) return MATQ_OK;
    if (!X || !xq || !scale || !rowsum) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(xq)) return MATQ_ERR_ALIGNMENT;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(X);
    cudaError_t e;
    // Many tokens: 128 threads (256 for long rows), so that an SM holds more rows between their two barriers (4096 x 14336: 36 us, with 1024 threads 52).  Few: as many
    // threads as hold a row in two loads each (600 x 9216 as many 6.1 us, 5 x 10608 as few 2.5 instead of 4.1).
#define MATQ_ROWS(V, THREADS) launch_overlapped(quantize_tokens_kernel<V, THREADS>, dim3((unsigned)M), dim3(THREADS), 0, st, x, K, ldx, xq, ldq, scale, rowsum, dev_status)
    const bool many = M >= 4 * sm_count();
    if (K <= 1024) e = MATQ_ROWS(1, 128);
    else if (K <= 2048) e = many ? MATQ_ROWS(2, 128) : MATQ_ROWS(1, 256);
    else if (K <= 4096) e = many ? MATQ_ROWS(4, 128) : MATQ_ROWS(2, 256);
    else if (K <= 8192) e = many ? MATQ_ROWS(8, 128) : MATQ_ROWS(2, 512);
    else if (K <= 16384) e = many ? MATQ_ROWS(8, 256) : MATQ_ROWS(2, 1024);
    else e = MATQ_ROWS(0, 512);
#undef MATQ_ROWS
    if (e != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}
