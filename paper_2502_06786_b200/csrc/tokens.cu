// matq_quantize_tokens: activations to 8 bits with one symmetric scale per token,
//   s_m = max(max_k |X[m,k]| / 127, 2^-126),  xq = clamp(rne(X / s_m), -127, 127),  sum_m = sum_k xq.
//
// One CTA per token; up to K = 16384 the row stays in registers between the two passes (one 16-byte load per thread and 2048
// elements), longer rows are read a second time, from the L2.  Two bytes in and one out per element: HBM-bound for many tokens,
// a launch and two trips to memory for few.
#include "common.cuh"

namespace matq {
namespace tok {

constexpr int kThreads = 256;

// largest of the eight magnitudes, as bf16 bit patterns (their order is that of the magnitudes, NaN above Inf above all)
__device__ __forceinline__ uint32_t abs_max8(uint4 v, uint32_t m) {
    m = __vmaxu2(m, v.x & 0x7fff7fffu);
    m = __vmaxu2(m, v.y & 0x7fff7fffu);
    m = __vmaxu2(m, v.z & 0x7fff7fffu);
    return __vmaxu2(m, v.w & 0x7fff7fffu);
}

// rne(fl(x / s)) in [-127, 127].  x * (1 / s) is within 1.5 * 2^-23 of x / s, relatively, so below 2^-15 absolutely at magnitudes up to 127:
// the two round alike unless the product lies that close to a half, and only then is the division done.
__device__ __forceinline__ int code_of(float x, float s, float inv) {
    const float r = x * inv;
    float k = rintf(r);
    if (fabsf(r - k) > 0.5f - 6.1035e-5f) k = rintf(__fdiv_rn(x, s));
    return (int)fminf(fmaxf(k, -127.f), 127.f);
}

__device__ __forceinline__ uint2 codes8(uint4 v, float s, float inv, int& sum) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c0 = code_of(__uint_as_float(w[2 * h] << 16), s, inv), c1 = code_of(__uint_as_float(w[2 * h] & 0xffff0000u), s, inv);
        const int c2 = code_of(__uint_as_float(w[2 * h + 1] << 16), s, inv), c3 = code_of(__uint_as_float(w[2 * h + 1] & 0xffff0000u), s, inv);
        sum += (c0 + c1) + (c2 + c3);
        o[h] = __byte_perm(__byte_perm((uint32_t)c0, (uint32_t)c1, 0x0040), __byte_perm((uint32_t)c2, (uint32_t)c3, 0x0040), 0x5410);
    }
    return make_uint2(o[0], o[1]);
}

// V > 0: the row fits V 16-byte pieces per thread and stays in registers; V == 0: any length, read twice
template <int V>
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
    const float s = fmaxf(__fdiv_rn(__uint_as_float(mx << 16), 127.f), 1.17549435e-38f);
    const float inv = __fdiv_rn(1.f, s);
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
    const dim3 grid((unsigned)M), block(kThreads);
    cudaError_t e;
    const int64_t per = 8 * kThreads;
    if (K <= per) e = launch_overlapped(quantize_tokens_kernel<1>, grid, block, 0, st, x, K, ldx, xq, ldq, scale, rowsum, dev_status);
    else if (K <= 2 * per) e = launch_overlapped(quantize_tokens_kernel<2>, grid, block, 0, st, x, K, ldx, xq, ldq, scale, rowsum, dev_status);
    else if (K <= 4 * per) e = launch_overlapped(quantize_tokens_kernel<4>, grid, block, 0, st, x, K, ldx, xq, ldq, scale, rowsum, dev_status);
    else if (K <= 8 * per) e = launch_overlapped(quantize_tokens_kernel<8>, grid, block, 0, st, x, K, ldx, xq, ldq, scale, rowsum, dev_status);
    else e = launch_overlapped(quantize_tokens_kernel<0>, grid, block, 0, st, x, K, ldx, xq, ldq, scale, rowsum, dev_status);
    if (e != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}
