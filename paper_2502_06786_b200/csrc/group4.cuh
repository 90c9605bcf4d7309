// The 4-bit group: a run of 32, 64 or 128 bf16 values that shares a scale and a low end, in weights (groups.cu) and in a cache (kv4_append.cu, attn4_*.cuh).
//   low = min x,  scale = bf16((max x - low) / 15)  (0 below 2^-120),  q = rne((x - low) * (1 / scale)),  value = scale * q + low,
// one binary32 operation per step.  q needs no clamp at 15: the scale's rounding makes (max x - low) / scale 15 (1 + 2^-8) at most.  Scale and low stand as two
// bf16 in one word, the scale in its low half.
#pragma once

#include "common.cuh"

namespace matq {

constexpr uint32_t kNoGroup = 0x7fc07fc0u;       // of a group with a NaN or Inf, or whose range passes binary32: scale and low NaN, codes 0

__device__ __forceinline__ float scale_of(uint32_t group) { return __uint_as_float(group << 16); }
__device__ __forceinline__ float low_of(uint32_t group) { return __uint_as_float(group & 0xffff0000u); }
__device__ __forceinline__ float exp2i(int e) { return __int_as_float((e + 127) << 23); }          // -126 <= e <= 127 (128: Inf)

__device__ __forceinline__ uint32_t bf16_rne(float x) { return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x)); }

// Codes (element i in bits 4 i) and group of eight of a group's values; the LANES neighbouring lanes that hold the group call it together.
template <int LANES>
__device__ __forceinline__ uint32_t quantise_piece(uint4 v, uint32_t& codes, uint32_t lanes = 0xffffffffu) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const auto h = [](uint32_t u) { return *reinterpret_cast<const __nv_bfloat162*>(&u); };
    const auto u = [](__nv_bfloat162 b) { return *reinterpret_cast<const uint32_t*>(&b); };
    __nv_bfloat162 lo = __hmin2_nan(__hmin2_nan(h(w[0]), h(w[1])), __hmin2_nan(h(w[2]), h(w[3])));
    __nv_bfloat162 hi = __hmax2_nan(__hmax2_nan(h(w[0]), h(w[1])), __hmax2_nan(h(w[2]), h(w[3])));
#pragma unroll
    for (int s = 1; s < LANES; s <<= 1) {
        lo = __hmin2_nan(lo, h(__shfl_xor_sync(lanes, u(lo), s)));
        hi = __hmax2_nan(hi, h(__shfl_xor_sync(lanes, u(hi), s)));
    }
    const float low = __bfloat162float(__hmin_nan(__low2bfloat16(lo), __high2bfloat16(lo))) + 0.f;         // -0 becomes 0
    const float range = __fsub_rn(__bfloat162float(__hmax_nan(__low2bfloat16(hi), __high2bfloat16(hi))), low);
    codes = 0u;
    if (!(range <= 3.402823466e38f)) return kNoGroup;
    uint32_t scale = bf16_rne(__fdiv_rn(range, 15.f));
    if (__uint_as_float(scale << 16) < 0x1p-120f) scale = 0u;
    if (scale) {
        const float inv = __frcp_rn(__uint_as_float(scale << 16));
        // adding 1.5 * 2^23 rounds to a whole number, half to even, and leaves it in the low bits: the word of sums below is taken modulo 2^32
        uint32_t sum = 0u;
#pragma unroll
        for (int i = 7; i >= 0; --i) {
            const float x = __uint_as_float((i & 1) ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
            sum = sum * 16u + __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x, low), inv), 12582912.f));
        }
        codes = sum - 0x4b400000u * 0x11111111u;
    }
    return scale | (__float_as_uint(low) & 0xffff0000u);
}

// ---------------------------------------------------------------- operands beside codes that enter a product as n * 2^-133 (see groups.cu)
// Eight values in the order of pairs in which masks take eight codes out of a word: (0, 4), (1, 5), (2, 6), (3, 7), all times 2^e and the second and fourth pair
// also times 2^-4.  e brings the largest value of a row near 2^126 (2^127 as a factor is enough for rows below 1): products stay within fp32, and so do the
// rest of the row's values down to 2^-120 of the largest.
__device__ __forceinline__ uint32_t top_of_piece(uint4 v) {             // largest magnitude as the bits of a float
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16) << 16;
}
__device__ __forceinline__ int scale_exponent(uint32_t top) { return min(126 - ((int)(top >> 23) - 127), 127); }      // -2 (NaN, Inf) .. 127
// sums come in units of 2^(133 - e)
__device__ __forceinline__ float in_units(float scaled) { return scaled * 0x1p-67f * 0x1p-66f; }          // of a value times 2^e
__device__ __forceinline__ float from_units(float sum, int e) { return sum * 128.f * exp2i(126 - e); }
__device__ __forceinline__ uint4 operand_of_piece(uint4 v, int e, float& sum) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const float f = exp2i(e);
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16) * f; x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u) * f; }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += in_units(x[i]);
    sum = s;
    const auto pack = [](float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632); };       // exact: a power of two was multiplied
    return make_uint4(pack(x[0], x[4]), pack(x[1] * 0.0625f, x[5] * 0.0625f), pack(x[2], x[6]), pack(x[3] * 0.0625f, x[7] * 0.0625f));
}

// a += codes * tokens: mma.sync m16n8k16, rows g and g + 8 from the words a and b of eight codes each, columns from operand_of_piece
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

}  // namespace matq
