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
// also times 2^-4.  e brings the largest value of a row near 2^118 (2^127 as a factor is enough for rows below 2^-9): products, and sums of values, stay within
// fp32, and so do the rest of the row's values down to 2^-110 of the largest.
__device__ __forceinline__ uint32_t top_of_piece(uint4 v) {             // largest magnitude as the bits of a float
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16) << 16;
}
__device__ __forceinline__ int scale_exponent(uint32_t top) { return min(118 - ((int)(top >> 23) - 127), 127); }      // -10 (NaN, Inf) .. 127
// sums come in units of 2^(133 - e)
__device__ __forceinline__ float unit_of(int e) { return exp2i(118 - e); }                        // times 2^15; at most 2^127 for finite values
__device__ __forceinline__ float from_units(float sum, int e) { return sum * 0x1p15f * unit_of(e); }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint4 operand_of_piece(uint4 v, int e, float& sum) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const uint32_t f = (uint32_t)(e + 127) * 0x00800080u, f4 = f - 4u * 0x00800080u;      // 2^e and 2^(e - 4), twice
    const float scale = exp2i(e);
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = fmaf(__uint_as_float(w[i] << 16), scale, __uint_as_float(w[i] & 0xffff0000u) * scale);
    sum = ((s[0] + s[1]) + (s[2] + s[3])) * 0x1p-67f * 0x1p-66f;         // 2^(e - 133) in all: 2^-133 itself is not a normal number
    return make_uint4(mul_bf16x2(__byte_perm(w[0], w[2], 0x5410), f), mul_bf16x2(__byte_perm(w[0], w[2], 0x7632), f4),
                      mul_bf16x2(__byte_perm(w[1], w[3], 0x5410), f), mul_bf16x2(__byte_perm(w[1], w[3], 0x7632), f4));
}

// a += codes * tokens: mma.sync m16n8k16, rows g and g + 8 from the words a and b of eight codes each, columns from operand_of_piece
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

}  // namespace matq
