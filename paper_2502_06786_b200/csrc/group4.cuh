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

// Two binary32 operations per instruction.  A sum of such products is taken one by one: the two together come out as one fused operation, whatever they say of rounding.
__device__ __forceinline__ uint64_t two(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t two_sums(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t two_products(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// range / 15 and 1 / scale with the result of a correctly rounded division: a quotient from the rounded reciprocal, corrected by its exact residual, is (Markstein); a
// Newton step on a reciprocal that is off by 2^-23 leaves 2^-46, and 1 / scale, the scale having eight bits, is no nearer than 2^-33 to the middle of two numbers.
__device__ __forceinline__ float fifteenth(float range) {
    constexpr float k = 1.f / 15.f;
    const float q = range * k;
    return fmaf(fmaf(-15.f, q, range), k, q);
}
__device__ __forceinline__ float inverse(float scale) {                 // of a normal number with eight bits
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(scale));
    return fmaf(fmaf(-scale, y, 1.f), y, y);
}

// Codes (element i in bits 4 i) and group of eight of a group's values; the LANES neighbouring lanes that hold the group call it together.
template <int LANES>
__device__ __forceinline__ uint32_t quantise_piece(uint4 v, uint32_t& codes, uint32_t lanes = 0xffffffffu) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const auto h = [](uint32_t u) { return *reinterpret_cast<const __nv_bfloat162*>(&u); };
    const auto u = [](__nv_bfloat162 b) { return *reinterpret_cast<const uint32_t*>(&b); };
    // the smallest value, and the largest one with its sign turned, side by side: one shuffle and one minimum a step (NaN stays NaN)
    const uint32_t lo = u(__hmin2_nan(__hmin2_nan(h(w[0]), h(w[1])), __hmin2_nan(h(w[2]), h(w[3]))));
    const uint32_t hi = u(__hmax2_nan(__hmax2_nan(h(w[0]), h(w[1])), __hmax2_nan(h(w[2]), h(w[3])))) ^ 0x80008000u;
    uint32_t ends = u(__hmin2_nan(h(__byte_perm(lo, hi, 0x5410)), h(__byte_perm(lo, hi, 0x7632))));
#pragma unroll
    for (int s = 1; s < LANES; s <<= 1) ends = u(__hmin2_nan(h(ends), h(__shfl_xor_sync(lanes, ends, s))));
    const float low = __uint_as_float(ends << 16) + 0.f;                // -0 becomes 0
    const float range = __fsub_rn(__uint_as_float((ends & 0xffff0000u) ^ 0x80000000u), low);
    uint32_t scale = bf16_rne(fifteenth(range));
    const bool flat = __uint_as_float(scale << 16) < 0x1p-120f;
    if (flat) scale = 0u;
    const float inv = flat ? 0.f : inverse(__uint_as_float(scale << 16));
    // adding 1.5 * 2^23 rounds to a whole number, half to even, and leaves it in the low bits: the word of sums below is taken modulo 2^32
    const uint64_t less = two(-low, -low), by = two(inv, inv);
    uint32_t sum = 0u;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
        const uint64_t t = two_products(two_sums(two(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), less), by);
        const uint32_t even = __float_as_uint(__fadd_rn(__uint_as_float((uint32_t)t), 12582912.f)), odd = __float_as_uint(__fadd_rn(__uint_as_float((uint32_t)(t >> 32)), 12582912.f));
        sum = (sum * 16u + odd) * 16u + even;
    }
    const bool none = !(range <= 3.402823466e38f);
    codes = none ? 0u : sum - 0x4b400000u * 0x11111111u;
    return none ? kNoGroup : scale | (__float_as_uint(low) & 0xffff0000u);
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

// codes * tokens, and a += codes * tokens: mma.sync m16n8k16, rows g and g + 8 from the words a and b of eight codes each, columns from operand_of_piece
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

}  // namespace matq
