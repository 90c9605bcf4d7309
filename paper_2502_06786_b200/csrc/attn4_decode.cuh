// Attention of few query rows over the paged cache in 4-bit groups (kv4_cache.cuh): a CTA takes 4, 8 or 16 rows (token, head of the group) of one key head and a
// part of the key range, as in attn_decode.cuh, and reads a quarter of the bytes.
//
// A page's tile of 16 keys of a head stands together, keys, values and groups.  A warp takes every kWarps-th tile of the CTA's range and brings its own tiles into
// its own ring (cp.async, 16 bytes a lane), so that nothing but the start and the end is shared between warps.  (One bulk copy a tile costs about 50 cycles of the
// SM's copy engine: filling the rings took 4600 cycles at D = 128, 6900 at D = 64.)  Two to four CTAs share an SM: one's start, 3000 cycles of trips to memory,
// and end run beside the other's tiles.  With a tile a warp does
//   S^T = K Q^T     the codes are the rows, masked out of their words without a conversion (groups.cu); per group of 64 elements
//                   s = scale * sum q code + low * sum q, in fp32;
//   O^T += V^T P^T  codes less 8, by one bf16 FMA that also lifts them out of the subnormal numbers; scale goes into the weights, p scale, before they are
//                   rounded to bf16, and low + 8 scale into a sum of its own, sum_j p_j (low + 8 scale), one per row and group.
// That rounding is 2^-8 of a weight's share of code - 8 at most: drafts over a window of 4096 are off by 2.3e-3 of their norm, of which rounding the outputs is 1.7e-3.  A second
// product for what it leaves out, as below, would be half as many products again, in registers that 8 and 16 rows do not have.
// Up to four rows (a single token of a group of four) would leave half of the columns empty, and the lanes that hold them with nothing to do.  There a row has two
// columns: in the first product two digits of the query as a 16-bit integer (its largest element near 2^14; u8 codes times s8 digits, exact; an element is off by
// 2^-15 of the largest at most), which also halves the products and the masks; in the second the weight and what its rounding to bf16 left out.
// ldmatrix with .trans brings two keys' codes of four elements into a word: the four masks of a word give rows of O^T four elements apart, which is undone when
// the lane stores its four neighbouring elements.
//
// Bound.  Single tokens of groups of two or four: HBM in part (64 ragged ones over 5 to 8000 keys, 16/8 heads of 256: 134 us, 4.1 TB/s) and the instructions of a tile;
// one token over 32768 keys, 32/8 heads of 128: 15.5 us, of which the tiles are 8, the start and the join the rest.  8 and 16 rows: instructions and their latencies (1.8
// to 2.3 a cycle of an SM), 46 us for 16 sequences of 8 to 24 rows over a window of 4096.
#pragma once

#include <type_traits>

#include "attn_common.cuh"
#include "kv4_cache.cuh"

namespace matq {
namespace attn {

struct Params4 {
    const __nv_bfloat16* q;
    const uint8_t* tiles;
    __nv_bfloat16* out;
    const int32_t *table, *cu_q, *kv_len;
    int64_t ldq, ldo, table_stride, table_width, n_pages, T;
    int64_t window;              // 0 = none
    int64_t most_rows;           // sequences with more rows (tokens times heads of a group) are left to other kernels
    int batch, q_heads, kv_heads, group, page_size, page_shift;
    int tiles_per_seq;           // row tiles that the grid holds per sequence (a sequence with more is walked in steps)
    int splits;
    int64_t split_keys;
    float scale, softcap;
    float* part_o;               // as in Params
    float2* part_ml;
    int32_t* dev_status;
};

__device__ __forceinline__ Sequence sequence(const Params4& P, int b) {
    Sequence s;
    s.q0 = P.cu_q[b];
    s.n_new = P.cu_q[b + 1] - s.q0;
    s.kv_len = max(P.kv_len[b], 0);
    if (s.n_new > P.most_rows / P.group) s.n_new = 0;
    if (s.n_new > 0 && (s.q0 < 0 || s.q0 + s.n_new > P.T || s.kv_len > P.table_width * P.page_size)) {
        report(P.dev_status, MATQ_ERR_PAGE);
        s.n_new = 0;
    }
    return s;
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transposed8x8(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// (code - 8) / 64 of the codes in bits 0..3 (or 4..7) of both halves of a word
__device__ __forceinline__ uint32_t centred_low(uint32_t w) { return fma_bf16x2(w & 0x000f000fu, 0x7f007f00u, 0xbe00be00u); }          // n 2^-133 * 2^127 - 2^-3
__device__ __forceinline__ uint32_t centred_high(uint32_t w) { return fma_bf16x2(w & 0x00f000f0u, 0x7d007d00u, 0xbe00be00u); }         // 16 n 2^-133 * 2^123 - 2^-3
// a += codes (u8) * digits (s8): mma.sync m16n8k32
__device__ __forceinline__ void mma_u8s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Digit `which` (0: the high one) of eight values times 2^(14 - e) as 16-bit integers: even elements' in the bytes of x, odd ones' in those of y.  An integer is at
// most 32639, so that its high digit fits.  Adding 1.5 * 2^23 rounds to a whole number and leaves it in the low bits; the low digit is their lowest byte, as a
// signed number, and the high one the next byte once half a unit of it has been added.  sum: of the values times 2^(18 - e), before they are rounded.
__device__ __forceinline__ uint2 digits_of_piece(uint4 v, int e, int which, float& sum) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const float f = exp2i(14 - e), magic = which ? 12582912.f : 12582912.f + 128.f;
    const uint32_t pick = which ? 0x0040u : 0x0051u;
    float x[8], s = 0.f;
    uint32_t n[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = __uint_as_float((i & 1) ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16) * f;
        n[i] = __float_as_uint(__fadd_rn(fminf(x[i], 32639.f), magic));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s += x[2 * i] + x[2 * i + 1];
    sum = 16.f * s;
    const auto four = [&](int o) { return __byte_perm(__byte_perm(n[o], n[o + 2], pick), __byte_perm(n[o + 4], n[o + 6], pick), 0x5410); };
    return make_uint2(four(0), four(1));
}

// CTAs of an SM and their warps: what 65536 registers hold without spills (D = 128, four rows: one token over 32768 keys 15.5 us, with ten warps a CTA 16.7; D = 64, four rows,
// 64 tokens over 4000 keys 42.4 us, with three CTAs of eight warps 47), but for D = 256 with four rows, where 16 warps that spill are faster than 12 (134 against 145 us).
__host__ __device__ constexpr int decode4_ctas(int D, int R) { return D == 64 && R == 4 ? 4 : 2; }
__host__ __device__ constexpr int decode4_warps(int D, int R) { return (D == 64 && R == 4) || (D == 256 && R == 8) || (D == 128 && R == 16) ? 6 : 8; }

// R: query rows of a CTA: 4 (two columns each), 8 or 16
template <int D, int R>
struct Dec4Cfg {
    static constexpr int kRows = R, kCtas = decode4_ctas(D, R);
    static constexpr int kWarps = decode4_warps(D, R), kThreads = 32 * kWarps;
    static constexpr int kTile = kv4::tile_bytes(D);
    // Tiles of a warp's ring.  80 KB in flight on an SM keep HBM busy; what is requested beyond that only stands in the way of other CTAs' queries and page numbers
    // (with rings of 200 KB an SM's queries took 5 us to come).
    static constexpr int kDepth = 80 * 1024 / (kCtas * kWarps * kTile) < 2 ? 2 : 80 * 1024 / (kCtas * kWarps * kTile);
    static constexpr int kMergeStride = D + 4;
    static constexpr size_t kRing = (size_t)kWarps * kDepth * kTile, kMerge = (size_t)kWarps * kRows * kMergeStride * 4;
    static constexpr size_t kSmem = kRing > kMerge ? kRing : kMerge;
    static_assert(kCtas * (kSmem + 8192) <= 227 * 1024, "shared memory");
};

template <int D, int R>
__global__ void __launch_bounds__(Dec4Cfg<D, R>::kThreads, Dec4Cfg<D, R>::kCtas) attn4_decode_kernel(const Params4 P) {
    using C = Dec4Cfg<D, R>;
    constexpr int kRows = C::kRows, kGroups64 = D / 64, kWarps = C::kWarps, kDepth = C::kDepth;
    constexpr bool kDigits = R == 4;
    constexpr int NT = R == 16 ? 2 : 1, V = kDigits ? 1 : 2;            // blocks of 8 columns; rows of a block that a lane holds
    extern __shared__ __align__(128) unsigned char smem_raw[];
    constexpr int kPieces = kDigits ? kGroups64 : D / 32;               // of a column's operand
    __shared__ uint4 s_q[NT][kPieces][32];
    __shared__ float s_sums[kRows][D / 32], s_mul[kRows];
    __shared__ float s_m[kRows][kWarps], s_l[kRows][kWarps];
    __shared__ Sequence s_seq;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    const int part = (int)(blockIdx.x % (unsigned)P.splits);
    const unsigned rest = blockIdx.x / (unsigned)P.splits;
    const int h = (int)(rest % (unsigned)P.kv_heads);
    const int bt = (int)(rest / (unsigned)P.kv_heads);
    const int b = bt / P.tiles_per_seq;
    after_previous_kernel();
    // Without a window the first keys of a part are known before the sequence's bounds are: their pages' numbers are looked up side by side with them.
    int early = -1;
    if (!P.window) {
        const int64_t pg = ((int64_t)part * P.split_keys + 16 * warp + 16ll * kWarps * lane) >> P.page_shift;
        if (pg < P.table_width) early = P.table[(int64_t)b * P.table_stride + pg];
    }
    if (tid == 0) s_seq = sequence(P, b);                               // read once: all warps act on the same numbers
    __syncthreads();
    let_next_kernel_start();
    const int64_t q0 = s_seq.q0, n_new = s_seq.n_new;
    const int kv_len = s_seq.kv_len;
    if (n_new <= 0) return;
    const int64_t n_rows = n_new * P.group, tiles = (n_rows + kRows - 1) / kRows;
    const int64_t ctx = kv_len - n_new;                                 // position of the first new token (negative: it sees nothing)
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem_raw) + (uint32_t)warp * (kDepth * C::kTile);

    for (int64_t tile = bt - (int64_t)b * P.tiles_per_seq; tile < tiles; tile += P.tiles_per_seq) {
        const int64_t r0 = tile * kRows, r1 = min(r0 + kRows, n_rows) - 1;           // first and last row
        // Row r of position p sees the keys [lo(p), p].  Positions stay below kv_len, an int.
        const auto lo = [&](int64_t p) { return P.window && p - P.window + 1 > 0 ? (int)(p - P.window + 1) : 0; };
        // Row i of this row tile is token tok0 + (rem0 + i) / group of the sequence.
        const unsigned group = (unsigned)P.group;
        const int64_t tok0 = r0 < 0xffffffffll ? (int64_t)((unsigned)r0 / group) : r0 / P.group;
        const unsigned rem0 = (unsigned)(r0 - tok0 * P.group);
        const int live_rows = (int)(r1 - r0) + 1;
        const int p_lo = (int)(ctx + tok0), p_hi = (int)(ctx + tok0 + (rem0 + live_rows - 1) / group);
        const int first = lo(p_lo), all_from = lo(p_hi);                // some row sees [first, p_hi], every row [all_from, p_lo]
        const int64_t k_lo = (first & ~15) + part * P.split_keys;
        int64_t k_hi = (int64_t)p_hi + 1;
        if (part + 1 < P.splits) k_hi = min(k_hi, k_lo + P.split_keys);
        // tiles of this CTA, and of this warp: the warp's n-th has the keys from k_lo + 16 (warp + kWarps n) on
        const int all = k_hi > k_lo ? (int)((k_hi - k_lo + 15) / 16) : 0, mine = all > warp ? (all - warp + kWarps - 1) / kWarps : 0;
        const int j_first = mine ? (int)k_lo + 16 * warp : 0;

        const int g = lane >> 2, q4 = lane & 3, c2 = q4 * 2;
        // ---------------- queries: made once, a piece of all columns by each warp, and read by all.  They are requested before the tiles, which would be in their way.
        static_assert(NT * kPieces <= 2 * kWarps, "a warp has at most two pieces");
        uint4 raw[D / 32];
        const auto request = [&](int u) {
            const int row = kDigits ? g >> 1 : u / kPieces * 8 + g;
            const bool live = row < live_rows;
            const unsigned tok = live ? (rem0 + row) / group : 0u, head = live ? rem0 + row - tok * group : 0u;
            const __nv_bfloat16* src = P.q + (q0 + tok0 + tok) * P.ldq + (int64_t)(h * P.group + (int)head) * D + 8 * q4;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) raw[i] = live ? *reinterpret_cast<const uint4*>(src + 32 * i) : make_uint4(0u, 0u, 0u, 0u);
        };
        if (warp < NT * kPieces) request(warp);
        // ---------------- copies
        const int64_t page_tiles = P.page_size >> 4;
        // lane y: the page of the warp's tile n + y, and where that tile stands (-1: its page is out of range); a block of 32 is looked up one block ahead
        const auto pages_from = [&](int n) {
            const int64_t pg = (int64_t)(j_first + 16ll * kWarps * (n + lane)) >> P.page_shift;
            return n + lane < mine && pg < P.table_width ? P.table[(int64_t)b * P.table_stride + pg] : -1;
        };
        const auto tile_at = [&](int page, int n) -> int64_t {
            const int key = (j_first + 16 * kWarps * (n + lane)) & (P.page_size - 1);
            return page >= 0 && page < P.n_pages ? ((int64_t)page * P.kv_heads + h) * page_tiles + (key >> 4) : -1;
        };
        int64_t where = tile_at(P.window || tile >= P.tiles_per_seq ? pages_from(0) : lane < mine ? early : -1, 0);
        int pages_next = pages_from(32), issued = 0;
        uint32_t in_at = ring;
        const auto issue = [&] {                                        // the warp's tile `issued` into the ring; an empty group of copies behind the last one
            if (issued < mine) {
                if ((issued & 31) == 0 && issued > 0) {
                    where = tile_at(pages_next, issued);
                    pages_next = pages_from(issued + 32);
                }
                const int64_t at = __shfl_sync(0xffffffffu, where, issued & 31);
                if (at >= 0) {
                    const uint8_t* src = P.tiles + at * C::kTile + lane * 16;
#pragma unroll
                    for (int i = 0; i < C::kTile / 512; ++i) copy16(in_at + lane * 16 + i * 512, src + i * 512);
                    if (C::kTile % 512 != 0 && lane < C::kTile % 512 / 16) copy16(in_at + lane * 16 + C::kTile / 512 * 512, src + C::kTile / 512 * 512);
                } else if (lane == 0) {
                    report(P.dev_status, MATQ_ERR_PAGE);
                }
                ++issued;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            in_at = in_at == ring + (kDepth - 1) * C::kTile ? ring : in_at + C::kTile;
        };
        const Score sc(P.scale, P.softcap);
        Score of_argument = sc;                                         // of what is tmul times a score already
        of_argument.tmul = 1.f;
        of_argument.mul = 2.f * kLog2e;
#pragma unroll 1
        for (int n = 0; n < kDepth; ++n) issue();
        for (int u = warp; u < NT * kPieces; u += kWarps) {
            if (u != warp) request(u);
            const int nt = u / kPieces, c = u % kPieces, row = kDigits ? g >> 1 : nt * 8 + g;
            uint32_t top = 0u;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) top = max(top, top_of_piece(raw[i]));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = kDigits ? max((int)(top >> 23) - 127, -112) : scale_exponent(top);
            // 2^(133 - e) a unit, or 2^(e - 18); NaN for a row with NaN or Inf, whose digits say nothing
            const float unit = kDigits ? (top >= 0x7f800000u ? NAN : exp2i(e)) : unit_of(e);
            if (c == 0 && q4 == 0) s_mul[row] = unit * (sc.cap2 > 0.f ? sc.tmul : sc.mul) * (kDigits ? 0x1p-18f : 0x1p15f);
#pragma unroll
            for (int i = 0; i < (kDigits ? 2 : 1); ++i) {               // pieces of 32 elements
                uint4 piece = raw[0];
#pragma unroll
                for (int j = 1; j < D / 32; ++j)
                    if (j == (kDigits ? 2 * c + i : c)) piece = raw[j];
                float sum;
                uint32_t* to = reinterpret_cast<uint32_t*>(&s_q[nt][c][lane]);
                if constexpr (kDigits) {
                    const uint2 d = digits_of_piece(piece, e, g & 1, sum);
                    to[i] = d.x;
                    to[2 + i] = d.y;
                } else {
                    *reinterpret_cast<uint4*>(to) = operand_of_piece(piece, e, sum);
                }
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if (q4 == 0) s_sums[row][kDigits ? 2 * c + i : c] = sum;
            }
        }
        __syncthreads();
        // Column g of the queries: operand_of_piece of elements 32 c + 8 q4 .., or per 64 elements the digits for even and for odd ones.  In registers where they fit.
        constexpr bool kHeld = R == 8 || (R == 4 && D == 64);
        uint4 held[kHeld ? NT : 1][kHeld ? kPieces : 1];
        // Of the rows that this lane holds scores of (q4, or 8 nt + c2 and the next): sums of the query per group of 64, in the score's units; the factor that makes
        // scores exponents of two (with a cap: arguments of its tanh) out of these units; the keys that they see, [see_lo, see_hi].
        float qs[NT][V][kGroups64], mul[NT][V];
        int see_hi[NT][V], see_lo[NT][V];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if constexpr (kHeld) {
#pragma unroll
                for (int c = 0; c < kPieces; ++c) held[nt][c] = s_q[nt][c][lane];
            }
#pragma unroll
            for (int w = 0; w < V; ++w) {
                const int row = kDigits ? q4 : nt * 8 + c2 + w;
#pragma unroll
                for (int i = 0; i < kGroups64; ++i) qs[nt][w][i] = s_sums[row][2 * i] + s_sums[row][2 * i + 1];
                mul[nt][w] = s_mul[row];
                see_hi[nt][w] = row < live_rows ? (int)(ctx + tok0 + (rem0 + row) / group) : p_hi;
                see_lo[nt][w] = lo(see_hi[nt][w]);
            }
        }
        // 16 t: elements 32 (t / 2) + 4 g + 2 (t & 1) (+ 1 from [2] on) of columns c2, c2 + 1
        float o[D / 16][NT][4];
        float extra[NT][V][kGroups64];                                  // sum_j p_j (low_j + 8 scale_j) over this lane's keys
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][nt][e] = 0.f;
        float m[NT][V], raise_at[NT][V], l[NT][V];                      // reference of a row's exponents (0 as long as it has none), where it moves, sum
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int w = 0; w < V; ++w) {
                raise_at[nt][w] = -INFINITY;
                m[nt][w] = l[nt][w] = 0.f;
#pragma unroll
                for (int i = 0; i < kGroups64; ++i) extra[nt][w][i] = 0.f;
            }
        const auto operand = [&](int nt, int c) {
            if constexpr (kHeld) return held[nt][c];
            else {
                uint4 f;                                                // not to be kept in registers: volatile
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(f.x), "=r"(f.y), "=r"(f.z), "=r"(f.w) : "r"((uint32_t)__cvta_generic_to_shared(&s_q[nt][c][lane])));
                return f;
            }
        };
        uint32_t at = ring;
        const auto take = [&](const int j0, auto masked_tile) {         // the tile in this slot; masked_tile: not every row sees every key
            constexpr bool masked = decltype(masked_tile)::value;
            const uint32_t kb = at, vb = kb + kv4::half_bytes(D);
            float x[NT][2][V];                                          // keys g and g + 8
#pragma unroll
            for (int c = 0; c < kGroups64; ++c) {
                uint32_t w[4];
                ldmatrix4(w, kb + c * 512 + lane * 16);                 // keys g and g + 8 of 32 elements, then of the next 32
                const uint32_t gr[2] = {lds32(kb + kv4::groups_at(D) + c * 64 + g * 4), lds32(kb + kv4::groups_at(D) + c * 64 + 32 + g * 4)};
                float acc[NT][2][V];
                if constexpr (kDigits) {
                    int even[4] = {}, odd[4] = {};                      // odd elements' codes come times 16
                    const uint4 f = operand(0, c);
                    mma_u8s8(even, w[0] & 0x0f0f0f0fu, w[1] & 0x0f0f0f0fu, w[2] & 0x0f0f0f0fu, w[3] & 0x0f0f0f0fu, f.x, f.y);
                    mma_u8s8(odd, w[0] & 0xf0f0f0f0u, w[1] & 0xf0f0f0f0u, w[2] & 0xf0f0f0f0u, w[3] & 0xf0f0f0f0u, f.z, f.w);
#pragma unroll
                    for (int kh = 0; kh < 2; ++kh) acc[0][kh][0] = (float)((16 * even[2 * kh] + odd[2 * kh]) * 256 + (16 * even[2 * kh + 1] + odd[2 * kh + 1]));
                } else {
                    float sums[NT][4] = {};
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const uint32_t a = w[2 * f], bb = w[2 * f + 1], a8 = a >> 8, b8 = bb >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint4 qv = operand(nt, 2 * c + f);
                            mma_bf16(sums[nt], a & 0x000f000fu, bb & 0x000f000fu, a & 0x00f000f0u, bb & 0x00f000f0u, qv.x, qv.y);
                            mma_bf16(sums[nt], a8 & 0x000f000fu, b8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x00f000f0u, qv.z, qv.w);
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[nt][e >> 1][(e & 1) % V] = sums[nt][e];
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            const float low = c == 0 ? low_of(gr[kh]) * qs[nt][v][c] : fmaf(low_of(gr[kh]), qs[nt][v][c], x[nt][kh][v]);
                            x[nt][kh][v] = fmaf(scale_of(gr[kh]), acc[nt][kh][v], low);
                        }
            }
            bool raise = false, seen[NT][2][V];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int kh = 0; kh < 2; ++kh)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float s = __fmul_rn(x[nt][kh][v], mul[nt][v]);
                        if (sc.cap2 > 0.f) s = capped(s, of_argument);
                        const int j = j0 + g + kh * 8;
                        seen[nt][kh][v] = !masked || (j <= see_hi[nt][v] && j >= see_lo[nt][v]);
                        x[nt][kh][v] = seen[nt][kh][v] ? s : -INFINITY;
                        raise |= x[nt][kh][v] > raise_at[nt][v];        // also from -inf to anything finite
                    }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float top = fmaxf(x[nt][0][v], x[nt][1][v]);
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                        const bool none = raise_at[nt][v] == -INFINITY;
                        if (top > (none ? -INFINITY : m[nt][v])) {
                            const float f = none ? 1.f : ex2(m[nt][v] - top);          // without a reference the sums are zero
                            m[nt][v] = top;
                            raise_at[nt][v] = top + kFar;
                            l[nt][v] *= f;
#pragma unroll
                            for (int c = 0; c < kGroups64; ++c) extra[nt][v][c] *= f;
#pragma unroll
                            for (int t = 0; t < D / 16; ++t)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (kDigits || (e & 1) == v) o[t][nt][e] *= f;
                        }
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int v = 0; v < V; ++v) {
#pragma unroll
                    for (int kh = 0; kh < 2; ++kh) x[nt][kh][v] = ex2(x[nt][kh][v] - m[nt][v]);
                    l[nt][v] += x[nt][0][v] + x[nt][1][v];
                }
#pragma unroll
            for (int c = 0; c < kGroups64; ++c) {
                const uint32_t gr[2] = {lds32(vb + kv4::groups_at(D) + c * 64 + g * 4), lds32(vb + kv4::groups_at(D) + c * 64 + 32 + g * 4)};
                uint32_t pb[NT][2];
#pragma unroll
                for (int kh = 0; kh < 2; ++kh) {
                    const float scale = scale_of(gr[kh]), mid = fmaf(scale, 8.f, low_of(gr[kh]));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float p[2];
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            // a weight of zero does not silence what a slot holds that the row does not see
                            p[v] = seen[nt][kh][v] ? x[nt][kh][v] * scale : 0.f;
                            extra[nt][v][c] = seen[nt][kh][v] ? fmaf(x[nt][kh][v], mid, extra[nt][v][c]) : extra[nt][v][c];
                        }
                        if (kDigits) {
                            const float hi = __uint_as_float(pack_bf16(0.f, p[0]));          // the rounded weight: its bits are the upper half
                            pb[nt][kh] = transposed8x8(pack_bf16(hi, p[0] - hi));
                        } else {
                            pb[nt][kh] = transposed8x8(pack_bf16(p[0], p[V - 1]));
                        }
                    }
                }
                uint32_t w[4];
                ldmatrix4t(w, vb + c * 512 + lane * 16);                // keys 2 q4 (+ 1) and 8 + 2 q4 (+ 1): elements 4 g .. of 32, then of the next 32
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const uint32_t a = w[2 * f], bb = w[2 * f + 1], a8 = a >> 8, b8 = bb >> 8;
                    const uint32_t e0 = centred_low(a), e1 = centred_high(a), e2 = centred_low(bb), e3 = centred_high(bb);
                    const uint32_t f0 = centred_low(a8), f1 = centred_high(a8), f2 = centred_low(b8), f3 = centred_high(b8);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma_bf16(o[4 * c + 2 * f][nt], e0, e1, e2, e3, pb[nt][0], pb[nt][1]);
                        mma_bf16(o[4 * c + 2 * f + 1][nt], f0, f1, f2, f3, pb[nt][0], pb[nt][1]);
                    }
                }
            }
        };
#pragma unroll 1
        for (int n = 0; n < mine; ++n) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
            __syncwarp();
            const int j0 = j_first + 16 * kWarps * n;
            if (j0 + 15 > p_lo || j0 < all_from) take(j0, std::true_type{});
            else take(j0, std::false_type{});
            __syncwarp();                                               // the slot has been read
            at = at == ring + (kDepth - 1) * C::kTile ? ring : at + C::kTile;
            issue();
        }
        // ---------------- join of the warps (their key sets are disjoint)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) l[nt][v] += __shfl_xor_sync(0xffffffffu, l[nt][v], w);
#pragma unroll
                for (int c = 0; c < kGroups64; ++c)
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) extra[nt][v][c] += __shfl_xor_sync(0xffffffffu, extra[nt][v][c], w);
                const int row = kDigits ? q4 : nt * 8 + c2 + v;
                if (g == 0) { s_m[row][warp] = raise_at[nt][v] == -INFINITY ? -INFINITY : m[nt][v]; s_l[row][warp] = l[nt][v]; }
            }
        __syncthreads();
        float* merge = reinterpret_cast<float*>(smem_raw);               // all copies of this row tile have been read
        if (mine > 0) {
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float z = extra[nt][v][c / 2];
                        const int row = kDigits ? q4 : nt * 8 + c2 + v;
                        const auto of = [&](const float (&a)[4], int e) { return fmaf(kDigits ? a[e] + a[e + 1] : a[e + v], 64.f, z); };
                        *reinterpret_cast<float4*>(merge + (size_t)(warp * kRows + row) * C::kMergeStride + 32 * c + 4 * g) =
                            make_float4(of(o[2 * c][nt], 0), of(o[2 * c][nt], 2), of(o[2 * c + 1][nt], 0), of(o[2 * c + 1][nt], 2));
                    }
        }
        __syncthreads();
        // Two neighbouring elements a thread; every thread makes the factors of its row's warps for itself.  A warp without keys has m = -inf and sums of zero;
        // all scores NaN leaves m = -inf and a sum of NaN.
        const int used = all < kWarps ? all : kWarps;                   // warps with keys
        for (int i = tid; i < live_rows * (D / 2); i += C::kThreads) {
            const int r = i / (D / 2), c = (i % (D / 2)) * 2;
            float f[kWarps], mx = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) { f[w] = s_m[r][w]; mx = fmaxf(mx, f[w]); }
            float2 a = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                f[w] = mx == -INFINITY ? 1.f : ex2(f[w] - mx);
                sum = fmaf(s_l[r][w], f[w], sum);
                const float2 v = w < used ? *reinterpret_cast<const float2*>(merge + (size_t)(w * kRows + r) * C::kMergeStride + c) : make_float2(0.f, 0.f);
                a.x = fmaf(v.x, f[w], a.x); a.y = fmaf(v.y, f[w], a.y);
            }
            const unsigned t = (rem0 + r) / group;
            const int64_t tok = tok0 + t;
            const int head = h * P.group + (int)(rem0 + r - t * group);
            if (P.splits > 1) {
                const int64_t row = (int64_t)part * (P.T * P.q_heads) + (q0 + tok) * P.q_heads + head;
                if (c == 0) P.part_ml[row] = make_float2(mx, sum);
                if (all > 0) *reinterpret_cast<float2*>(P.part_o + row * D + c) = a;
            } else {
                const float inv = 1.f / sum;
                *reinterpret_cast<uint32_t*>(P.out + (q0 + tok) * P.ldo + (int64_t)head * D + c) = ctx + tok < 0 ? 0u : pack_bf16(a.x * inv, a.y * inv);
            }
        }
        __syncthreads();                                                // before the next row tile's copies
    }
}

}  // namespace attn
}  // namespace matq
