// Attention of few query rows over the paged cache in 4-bit groups (kv4_cache.cuh): a CTA takes 8 or 16 rows (token, head of the group) of one key head and a
// part of the key range, as in attn_decode.cuh, and reads a quarter of the bytes.
//
// One producer warp fills a ring with bulk copies: a page's tiles of a head stand together, keys, values and groups, so a stage is one to eight copies.
// A consumer warp takes a tile of 16 keys:
//   S^T = K Q^T     the codes are the rows, masked out of their words without a conversion (groups.cu); per group of 64 elements
//                   s = scale * sum q code + low * sum q, in fp32;
//   O^T += V^T P^T  codes less 8, by one bf16 FMA that also lifts them out of the subnormal numbers; scale goes into the weights, p scale, before they are
//                   rounded to bf16, and low + 8 scale into a sum of its own, sum_j p_j (low + 8 scale), one per row and group.
// ldmatrix with .trans brings two keys' codes of four elements into a word: the four masks of a word give rows of O^T four elements apart, which is undone when
// the lane stores its four neighbouring elements.
#pragma once

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
    long long wait_cycles;
    int hold;
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
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
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
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// NT: columns of 8 query rows
template <int D, int NT>
struct Dec4Cfg {
    static constexpr int kRows = 8 * NT;
    static constexpr int kKeys = D == 64 ? 128 : 64;                    // keys per stage
    static constexpr int kGroupWarps = kKeys / 16;                      // a tile each
    static constexpr int kGroups = D == 64 ? 2 : D == 256 || NT == 2 ? 3 : 4;
    static constexpr int kWarps = kGroups * kGroupWarps, kSoft = 32 * kWarps, kThreads = kSoft + 32;
    static constexpr int kTile = kv4::tile_bytes(D), kStage = kGroupWarps * kTile;
    static constexpr int kStages = 190 * 1024 / kStage / kGroups * kGroups;       // a slot always belongs to the same group (see DecCfg)
    static constexpr int kMergeStride = D + 4;
    static constexpr size_t kRing = (size_t)kStages * kStage, kMerge = (size_t)kWarps * kRows * kMergeStride * 4;
    static constexpr size_t kSmem = (kRing > kMerge ? kRing : kMerge) + 128;
    static_assert(kSmem <= 220 * 1024, "shared memory");
};

template <int D, int NT>
__global__ void __launch_bounds__(Dec4Cfg<D, NT>::kThreads, 1) attn4_decode_kernel(const Params4 P) {
    using C = Dec4Cfg<D, NT>;
    constexpr int kKeys = C::kKeys, kRows = C::kRows, kGroups64 = D / 64;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[C::kStages], s_empty[C::kStages], s_tile;
    __shared__ float s_m[C::kWarps][kRows], s_l[C::kWarps][kRows], s_f[C::kWarps][kRows], s_inv[kRows];
    __shared__ int s_timeout, s_gave_up[C::kWarps];
    __shared__ Sequence s_seq;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char* ring = smem_raw;

    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) { tc::mbar_init(tc::smem_u32(&s_full[s]), 1); tc::mbar_init(tc::smem_u32(&s_empty[s]), C::kGroupWarps); }
        tc::mbar_init(tc::smem_u32(&s_tile), C::kWarps);
        tc::mbar_init_fence();
        s_timeout = 0;
    }
    const int part = (int)(blockIdx.x % (unsigned)P.splits);
    const unsigned rest = blockIdx.x / (unsigned)P.splits;
    const int h = (int)(rest % (unsigned)P.kv_heads);
    const int bt = (int)(rest / (unsigned)P.kv_heads);
    const int b = bt / P.tiles_per_seq;
    after_previous_kernel();
    if (tid == 0) s_seq = sequence(P, b);                               // read once: all warps act on the same numbers
    __syncthreads();
    let_next_kernel_start();
    const int64_t q0 = s_seq.q0, n_new = s_seq.n_new;
    const int kv_len = s_seq.kv_len;
    if (n_new <= 0) return;
    const int64_t n_rows = n_new * P.group, tiles = (n_rows + kRows - 1) / kRows;
    const int64_t ctx = kv_len - n_new;                                 // position of the first new token (negative: it sees nothing)

    int it = 0, issued = 0;                                             // stages used so far by this CTA
    int round = 0;                                                      // row tiles with keys so far: only those use the ring, and the barrier that hands it back
    for (int64_t tile = bt - (int64_t)b * P.tiles_per_seq; tile < tiles; tile += P.tiles_per_seq) {
        const int64_t r0 = tile * kRows, r1 = min(r0 + kRows, n_rows) - 1;           // first and last row
        // Row r of position p sees the keys [lo(p), p].  Positions stay below kv_len, an int.
        const auto lo = [&](int64_t p) { return P.window && p - P.window + 1 > 0 ? (int)(p - P.window + 1) : 0; };
        const int p_lo = (int)(ctx + r0 / P.group), p_hi = (int)(ctx + r1 / P.group);
        const int first = lo(p_lo), all_from = lo(p_hi);                // some row sees [first, p_hi], every row [all_from, p_lo]
        int64_t k_lo64 = (first & ~(kKeys - 1)) + part * P.split_keys;
        int64_t k_hi64 = (int64_t)p_hi + 1;
        if (part + 1 < P.splits) k_hi64 = min(k_hi64, k_lo64 + P.split_keys);
        const int n_it = k_hi64 > k_lo64 ? (int)((k_hi64 - k_lo64 + kKeys - 1) / kKeys) : 0;
        const int k_lo = n_it ? (int)k_lo64 : 0, k_hi = n_it ? (int)k_hi64 : 0;

        if (warp >= C::kWarps) {
            // ---------------- producer
            const int run_keys = min(P.page_size, kKeys);               // keys of a copy, a power of two
            const int runs = kKeys / run_keys;                          // copies of a stage
            const int steps_block = 32 / runs;                          // stages whose pages one lookup of 32 covers
            const int run = lane & (runs - 1);
            const uint32_t bytes = (uint32_t)(run_keys / 16) * C::kTile;
            const uint32_t dst = tc::smem_u32(ring) + (uint32_t)run * bytes;
            const int64_t page_tiles = P.page_size >> 4;
            // lane y: the first tile of run y % runs of stage i + y / runs, or -1 where no query sees a key of it, or its page is out of range
            const auto tile_of = [&](int i) -> int64_t {
                const int64_t key = (int64_t)k_lo + (int64_t)i * kKeys + lane * run_keys;
                if (key >= k_hi || key + run_keys <= first) return -1;
                const int64_t pg = key >> P.page_shift;
                const int64_t page = pg < P.table_width ? P.table[(int64_t)b * P.table_stride + pg] : -1;
                if (page < 0 || page >= P.n_pages) { report(P.dev_status, MATQ_ERR_PAGE); return -1; }
                return (page * P.kv_heads + h) * page_tiles + ((key & (P.page_size - 1)) >> 4);
            };
            int64_t now = -1, next = n_it > 0 ? tile_of(0) : -1;
            int in_block = 0;
            bool ok = n_it == 0 || round == 0 || tc::mbar_wait(tc::smem_u32(&s_tile), (uint32_t)(round - 1) & 1u, P.wait_cycles);
            ok = __all_sync(0xffffffffu, ok) && !P.hold;
            int s = it % C::kStages;
            uint32_t phase = (uint32_t)(it / C::kStages) & 1u;
            for (int i = 0; i < n_it && ok; ++i) {
                if (in_block == 0) {
                    now = next;
                    if (i + steps_block < n_it) next = tile_of(i + steps_block);
                }
                const int64_t t = __shfl_sync(0xffffffffu, now, in_block * runs + run);
                const bool copies = lane < runs && t >= 0;
                const int n = __popc(__ballot_sync(0xffffffffu, copies));
                ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_empty[s]), phase ^ 1u, P.wait_cycles));
                if (!ok) break;
                const uint32_t bar = tc::smem_u32(&s_full[s]);
                if (lane == 0) tc::mbar_expect_tx(bar, (uint32_t)n * bytes);
                __syncwarp();
                if (copies) bulk_load(dst + (uint32_t)s * C::kStage, P.tiles + t * C::kTile, bytes, bar);
                ++issued;
                if (++s == C::kStages) { s = 0; phase ^= 1u; }
                if (++in_block == steps_block) in_block = 0;
            }
            if (n_it > 0 && !ok) {
                if (lane == 0) *(volatile int*)&s_timeout = 1;
                break;
            }
            it += n_it;
            if (n_it > 0) ++round;
            continue;
        }

        // ---------------- consumers
        const int g = lane >> 2, q4 = lane & 3, c2 = q4 * 2;
        uint32_t qf[NT][D / 32][4];                                     // column g of the queries: operand_of_piece of elements 32 c + 8 q4 ..
        float qs[NT][2][kGroups64];                                     // sums of rows 8 nt + c2 (+ 1) per group of 64, in units of 2^(133 - e)
        float back[NT][2];                                              // 2^(126 - e) of these rows
        int see_hi[NT][2], see_lo[NT][2];                               // these rows see the keys [see_lo, see_hi]
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int64_t r = r0 + nt * 8 + g;
            const bool live = r <= r1;
            const int64_t tok = live ? r / P.group : 0;
            const __nv_bfloat16* src = P.q + (q0 + tok) * P.ldq + (int64_t)(h * P.group + (live ? (int)(r - tok * P.group) : 0)) * D + 8 * q4;
            uint4 piece[D / 32];
            uint32_t top = 0u;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                piece[c] = live ? *reinterpret_cast<const uint4*>(src + 32 * c) : make_uint4(0u, 0u, 0u, 0u);
                top = max(top, top_of_piece(piece[c]));
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = scale_exponent(top);
            float sums[kGroups64];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                float sum;
                const uint4 o = operand_of_piece(piece[c], e, sum);
                qf[nt][c][0] = o.x; qf[nt][c][1] = o.y; qf[nt][c][2] = o.z; qf[nt][c][3] = o.w;
                if (c & 1) sums[c / 2] += sum;
                else sums[c / 2] = sum;
            }
#pragma unroll
            for (int i = 0; i < kGroups64; ++i) {
                sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], 1);
                sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], 2);
#pragma unroll
                for (int w = 0; w < 2; ++w) qs[nt][w][i] = __shfl_sync(0xffffffffu, sums[i], (c2 + w) * 4);
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                back[nt][w] = exp2i(126 - __shfl_sync(0xffffffffu, e, (c2 + w) * 4));
                const int64_t re = r0 + nt * 8 + c2 + w;
                see_hi[nt][w] = re <= r1 ? (int)(ctx + re / P.group) : p_hi;
                see_lo[nt][w] = lo(see_hi[nt][w]);
            }
        }
        float o[D / 16][NT][4];                                         // 16 t: elements 32 (t / 2) + 4 g + 2 (t & 1) (+ 1 from [2] on) of rows c2, c2 + 1
        float extra[NT][2][kGroups64];                                  // sum_j p_j (low_j + 8 scale_j) over this lane's keys
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][nt][e] = 0.f;
        float m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                m[nt][w] = -INFINITY;
                l[nt][w] = 0.f;
#pragma unroll
                for (int i = 0; i < kGroups64; ++i) extra[nt][w][i] = 0.f;
            }
        const Score sc(P.scale, P.softcap);
        const int grp = warp / C::kGroupWarps, wg = warp % C::kGroupWarps;
        bool ok = true;
        for (int i = (grp + C::kGroups - it % C::kGroups) % C::kGroups; i < n_it; i += C::kGroups) {     // this group's stages
            const int u = it + i, s = u % C::kStages;
            ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_full[s]), (uint32_t)(u / C::kStages) & 1u, P.wait_cycles));
            if (!ok) break;
            const int j0 = k_lo + i * kKeys + wg * 16;                  // this warp's first key
            if (j0 < k_hi && j0 + 15 >= first) {
                const uint32_t kb = tc::smem_u32(ring) + (uint32_t)s * C::kStage + (uint32_t)wg * C::kTile, vb = kb + kv4::half_bytes(D);
                float x[NT][4];                                         // key g: rows c2, c2 + 1; key g + 8: rows c2, c2 + 1
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[nt][e] = 0.f;
#pragma unroll
                for (int c = 0; c < kGroups64; ++c) {
                    uint32_t w[4];
                    ldmatrix4(w, kb + c * 512 + lane * 16);             // keys g and g + 8 of 32 elements, then of the next 32
                    const uint32_t ga = lds32(kb + kv4::groups_at(D) + c * 64 + g * 4), gb = lds32(kb + kv4::groups_at(D) + c * 64 + 32 + g * 4);
                    float acc[NT][2][4] = {};
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const uint32_t a = w[2 * f], bb = w[2 * f + 1], a8 = a >> 8, b8 = bb >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma_bf16(acc[nt][f], a & 0x000f000fu, bb & 0x000f000fu, a & 0x00f000f0u, bb & 0x00f000f0u, qf[nt][2 * c + f][0], qf[nt][2 * c + f][1]);
                            mma_bf16(acc[nt][f], a8 & 0x000f000fu, b8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x00f000f0u, qf[nt][2 * c + f][2], qf[nt][2 * c + f][3]);
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t gr = e < 2 ? ga : gb;
                            x[nt][e] = fmaf(scale_of(gr), acc[nt][0][e] + acc[nt][1][e], fmaf(low_of(gr), qs[nt][e & 1][c], x[nt][e]));
                        }
                }
                const bool masked = j0 + 15 > p_lo || j0 < all_from;
                bool raise = false;
                uint32_t seen = 0xffffffffu;                            // bit 4 nt + e: the row sees the key
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = x[nt][e] * 128.f * back[nt][e & 1];
                        v = sc.cap2 > 0.f ? capped(v, sc) : __fmul_rn(v, sc.mul);
                        if (masked) {
                            const int j = j0 + g + (e >> 1) * 8;
                            if (j > see_hi[nt][e & 1] || j < see_lo[nt][e & 1]) { v = -INFINITY; seen &= ~(1u << (4 * nt + e)); }
                        }
                        x[nt][e] = v;
                        raise |= v > m[nt][e & 1] + kFar;               // also from -inf to anything finite
                    }
                if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = fmaxf(x[nt][e], x[nt][e + 2]);
#pragma unroll
                            for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                            if (top > m[nt][e]) {
                                const float f = ex2(m[nt][e] - top);
                                m[nt][e] = top;
                                l[nt][e] *= f;
#pragma unroll
                                for (int c = 0; c < kGroups64; ++c) extra[nt][e][c] *= f;
#pragma unroll
                                for (int t = 0; t < D / 16; ++t) { o[t][nt][e] *= f; o[t][nt][e + 2] *= f; }
                            }
                        }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[nt][e] = ex2(x[nt][e] - (m[nt][e & 1] == -INFINITY ? 0.f : m[nt][e & 1]));
                    l[nt][0] += x[nt][0] + x[nt][2];
                    l[nt][1] += x[nt][1] + x[nt][3];
                }
#pragma unroll
                for (int c = 0; c < kGroups64; ++c) {
                    const uint32_t ga = lds32(vb + kv4::groups_at(D) + c * 64 + g * 4), gb = lds32(vb + kv4::groups_at(D) + c * 64 + 32 + g * 4);
                    const float sa = scale_of(ga), sb = scale_of(gb), la = fmaf(sa, 8.f, low_of(ga)), lb = fmaf(sb, 8.f, low_of(gb));
                    uint32_t pb[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float p[4], z[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            p[e] = x[nt][e] * (e < 2 ? sa : sb);
                            z[e] = x[nt][e] * (e < 2 ? la : lb);
                            // A weight of zero does not silence what a slot holds that the row does not see.
                            if (masked && !((seen >> (4 * nt + e)) & 1u)) p[e] = z[e] = 0.f;
                        }
                        extra[nt][0][c] += z[0] + z[2];
                        extra[nt][1][c] += z[1] + z[3];
                        pb[nt][0] = transposed8x8(pack_bf16(p[0], p[1]));
                        pb[nt][1] = transposed8x8(pack_bf16(p[2], p[3]));
                    }
                    uint32_t w[4];
                    ldmatrix4t(w, vb + c * 512 + lane * 16);            // keys 2 q4 (+ 1) and 8 + 2 q4 (+ 1): elements 4 g .. of 32, then of the next 32
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
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&s_empty[s]));
        }
        it += n_it;
        // ---------------- join of the warps (their key sets are disjoint)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], w);
#pragma unroll
                for (int c = 0; c < kGroups64; ++c)
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) extra[nt][e][c] += __shfl_xor_sync(0xffffffffu, extra[nt][e][c], w);
                if (g == 0) { s_m[warp][nt * 8 + c2 + e] = m[nt][e]; s_l[warp][nt * 8 + c2 + e] = l[nt][e]; }
            }
        if (lane == 0) s_gave_up[warp] = !ok;
        asm volatile("bar.sync 1, %0;" ::"n"(C::kSoft) : "memory");
        int gave_up = 0;
#pragma unroll
        for (int w = 0; w < C::kWarps; ++w) gave_up |= s_gave_up[w];
        if (gave_up) {                                                  // written before the barrier only: the warps leave together and nothing is stored
            *(volatile int*)&s_timeout = 1;
            break;
        }
        // A row tile without keys leaves the ring alone: the producer does not wait for such tiles and may be filling it for a later one.
        float* merge = reinterpret_cast<float*>(ring);
        if (n_it > 0) {
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float z = extra[nt][e][c / 2];
                        *reinterpret_cast<float4*>(merge + (size_t)(warp * kRows + nt * 8 + c2 + e) * C::kMergeStride + 32 * c + 4 * g) =
                            make_float4(fmaf(o[2 * c][nt][e], 64.f, z), fmaf(o[2 * c][nt][2 + e], 64.f, z), fmaf(o[2 * c + 1][nt][e], 64.f, z), fmaf(o[2 * c + 1][nt][2 + e], 64.f, z));
                    }
        }
        if (tid < kRows && r0 + tid <= r1) {
            float mx = s_m[0][tid];
#pragma unroll
            for (int w = 1; w < C::kWarps; ++w) mx = fmaxf(mx, s_m[w][tid]);
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < C::kWarps; ++w) {
                // a warp without keys has m = -inf and sums of zero; all scores NaN leaves m = -inf and a sum of NaN
                const float f = mx == -INFINITY ? 1.f : ex2(s_m[w][tid] - mx);
                s_f[w][tid] = f;
                sum += s_l[w][tid] * f;
            }
            const int64_t rr = r0 + tid, tok = rr / P.group;
            s_inv[tid] = ctx + tok >= 0 ? 1.f / sum : -1.f;             // negative: the row sees no key
            if (P.splits > 1)
                P.part_ml[(int64_t)part * (P.T * P.q_heads) + (q0 + tok) * P.q_heads + h * P.group + (rr - tok * P.group)] = make_float2(mx, sum);
        }
        asm volatile("bar.sync 1, %0;" ::"n"(C::kSoft) : "memory");
        for (int i = tid; i < kRows * (D / 4); i += C::kSoft) {
            const int r = i / (D / 4), c = (i % (D / 4)) * 4;
            const int64_t rr = r0 + r;
            if (rr > r1) break;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
            if (n_it > 0) {
#pragma unroll
                for (int w = 0; w < C::kWarps; ++w) {
                    const float4 v = *reinterpret_cast<const float4*>(merge + (size_t)(w * kRows + r) * C::kMergeStride + c);
                    const float f = s_f[w][r];
                    a.x = fmaf(v.x, f, a.x); a.y = fmaf(v.y, f, a.y); a.z = fmaf(v.z, f, a.z); a.w = fmaf(v.w, f, a.w);
                }
            }
            const int64_t tok = rr / P.group;
            const int head = h * P.group + (int)(rr - tok * P.group);
            if (P.splits > 1) {
                if (n_it > 0) *reinterpret_cast<float4*>(P.part_o + ((int64_t)part * (P.T * P.q_heads) + (q0 + tok) * P.q_heads + head) * D + c) = a;
            } else {
                const float inv = s_inv[r];
                *reinterpret_cast<uint2*>(P.out + (q0 + tok) * P.ldo + (int64_t)head * D + c) =
                    inv < 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync 1, %0;" ::"n"(C::kSoft) : "memory");
        if (n_it > 0 && lane == 0) tc::mbar_arrive(tc::smem_u32(&s_tile));
    }
    // No copy may be in flight when the CTA ends.  Consumers that gave up may have left some: the producer waits for what it issued.
    if (warp >= C::kWarps)
        for (int u = max(0, issued - C::kStages); u < issued; ++u)
            tc::mbar_wait(tc::smem_u32(&s_full[u % C::kStages]), (uint32_t)(u / C::kStages) & 1u, P.wait_cycles);
    __syncthreads();
    if (tid == 0 && s_timeout) report(P.dev_status, MATQ_ERR_TIMEOUT);
}

}  // namespace attn
}  // namespace matq
