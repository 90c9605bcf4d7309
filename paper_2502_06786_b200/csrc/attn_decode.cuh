// Attention of few query rows over the paged cache: a CTA takes 8 or 16 rows (token, head of the group) of one key head and a part of the
// key range.  Every key and value is read once for the whole group, so the cache's bytes are what bounds it.
//
// Two producer warps, one for keys and one for values, fill a ring that takes the SM's shared memory (one box per page and 64 columns, 128-byte
// swizzle, one lane per box; the page numbers are fetched 32 at a time, a block ahead).  A lane's box costs its warp about 65 cycles: with pages of
// 16 keys one warp for both kept up with two thirds of HBM only (32768 keys of 8 x 128: 28.8 us a pass against 18.9 with pages of 64).  Consumer warps in groups that take the stages in turn work on 16 keys each:
//   S^T = K Q^T    (mma.sync m16n8k16: keys are the rows, queries the 8 columns),
//   O^T += V^T P^T (the head dimension is the rows).
// Queries as the narrow operand: the other way round 16 rows would be multiplied for the 4 or 2 of a group, and O would take twice the registers.
// The row maximum is a reference only (see kFar): the lanes that share a row meet only when it moves.  The warps meet at the end, where their partial results are joined in shared memory.
//
// 64 sequences of up to 8000 keys, 16/8 heads of 256: 322 us = 6.8 TB/s.  One over 32768 keys, 8 heads of 128: 134 MB in 29.4 us with the start and the join.
#pragma once

#include "attn_common.cuh"

namespace matq {
namespace attn {

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// NT: columns of 8 query rows
template <int D, int NT>
struct DecCfg {
    static constexpr int kRows = 8 * NT;
    static constexpr int kKeys = D == 256 ? 32 : 64;                    // keys per stage
    static constexpr int kGroupWarps = kKeys / 16;
    // Warps: enough that the chains of their units (about a thousand cycles each) keep up with HBM, few enough that accumulators and queries stay in registers.
    static constexpr int kGroups = NT == 1 || D == 256 ? 3 : 2;
    static constexpr int kWarps = kGroups * kGroupWarps, kSoft = 32 * kWarps, kThreads = kSoft + 64;
    static constexpr int kPanels = D / 64;                              // 64-column panels of 128-byte rows
    static constexpr int kTile = kKeys * D * 2;                         // bytes of a stage's keys (or values)
    static constexpr int kStages = 192 * 1024 / (2 * kTile);            // 12, 6, 6
    // A slot of the ring always belongs to the same group.  Otherwise a group would meet a slot only every other phase, and its parity
    // wait could pass on the phase before the other group's.
    static_assert(kStages % kGroups == 0, "see above");
    static constexpr int kMergeStride = D + 4;                          // floats: the four lanes of a quad store 8 banks apart
    static constexpr size_t kRing = (size_t)kStages * 2 * kTile, kMerge = (size_t)kWarps * kRows * kMergeStride * 4;
    static constexpr size_t kSmem = (kRing > kMerge ? kRing : kMerge) + 1024;         // the join at the end reuses the ring
};

template <int D, int NT>
__global__ void __launch_bounds__(DecCfg<D, NT>::kThreads, 1)
attn_decode_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Params P) {
    using C = DecCfg<D, NT>;
    constexpr int kKeys = C::kKeys, kRows = C::kRows;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[C::kStages], s_empty[C::kStages], s_tile;
    __shared__ float s_m[C::kWarps][kRows], s_l[C::kWarps][kRows], s_f[C::kWarps][kRows], s_inv[kRows];
    __shared__ int s_timeout, s_gave_up[C::kWarps];
    __shared__ Sequence s_seq;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char* ring = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);

    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) { tc::mbar_init(tc::smem_u32(&s_full[s]), 2); tc::mbar_init(tc::smem_u32(&s_empty[s]), C::kGroupWarps); }
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
    // Without a window the first keys of a part are known before the sequence's bounds are: their pages' numbers are looked up side by side with them.
    int early_page = -1;
    if (warp >= C::kWarps && !P.window) {
        const int64_t pg = ((int64_t)part * P.split_keys + (int64_t)lane * min(P.page_size, kKeys)) >> P.page_shift;
        if (pg < P.table_width) early_page = P.table[(int64_t)b * P.table_stride + pg];
    }
    if (tid == 0) s_seq = sequence(P, b);                               // read once: all warps act on the same numbers
    __syncthreads();
    let_next_kernel_start();
    const int64_t q0 = s_seq.q0, n_new = s_seq.n_new;
    const int kv_len = s_seq.kv_len;
    if (n_new <= 0) return;
    const int64_t n_rows = n_new * P.group, tiles = (n_rows + kRows - 1) / kRows;
    const int64_t ctx = kv_len - n_new;                                 // position of the first new token (negative: it sees nothing)

    int it = 0, issued = 0;                                             // stages used so far by this CTA
    int round = 0;                                                      // tiles with keys so far: only those use the ring, and the barrier that hands it back
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
            // ---------------- producers: keys (v = 0) and values (v = 1)
            const int v = warp - C::kWarps;
            const CUtensorMap* tm = v ? &tm_v : &tm_k;
            const int rows_box = min(P.page_size, kKeys);               // rows of a box, a power of two
            const int runs = kKeys / rows_box, boxes = runs * C::kPanels;
            const int steps_block = 32 / runs;                          // stages whose boxes' rows one lookup of 32 covers
            const int run = lane & (runs - 1), x = (lane / runs) * 64;  // this lane's box of a stage
            const uint32_t dst = tc::smem_u32(ring) + (uint32_t)v * C::kTile + (uint32_t)(x >> 6) * (kKeys * 128) + (uint32_t)run * rows_box * 128;
            const auto rows_of = [&](int i) {                           // lane y: the row of run y % runs of stage i + y / runs
                const int64_t key = (int64_t)k_lo + (int64_t)i * kKeys + lane * rows_box;
                return key < k_hi ? cache_row(P, b, h, key, rows_box, first, kv_len) : (int)(P.n_pages * P.kv_heads * P.page_size);
            };
            int rows_now = 0, rows_next = 0, in_block = 0;
            if (n_it > 0) {
                if (P.window) {
                    rows_next = rows_of(0);
                } else {
                    const int64_t key = (int64_t)k_lo + lane * rows_box;
                    rows_next = key < k_hi ? page_row(P, h, key, early_page) : (int)(P.n_pages * P.kv_heads * P.page_size);
                }
            }
            bool ok = n_it == 0 || round == 0 || tc::mbar_wait(tc::smem_u32(&s_tile), (uint32_t)(round - 1) & 1u, P.wait_cycles);
            ok = __all_sync(0xffffffffu, ok) && !P.hold;
            int s = it % C::kStages;
            uint32_t phase = (uint32_t)(it / C::kStages) & 1u;
            for (int i = 0; i < n_it && ok; ++i) {
                if (in_block == 0) {
                    rows_now = rows_next;
                    if (i + steps_block < n_it) rows_next = rows_of(i + steps_block);
                }
                const int y = __shfl_sync(0xffffffffu, rows_now, in_block * runs + run);
                ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_empty[s]), phase ^ 1u, P.wait_cycles));
                if (!ok) break;
                const uint32_t bar = tc::smem_u32(&s_full[s]);
                if (lane == 0) tc::mbar_expect_tx(bar, C::kTile);       // the phase cannot end before this arrival, whichever copy comes first
                if (lane < boxes) tc::tma_load_2d(dst + (uint32_t)(s * 2) * C::kTile, tm, x, y, bar);
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
        const int g = lane >> 2, c2 = (lane & 3) * 2, mi = lane >> 3, mr = lane & 7;
        uint32_t qf[NT][D / 16][2];                                     // column g of the queries
        int see_hi[NT][2], see_lo[NT][2];                               // rows 8 nt + c2 (+ 1) see the keys [see_lo, see_hi]
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int64_t r = r0 + nt * 8 + g;
            const bool live = r <= r1;
            const int64_t tok = live ? r / P.group : 0;
            const __nv_bfloat16* src = P.q + (q0 + tok) * P.ldq + (int64_t)(h * P.group + (live ? (int)(r - tok * P.group) : 0)) * D;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                qf[nt][ks][0] = live ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + c2) : 0u;
                qf[nt][ks][1] = live ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + 8 + c2) : 0u;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int64_t re = r0 + nt * 8 + c2 + e;
                see_hi[nt][e] = re <= r1 ? (int)(ctx + re / P.group) : p_hi;
                see_lo[nt][e] = lo(see_hi[nt][e]);
            }
        }
        float o[D / 16][NT][4];                                         // (d, row): rows d = 16 t + g (+ 8), columns as see_hi
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][nt][e] = 0.f;
        float m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) { m[nt][0] = m[nt][1] = -INFINITY; l[nt][0] = l[nt][1] = 0.f; }
        const Score sc(P.scale, P.softcap);
        const int grp = warp / C::kGroupWarps, wg = warp % C::kGroupWarps;
        bool ok = true;
        for (int i = (grp + C::kGroups - it % C::kGroups) % C::kGroups; i < n_it; i += C::kGroups) {     // this group's stages
            const int u = it + i, s = u % C::kStages;
            ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_full[s]), (uint32_t)(u / C::kStages) & 1u, P.wait_cycles));
            if (!ok) break;
            const int j0 = k_lo + i * kKeys + wg * 16;                  // this warp's first key
            if (j0 < k_hi && j0 + 15 >= first) {
                const uint32_t kb = tc::smem_u32(ring) + (uint32_t)(s * 2) * C::kTile + (uint32_t)(wg * 16) * 128;
                const uint32_t vb = kb + C::kTile;
                float sv[NT][2][4] = {};                                // two chains per column of rows
                {
                    const int key = (mi & 1) * 8 + mr;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        uint32_t a[4];
                        ldsm4(a, kb + (uint32_t)(ks / 4) * (kKeys * 128) + key * 128 + ((((2 * ks + (mi >> 1)) & 7) ^ mr) << 4));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(sv[nt][ks & 1], a, qf[nt][ks][0], qf[nt][ks][1]);
                    }
                }
                const bool masked = j0 + 15 > p_lo || j0 < all_from;
                float x[NT][4];                                         // key g: rows c2, c2 + 1; key g + 8: rows c2, c2 + 1
                bool raise = false, near = true;
                if (sc.cap2 > 0.f) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) near &= fabsf((sv[nt][0][e] + sv[nt][1][e]) * sc.tmul) <= kTanhMax;
                    near = __all_sync(0xffffffffu, near);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = sv[nt][0][e] + sv[nt][1][e];
                        v = sc.cap2 > 0.f ? near ? capped_near(v * sc.tmul, sc.cap2) : capped(v, sc) : __fmul_rn(v, sc.mul);
                        if (masked) {
                            const int j = j0 + g + (e >> 1) * 8;
                            if (j > see_hi[nt][e & 1] || j < see_lo[nt][e & 1]) v = -INFINITY;
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
                                for (int t = 0; t < D / 16; ++t) { o[t][nt][e] *= f; o[t][nt][e + 2] *= f; }
                            }
                        }
                }
                uint32_t pb[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = ex2(x[nt][e] - (m[nt][e & 1] == -INFINITY ? 0.f : m[nt][e & 1]));
                    l[nt][0] += p[0] + p[2];
                    l[nt][1] += p[1] + p[3];
                    pb[nt][0] = transpose8x8(pack_bf16(p[0], p[1]));
                    pb[nt][1] = transpose8x8(pack_bf16(p[2], p[3]));
                }
                if (masked) {
                    // A weight of zero does not silence a NaN or Inf: values that no row sees become zero, and non-finite ones that only some
                    // rows see are taken out of the tile and added to those rows by hand.
                    const int j = j0 + (lane & 15);
                    const bool unseen = j > p_hi || j < first, all = j <= p_lo && j >= all_from;
                    bool bad = false;
                    if (!all) {
                        for (int ch = lane >> 4; ch < D / 8; ch += 2) {
                            const uint32_t at = vb + (uint32_t)(ch >> 3) * (kKeys * 128) + (lane & 15) * 128 + (((ch & 7) ^ (lane & 7)) << 4);
                            if (unseen) {
                                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at), "r"(0) : "memory");
                            } else {
                                uint32_t w[4];
                                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
#pragma unroll
                                for (int v = 0; v < 4; ++v) bad |= nonfinite_bf16(w[v]) || nonfinite_bf16(w[v] >> 16);
                            }
                        }
                    }
                    uint32_t bads = __ballot_sync(0xffffffffu, bad);
                    bads = (bads | (bads >> 16)) & 0xffffu;
                    while (bads) {
                        const int key = __ffs(bads) - 1, jb = j0 + key;
                        bads &= bads - 1;
#pragma unroll
                        for (int t = 0; t < D / 16; ++t)
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const int ch = 2 * t + half;            // column ch * 8 + g
                                const uint32_t at = vb + (uint32_t)(ch >> 3) * (kKeys * 128) + key * 128 + (((ch & 7) ^ (key & 7)) << 4) + g * 2;
                                uint16_t w;
                                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(at) : "memory");
                                const bool here = nonfinite_bf16(w);
                                const float add = bf16_bits_to_float(w);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int e = 0; e < 2; ++e)
                                        if (here && jb <= see_hi[nt][e] && jb >= see_lo[nt][e]) o[t][nt][2 * half + e] += add;
                                __syncwarp();
                                if (here && c2 == 0) asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"((uint16_t)0) : "memory");
                            }
                    }
                    __syncwarp();
                }
                {
                    const int key = (mi >> 1) * 8 + mr;
#pragma unroll
                    for (int t = 0; t < D / 16; ++t) {
                        uint32_t a[4];
                        ldsm4t(a, vb + (uint32_t)(t / 4) * (kKeys * 128) + key * 128 + ((((2 * t + (mi & 1)) & 7) ^ mr) << 4));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(o[t][nt], a, pb[nt][0], pb[nt][1]);
                    }
                }
                if (masked) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // this warp's stores before the next copy's
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
        // A tile without keys leaves the ring alone: the producers do not wait for such tiles and may be filling it for a later one.
        float* merge = reinterpret_cast<float*>(ring);
        if (n_it > 0) {
#pragma unroll
            for (int t = 0; t < D / 16; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        merge[(size_t)(warp * kRows + nt * 8 + c2 + (e & 1)) * C::kMergeStride + t * 16 + g + (e >> 1) * 8] = o[t][nt][e];
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
        for (int x = tid; x < kRows * (D / 4); x += C::kSoft) {
            const int r = x / (D / 4), c = (x % (D / 4)) * 4;
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
    // No copy may be in flight when the CTA ends.  Consumers that gave up may have left some: the producers wait for what they issued (each for
    // the whole stage; should the other have stopped before it, the wait ends at its limit, by when the copies have long landed).
    if (warp >= C::kWarps)
        for (int u = max(0, issued - C::kStages); u < issued; ++u)
            tc::mbar_wait(tc::smem_u32(&s_full[u % C::kStages]), (uint32_t)(u / C::kStages) & 1u, P.wait_cycles);
    __syncthreads();
    if (tid == 0 && s_timeout) report(P.dev_status, MATQ_ERR_TIMEOUT);
}

}  // namespace attn
}  // namespace matq
