// Attention of few query rows over the paged cache: a CTA takes 16 rows (token, head of the group) of one key head and a part of the
// key range.  Every key and value is read once for the whole group, so the cache's bytes are what bounds it.
//
// A producer warp brings 64 keys and values per stage into a ring (one box per page and 64 columns, 128-byte swizzle, one lane per box,
// so that the page numbers of a stage are fetched side by side).  Eight consumer warps in two groups that take the stages in turn, 16 keys per
// warp: scores by mma.sync m16n8k16, a running maximum and sum per row, and the product with the values into 16 x D fp32 accumulators in
// registers.  The warps meet only at the end, where their partial results are joined in shared memory.
// One CTA per SM: a unit of 16 keys is a chain of some thousand cycles in its warp, so the warps have to be eight, and the ring takes the rest of the
// SM's shared memory (about 190 KB in flight).
#pragma once

#include "attn_common.cuh"

namespace matq {
namespace attn {

constexpr int kDecRows = 16, kDecKeys = 64, kDecWarps = 8, kDecThreads = 32 * (kDecWarps + 1);

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D>
struct DecCfg {
    static constexpr int kPanels = D / 64;                              // 64-column panels of 128-byte rows
    static constexpr int kTile = kDecKeys * D * 2;                      // bytes of 64 keys (or values)
    // Even, so that a slot of the ring always belongs to the same group of consumer warps.  With an odd count a group would meet a slot only every
    // other phase, and its parity wait could pass on the phase before the other group's.
    static constexpr int kStages = D == 256 ? 2 : 192 * 1024 / (2 * kTile);
    static_assert(kStages % 2 == 0, "see above");
    static constexpr bool kQShared = D == 256;                          // 64 registers of queries beside 128 of accumulators would not fit
    static constexpr int kQStride = D * 2 + 16;                         // bytes; rows 16 bytes apart modulo the banks
    static constexpr int kMergeStride = D + 8;                          // floats; rows 32 bytes apart modulo the banks
    static constexpr size_t kRing = (size_t)kStages * 2 * kTile, kMerge = (size_t)kDecWarps * kDecRows * kMergeStride * 4;
    static constexpr size_t kSmem = (kRing > kMerge ? kRing : kMerge) + 1024;         // the join at the end reuses the ring
};

template <int D>
__global__ void __launch_bounds__(kDecThreads, 1)
attn_decode_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Params P) {
    using C = DecCfg<D>;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[C::kStages], s_empty[C::kStages], s_tile;
    __shared__ float s_m[kDecWarps][kDecRows], s_l[kDecWarps][kDecRows];
    __shared__ int s_timeout, s_gave_up[kDecWarps];
    __shared__ Sequence s_seq;
    __shared__ __align__(16) unsigned char s_q[C::kQShared ? kDecRows * C::kQStride : 16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char* ring = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);

    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) { tc::mbar_init(tc::smem_u32(&s_full[s]), 1); tc::mbar_init(tc::smem_u32(&s_empty[s]), kDecWarps / 2); }
        tc::mbar_init(tc::smem_u32(&s_tile), kDecWarps);
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
    const int64_t n_rows = n_new * P.group, tiles = (n_rows + kDecRows - 1) / kDecRows;
    const int64_t ctx = kv_len - n_new;                                 // position of the first new token (negative: it sees nothing)

    int it = 0, issued = 0;                                             // stages used so far by this CTA
    int round = 0;
    for (int64_t tile = bt - (int64_t)b * P.tiles_per_seq; tile < tiles; tile += P.tiles_per_seq, ++round) {
        const int64_t r0 = tile * kDecRows, r1 = min(r0 + kDecRows, n_rows) - 1;     // first and last row
        // Row r of position p sees the keys [lo(p), p].  Positions stay below kv_len, an int.
        const auto lo = [&](int64_t p) { return P.window && p - P.window + 1 > 0 ? (int)(p - P.window + 1) : 0; };
        const int p_lo = (int)(ctx + r0 / P.group), p_hi = (int)(ctx + r1 / P.group);
        const int first = lo(p_lo), all_from = lo(p_hi);                // some row sees [first, p_hi], every row [all_from, p_lo]
        int64_t k_lo64 = (first & ~(kDecKeys - 1)) + part * P.split_keys;
        int64_t k_hi64 = (int64_t)p_hi + 1;
        if (part + 1 < P.splits) k_hi64 = min(k_hi64, k_lo64 + P.split_keys);
        const int n_it = k_hi64 > k_lo64 ? (int)((k_hi64 - k_lo64 + kDecKeys - 1) / kDecKeys) : 0;
        const int k_lo = n_it ? (int)k_lo64 : 0, k_hi = n_it ? (int)k_hi64 : 0;

        if (warp == kDecWarps) {
            // ---------------- producer
            if (round > 0 && !tc::mbar_wait(tc::smem_u32(&s_tile), (uint32_t)(round - 1) & 1u, P.wait_cycles)) { s_timeout = 1; break; }
            const int rows_box = min(P.page_size, kDecKeys);            // rows of a box
            const int runs = kDecKeys / rows_box, boxes = runs * C::kPanels * 2;
            bool ok = true;
            int next_row = lane < runs && n_it > 0 ? cache_row(P, b, h, (int64_t)k_lo + lane * rows_box, rows_box, first, kv_len) : 0;
            for (int i = 0; i < n_it && ok; ++i) {
                const int s = (it + i) % C::kStages, row = next_row;    // the page of the next stage is looked up while this one waits
                if (lane < runs && i + 1 < n_it) next_row = cache_row(P, b, h, (int64_t)k_lo + (i + 1) * kDecKeys + lane * rows_box, rows_box, first, kv_len);
                ok = tc::mbar_wait(tc::smem_u32(&s_empty[s]), ((uint32_t)((it + i) / C::kStages) & 1u) ^ 1u, P.wait_cycles);
                if (!__all_sync(0xffffffffu, ok) || P.hold) { ok = false; break; }
                const uint32_t bar = tc::smem_u32(&s_full[s]);
                if (lane == 0) tc::mbar_expect_tx(bar, 2 * C::kTile);
                __syncwarp();
                for (int x0 = 0; x0 < boxes; x0 += 32) {
                    const int x = x0 + lane;
                    const int run = x % runs;
                    const int y = __shfl_sync(0xffffffffu, row, run);
                    if (x < boxes) {
                        const int which = x / runs, panel = which % C::kPanels, v = which / C::kPanels;
                        const uint32_t dst = tc::smem_u32(ring) + (uint32_t)(s * 2 + v) * C::kTile + (uint32_t)panel * (kDecKeys * 128) + (uint32_t)run * rows_box * 128;
                        tc::tma_load_2d(dst, v ? &tm_v : &tm_k, panel * 64, y, bar);
                    }
                }
                issued = it + i + 1;
            }
            if (!ok) {
                if (lane == 0) *(volatile int*)&s_timeout = 1;
                break;
            }
            it += n_it;
            continue;
        }

        // ---------------- consumers
        const int g = lane >> 2, c2 = (lane & 3) * 2;
        uint32_t qf[C::kQShared ? 1 : D / 16][4];
        int see_hi[2], see_lo[2];                                       // rows g and g + 8 see the keys [see_lo, see_hi]
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t r = r0 + g + 8 * i;
            const bool live = r <= r1;
            const int64_t tok = live ? r / P.group : 0;
            see_hi[i] = live ? (int)(ctx + tok) : p_hi;
            see_lo[i] = lo(see_hi[i]);
            const __nv_bfloat16* src = P.q + (q0 + tok) * P.ldq + (int64_t)(h * P.group + (live ? (int)(r - tok * P.group) : 0)) * D;
            if constexpr (!C::kQShared) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    qf[ks][i] = live ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + c2) : 0u;
                    qf[ks][2 + i] = live ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + 8 + c2) : 0u;
                }
            }
        }
        if constexpr (C::kQShared) {
            for (int x = tid; x < kDecRows * (D / 8); x += kDecWarps * 32) {
                const int rr = x / (D / 8), ch = x % (D / 8);
                const int64_t r = r0 + rr, tok = r <= r1 ? r / P.group : 0;
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (r <= r1) v = *reinterpret_cast<const uint4*>(P.q + (q0 + tok) * P.ldq + (int64_t)(h * P.group + (int)(r - tok * P.group)) * D + ch * 8);
                *reinterpret_cast<uint4*>(s_q + rr * C::kQStride + ch * 16) = v;
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
        }
        float o[D / 8][4];
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        const Score sc(P.scale, P.softcap);
        bool ok = true;
        for (int i = (it ^ (warp >> 2)) & 1; i < n_it; i += 2) {        // this group's stages
            const int s = (it + i) % C::kStages;
            ok = tc::mbar_wait(tc::smem_u32(&s_full[s]), (uint32_t)((it + i) / C::kStages) & 1u, P.wait_cycles);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            const int j0 = k_lo + i * kDecKeys + (warp & 3) * 16;       // this warp's first key
            if (j0 < k_hi && j0 + 15 >= first) {
                const uint32_t kb = tc::smem_u32(ring) + (uint32_t)(s * 2) * C::kTile + (uint32_t)((warp & 3) * 16) * 128;
                const uint32_t vb = kb + C::kTile;
                float sv[2][4] = {};
                const int mi = lane >> 3, mr = lane & 7;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t r[4];
                    const int key = (mi >> 1) * 8 + mr, ch = (2 * ks + (mi & 1)) & 7;
                    ldsm4(r, kb + (uint32_t)(ks / 4) * (kDecKeys * 128) + key * 128 + ((ch ^ (key & 7)) << 4));
                    if constexpr (C::kQShared) {
                        uint32_t a[4];
                        ldsm4(a, tc::smem_u32(s_q) + ((mi & 1) * 8 + mr) * C::kQStride + ks * 32 + (mi >> 1) * 16);
                        mma16816(sv[0], a, r[0], r[1]);
                        mma16816(sv[1], a, r[2], r[3]);
                    } else {
                        mma16816(sv[0], qf[ks], r[0], r[1]);
                        mma16816(sv[1], qf[ks], r[2], r[3]);
                    }
                }
                const bool masked = j0 + 15 > p_lo || j0 < all_from;
                // fold scale and cap in; hide what a row does not see
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = sc.cap2 > 0.f ? capped(sv[nt][e], sc.mul, sc.cap2) : sv[nt][e] * sc.mul;
                        if (masked) {
                            const int j = j0 + nt * 8 + c2 + (e & 1);
                            if (j > see_hi[e >> 1] || j < see_lo[e >> 1]) x = -INFINITY;
                        }
                        sv[nt][e] = x;
                    }
                float f[2];
#pragma unroll
                for (int i2 = 0; i2 < 2; ++i2) {
                    float mx = fmaxf(fmaxf(sv[0][2 * i2], sv[0][2 * i2 + 1]), fmaxf(sv[1][2 * i2], sv[1][2 * i2 + 1]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    mx = fmaxf(mx, m[i2]);
                    const float use = mx == -INFINITY ? 0.f : mx;
                    f[i2] = ex2(m[i2] - use);
                    m[i2] = mx;
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) {
                        sv[nt][2 * i2] = ex2(sv[nt][2 * i2] - use);
                        sv[nt][2 * i2 + 1] = ex2(sv[nt][2 * i2 + 1] - use);
                    }
                    l[i2] = fmaf(l[i2], f[i2], (sv[0][2 * i2] + sv[0][2 * i2 + 1]) + (sv[1][2 * i2] + sv[1][2 * i2 + 1]));
                }
                if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) { o[j][0] *= f[0]; o[j][1] *= f[0]; o[j][2] *= f[1]; o[j][3] *= f[1]; }
                }
                if (masked) {
                    // A weight of zero does not silence a NaN or Inf: values that no row sees become zero, and non-finite ones that only some
                    // rows see are taken out of the tile and added to those rows by hand.
                    const int j = j0 + (lane & 15);
                    const bool unseen = j > p_hi || j < first, all = j <= p_lo && j >= all_from;
                    bool bad = false;
                    if (!all) {
                        for (int ch = lane >> 4; ch < D / 8; ch += 2) {
                            const uint32_t at = vb + (uint32_t)(ch >> 3) * (kDecKeys * 128) + (lane & 15) * 128 + (((ch & 7) ^ (lane & 7)) << 4);
                            if (unseen) {
                                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at), "r"(0) : "memory");
                            } else {
                                uint32_t w[4];
                                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
#pragma unroll
                                for (int u = 0; u < 4; ++u) bad |= nonfinite_bf16(w[u]) || nonfinite_bf16(w[u] >> 16);
                            }
                        }
                    }
                    uint32_t bads = __ballot_sync(0xffffffffu, bad);
                    bads = (bads | (bads >> 16)) & 0xffffu;
                    while (bads) {
                        const int key = __ffs(bads) - 1;
                        bads &= bads - 1;
                        const int jb = j0 + key;
                        const bool see0 = jb <= see_hi[0] && jb >= see_lo[0], see1 = jb <= see_hi[1] && jb >= see_lo[1];
#pragma unroll
                        for (int nt = 0; nt < D / 8; ++nt) {
                            const uint32_t at = vb + (uint32_t)(nt >> 3) * (kDecKeys * 128) + key * 128 + (((nt & 7) ^ (key & 7)) << 4) + c2 * 2;
                            uint32_t w;
                            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
                            const float a = __uint_as_float(w << 16), c = __uint_as_float(w & 0xffff0000u);
                            const bool na = nonfinite_bf16(w), nc = nonfinite_bf16(w >> 16);
                            if (na && see0) o[nt][0] += a;
                            if (nc && see0) o[nt][1] += c;
                            if (na && see1) o[nt][2] += a;
                            if (nc && see1) o[nt][3] += c;
                            __syncwarp();
                            if (g == 0) {                              // only what is not finite leaves the tile
                                if (na) w &= 0xffff0000u;
                                if (nc) w &= 0x0000ffffu;
                                asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(w) : "memory");
                            }
                        }
                    }
                    __syncwarp();
                }
                const uint32_t pa[4] = {pack_bf16(sv[0][0], sv[0][1]), pack_bf16(sv[0][2], sv[0][3]), pack_bf16(sv[1][0], sv[1][1]), pack_bf16(sv[1][2], sv[1][3])};
#pragma unroll
                for (int t2 = 0; t2 < D / 16; ++t2) {
                    uint32_t r[4];
                    const int key = (mi & 1) * 8 + mr, ch = (2 * t2 + (mi >> 1)) & 7;
                    ldsm4t(r, vb + (uint32_t)(t2 / 4) * (kDecKeys * 128) + key * 128 + ((ch ^ (key & 7)) << 4));
                    mma16816(o[2 * t2], pa, r[0], r[1]);
                    mma16816(o[2 * t2 + 1], pa, r[2], r[3]);
                }
                if (masked) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // this warp's stores before the next copy's
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&s_empty[s]));
        }
        it += n_it;
        // ---------------- join of the warps (their key sets are disjoint)
        if (lane == 0) s_gave_up[warp] = !ok;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            if ((lane & 3) == 0) { s_m[warp][g + 8 * i] = m[i]; s_l[warp][g + 8 * i] = l[i]; }
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        int gave_up = 0;
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) gave_up |= s_gave_up[w];
        if (gave_up) {                                                   // written before the barrier only: the warps leave together and nothing is stored
            *(volatile int*)&s_timeout = 1;
            break;
        }
        const auto row_max = [&](int r) {
            float mx = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kDecWarps; ++w) mx = fmaxf(mx, s_m[w][r]);
            return mx;
        };
        float* merge = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = g + 8 * i;
            const float mx = row_max(r);
            const float f = mx == -INFINITY ? 0.f : ex2(m[i] - mx);
#pragma unroll
            for (int j = 0; j < D / 8; ++j)
                *reinterpret_cast<float2*>(merge + (size_t)(warp * kDecRows + r) * C::kMergeStride + j * 8 + c2) = make_float2(o[j][2 * i] * f, o[j][2 * i + 1] * f);
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        {
            const int r = tid >> 4, c0 = tid & 15;                      // sixteen threads per row, four columns at a time
            const int64_t rr = r0 + r;
            if (rr <= r1) {
                const float mx = row_max(r);
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < kDecWarps; ++w) sum += mx == -INFINITY ? s_l[w][r] : s_l[w][r] * ex2(s_m[w][r] - mx);
                const int64_t tok = rr / P.group, row = (q0 + tok) * P.q_heads + h * P.group + (rr - tok * P.group);
                const bool any = ctx + tok >= 0;                        // the row sees a key (its own, at least)
                const float inv = any ? 1.f / sum : 0.f;
                if (P.splits > 1 && c0 == 0) P.part_ml[(int64_t)part * (P.T * P.q_heads) + row] = make_float2(mx, sum);
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const int c = j * 64 + c0 * 4;
                    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int w = 0; w < kDecWarps; ++w) {
                        const float4 v = *reinterpret_cast<const float4*>(merge + (size_t)(w * kDecRows + r) * C::kMergeStride + c);
                        a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
                    }
                    if (P.splits > 1) {
                        if (n_it > 0) *reinterpret_cast<float4*>(P.part_o + ((int64_t)part * (P.T * P.q_heads) + row) * D + c) = a;
                    } else {
                        const uint2 w2 = any ? make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv)) : make_uint2(0u, 0u);
                        *reinterpret_cast<uint2*>(P.out + (q0 + tok) * P.ldo + (int64_t)(h * P.group + (int)(rr - tok * P.group)) * D + c) = w2;
                    }
                }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (lane == 0) tc::mbar_arrive(tc::smem_u32(&s_tile));
    }
    if (warp == kDecWarps)                                              // no copy may be in flight when the CTA ends, whatever became of its consumers
        for (int i = max(0, issued - C::kStages); i < issued; ++i)
            tc::mbar_wait(tc::smem_u32(&s_full[i % C::kStages]), (uint32_t)(i / C::kStages) & 1u, P.wait_cycles);
    __syncthreads();
    if (tid == 0 && s_timeout) report(P.dev_status, MATQ_ERR_TIMEOUT);
}

}  // namespace attn
}  // namespace matq
