// Attention of a chunk of new tokens over the paged cache on the fifth-generation tensor cores.
//
// A query tile is 128 accumulator rows: floor(128 / group) tokens times the heads of one key head's group, so that a key is read once for the
// whole group.  A CTA takes kTiles such tiles and walks the keys that they see, kKeys at a time:
//   warps 8, 9         producers: queries once and keys; values; a ring each (one box per page and 64 columns, 128-byte swizzle);
//   warps 10, 11       one thread each issues S = Q K^T and O += P V (tcgen05.mma, accumulators and P in tensor memory): one takes the scores
//                      and the other the products, so that a wait of the one, 250 cycles even on a barrier that has been arrived on, leaves the tensor
//                      cores the other's work.  With two tiles the first warp issues all of it: a tile's next scores have to follow the product that
//                      reads P in the same place, and the other tile's work fills the waits (a warp per tile was slower).
//   warps 0 .. 7       softmax, one thread per row (two, with half of the keys each, when there is one tile): S from tensor memory, exponentials,
//                      P back over S as bf16.
// P takes the place of S: the product with V that reads it is issued before the scores that overwrite it.  The row maximum is a reference only (see kFar).
// D <= 128: two tiles, whose softmax and tensor work alternate.  One tile (D = 256, or few rows): two S buffers, so that the scores of the next
// keys are computed while the present ones are exponentiated.  A step is 128 keys, also at D = 256 (with steps of 64 the
// softmax's fixed part, about 1300 cycles of latencies, came twice as often: 500 tokens over 6011 at 16/8 x 256 heads 70 us in the kernel).
//
// Bound: 8192 tokens over 16384 keys, 32/8 heads of 128: 1.43 ms = 1150 TFLOP/s (1.65 ms in a long run, at the power cap).  A step of two tiles takes about
// 3500 cycles for 2048 of products: a tile's chain is its softmax pass 1500, the store of P 170, two hand-overs of some 250 and its products 1024, and two
// tiles cover each other's products but not all of the rest.  500 over 6511 at 16/8 x 256, with the cap: 54 us, 2.4 us a step, of which
// the copies alone need 1.6 (128 KB at 80 GB/s; every SM reads all keys and values of its tile from the L2), the products 1.05.
#pragma once

#include <type_traits>

#include <cuda_fp16.h>

#include "attn_common.cuh"

namespace matq {
namespace attn {

// A reference of kLarge or more is not the sum of the old one and a distance to it, whose rounding would pass many exponents, but the row's largest score itself, looked
// up again; and it is taken off the scores before they are multiplied (fused) or, with the cap, off rounded values.
// The cap's tanh with one coefficient less than in capped(): relative error 2.6e-6, so at most 1e-3 of an exponent for caps up to kShortCap, half of what a weight's
// rounding to bf16 is.  Larger caps, and scores past kTanhMax of one, go score by score: 500 tokens over 6511, 16/8 heads of 256, 58 us below and 110 above.
constexpr float kShortCap = 512.f, kShort1 = -0.333190745f, kShort2 = 0.130864184f, kShort3 = -0.0413877882f;
constexpr int kMaxMasked = 16;          // tiles at a range's ends that some row does not see in full

template <int D, int TILES>
struct ChunkCfg {
    static constexpr int kTiles = TILES;
    static_assert(TILES == 1 || (TILES == 2 && D <= 128), "two accumulators and their scores must fit 512 columns");
    static constexpr int kKeys = 128;                                   // keys of a step
    // Ring stages of a step.  Keys come as column panels (all keys of the step, half of the columns), so that a product is 128 keys wide; values as rows, half
    // of the keys each.  (Keys as rows too, and products 64 wide, read Q from shared memory twice as often: 500 tokens over 6511, 16/8 heads of 256, 61 us
    // instead of 55.  Stages of a quarter: keys the same, values 64 us, a stage's wait and commit being what they cost.)
    static constexpr int kSub = D == 256 ? 2 : 1, kStageKeys = kKeys / kSub;         // kStageKeys: of a stage of values
    static constexpr int kPanels = D / 64;
    static constexpr int kQBytes = 128 * D * 2;                         // one query tile
    static constexpr int kKvBytes = kKeys * D * 2 / kSub;               // the keys, or the values, of a stage
    static constexpr int kStagesK = D == 64 ? 4 : 3, kStagesV = D == 64 ? 4 : TILES * D == 128 ? 3 : 2;
    static constexpr int kSoft = 256;                                   // softmax threads: one per row of two tiles, two per row of one
    static constexpr int kCols = kKeys * TILES / 2;                     // keys of a step per softmax thread
    static constexpr int kThreads = kSoft + 128;
    static constexpr int kTmemO = 256;                                  // first column of the output accumulators; S starts at column 0
    static constexpr size_t kSmem = (size_t)kTiles * kQBytes + (size_t)(kStagesK + kStagesV) * kKvBytes + 1024;
};

__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* d) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 ::"r"(d[0]), "r"(d[1]), "r"(d[2]), "r"(d[3]), "r"(d[4]), "r"(d[5]), "r"(d[6]), "r"(d[7]),
                   "r"(d[8]), "r"(d[9]), "r"(d[10]), "r"(d[11]), "r"(d[12]), "r"(d[13]), "r"(d[14]), "r"(d[15]),
                   "r"(d[16]), "r"(d[17]), "r"(d[18]), "r"(d[19]), "r"(d[20]), "r"(d[21]), "r"(d[22]), "r"(d[23]),
                   "r"(d[24]), "r"(d[25]), "r"(d[26]), "r"(d[27]), "r"(d[28]), "r"(d[29]), "r"(d[30]), "r"(d[31]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* d) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::"r"(d[0]), "r"(d[1]), "r"(d[2]), "r"(d[3]), "r"(d[4]), "r"(d[5]), "r"(d[6]), "r"(d[7]),
                   "r"(d[8]), "r"(d[9]), "r"(d[10]), "r"(d[11]), "r"(d[12]), "r"(d[13]), "r"(d[14]), "r"(d[15]), "r"(addr) : "memory");
}
// 32 bytes, a whole sector: in one store where the address allows it (a thread's row lies apart from its neighbours', so that smaller stores cost a
// transaction each all the same)
__device__ __forceinline__ void store32(void* p, const uint32_t* v, bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}
// D = fp32, A = B = bf16 (or fp16), 128 rows
__device__ __forceinline__ constexpr uint32_t idesc_16bit(int n, bool b_mn_major, bool half) {
    return (1u << 4) | (half ? 0u : (1u << 7) | (1u << 10)) | (b_mn_major ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}

// The largest of a thread's scores in columns lo .. hi of its COLS (with the cap: its exponent).  Rare, and kept out of the loop over the keys, whose code it would spread.
template <bool CAP, int COLS>
__device__ __noinline__ float largest_score(uint32_t addr, int lo, int hi, Score sc) {
    float best = -INFINITY;
#pragma unroll 1
    for (int c = 0; c < COLS; c += 32) {
        uint32_t v[32];
        tc::tmem_ld32(addr + c, v);
        tc::tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; ++e)
            if (c + e >= lo && c + e <= hi) best = fmaxf(best, CAP ? capped(__uint_as_float(v[e]), sc) : __uint_as_float(v[e]));
    }
    return best;
}
// The same where every row sees every key.
template <bool CAP, int COLS>
__device__ __forceinline__ float largest_of_all(uint32_t addr, const Score& sc) {
    float best = -INFINITY;
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        uint32_t v[32];
        tc::tmem_ld32(addr + c, v);
        tc::tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; e += 2) best = max3(best, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
    }
    return CAP ? capped(best, sc) : best;
}
// Takes a large reference off the scores.
template <int COLS>
__device__ __noinline__ void lift_scores(uint32_t addr, float by) {
#pragma unroll 1
    for (int c = 0; c < COLS; c += 32) {
        uint32_t v[32];
        tc::tmem_ld32(addr + c, v);
        tc::tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) - by);
        tmem_st32(addr + c, v);
    }
    tc::tmem_wait_st();
}

// HALF: queries, keys and values are fp16, scaled by powers of two (Params::q_scale and the others; see attn4.cu), and so are the weights, whose range has to hold both
// weights above the reference and what is far below it: a prompt's first key may draw nearly all of a row's weight and leave the rest to thousands.  So a row's
// first reference is its largest score in the first step that shows it a key, never 0, and stands for a weight of 2^kRoomHalf: weights down to 2^-18 of the largest keep
// all their bits and the rest are off by 2^-29 of it at most, and scores up to 11 (in exponents of two) above the reference fit.  It is looked up before the first step's
// pass (4096 tokens over 8192, 32/8 heads of 128, 453 us, 2048 over themselves 67.4; with that pass done twice 455 and 69.6; with 0 for a reference where the scores lie
// around it 451 and 66.5, but weights below 2^-19 of the largest became zero).  References from kLarge on are taken as they are.
constexpr float kFarHalf = 15.f, kRoomHalf = 4.f;
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// CAP: with the cap on the scores
template <int D, int TILES, bool CAP, bool HALF = false>
__global__ void __launch_bounds__(ChunkCfg<D, TILES>::kThreads, 1)
attn_chunk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Params P) {
    using C = ChunkCfg<D, TILES>;
    constexpr int kKeys = C::kKeys, kStageKeys = C::kStageKeys, kSub = C::kSub;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_kfull[C::kStagesK], s_kempty[C::kStagesK], s_vfull[C::kStagesV], s_vempty[C::kStagesV], s_q, s_score[2], s_prob[2], s_pv[2], s_out, s_read;
    __shared__ uint32_t s_tmem;
    __shared__ Sequence s_seq;
    __shared__ int s_timeout, s_any_bad, s_bad_key[kMaxMasked];
    __shared__ uint32_t s_bad[kMaxMasked][kKeys / 32];
    __shared__ float s_half[2][128];                                    // one tile: what the two threads of a row tell one another
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char* smem = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);
    unsigned char* ring_k = smem + C::kTiles * C::kQBytes;
    unsigned char* ring_v = ring_k + C::kStagesK * C::kKvBytes;
    constexpr int kWarpK = C::kSoft / 32, kWarpV = kWarpK + 1, kWarpMma = kWarpK + 2;      // and kWarpMma + 1

    if (tid == 0) {
        for (int s = 0; s < C::kStagesK; ++s) { tc::mbar_init(tc::smem_u32(&s_kfull[s]), 1); tc::mbar_init(tc::smem_u32(&s_kempty[s]), 1); }
        for (int s = 0; s < C::kStagesV; ++s) { tc::mbar_init(tc::smem_u32(&s_vfull[s]), 1); tc::mbar_init(tc::smem_u32(&s_vempty[s]), 1); }
        tc::mbar_init(tc::smem_u32(&s_q), 1);
        for (int t = 0; t < 2; ++t) { tc::mbar_init(tc::smem_u32(&s_score[t]), 1); tc::mbar_init(tc::smem_u32(&s_prob[t]), C::kSoft / C::kTiles); }
        for (int x = 0; x < 2; ++x) tc::mbar_init(tc::smem_u32(&s_pv[x]), 1);
        tc::mbar_init(tc::smem_u32(&s_out), 1);
        tc::mbar_init(tc::smem_u32(&s_read), C::kSoft);
        tc::mbar_init_fence();
        s_timeout = 0;
    }
    if (warp == kWarpMma) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&s_tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const int part = (int)(blockIdx.x % (unsigned)P.splits);
    const unsigned rest = blockIdx.x / (unsigned)P.splits;
    const int h = (int)(rest % (unsigned)P.kv_heads);
    const int bt = (int)(rest / (unsigned)P.kv_heads);
    const int b = bt / P.tiles_per_seq;
    after_previous_kernel();
    if (tid == 0) s_seq = sequence(P, b);                               // read once: all warps act on the same numbers
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    let_next_kernel_start();
    const uint32_t tmem = s_tmem;
    const int64_t q0 = s_seq.q0, n_new = s_seq.n_new;
    const int kv_len = s_seq.kv_len;
    const int tok_tile = 128 / P.group, rows_tile = tok_tile * P.group;  // tokens and used rows of a query tile
    const int tok_cta = tok_tile * C::kTiles;
    const int64_t tiles = n_new > 0 ? (n_new + tok_cta - 1) / tok_cta : 0;
    const int64_t ctx = kv_len - n_new;
    const auto lo = [&](int64_t p) { return P.window && p - P.window + 1 > 0 ? (int)(p - P.window + 1) : 0; };

    int it = 0, issued = 0, q_issued = 0;                               // steps over keys so far; copies issued (producer)
    int round = 0;                                                      // tiles with keys so far
    // the last tiles see the most keys: they are started first
    for (int64_t tile = P.tiles_per_seq - 1 - (bt - (int64_t)b * P.tiles_per_seq); tile < tiles; tile += P.tiles_per_seq) {
        const int64_t t0 = tile * tok_cta, t1 = min(t0 + tok_cta, n_new) - 1;      // first and last token
        const int p_lo = (int)(ctx + t0), p_hi = (int)(ctx + t1);
        const int first = lo(p_lo), all_from = lo(p_hi);                // some row sees [first, p_hi], every row [all_from, p_lo]
        const int64_t k_lo64 = (int64_t)(first & ~(kKeys - 1)) + part * P.split_keys;
        int64_t k_hi64 = (int64_t)p_hi + 1;
        if (part + 1 < P.splits) k_hi64 = min(k_hi64, k_lo64 + P.split_keys);
        const int n_it = k_hi64 > k_lo64 ? (int)((k_hi64 - k_lo64 + kKeys - 1) / kKeys) : 0;
        const int k_lo = n_it ? (int)k_lo64 : 0;
        const auto is_masked = [&](int j0) { return j0 + kKeys - 1 > p_lo || j0 < all_from; };

        if (warp == kWarpK || warp == kWarpV) {
            // ---------------- producers
            const bool v = warp == kWarpV;
            const CUtensorMap* tm = v ? &tm_v : &tm_k;
            const int stages = v ? C::kStagesV : C::kStagesK;
            const int keys = v ? kStageKeys : kKeys, panels = v ? C::kPanels : C::kPanels / kSub;
            const int rows_box = min(P.page_size, keys), runs = keys / rows_box, boxes = runs * panels;       // powers of two, 32 boxes at most
            const int run = lane & (runs - 1), x = (lane / runs) * 64;  // this lane's box of a step
            const uint32_t dst = tc::smem_u32(v ? ring_v : ring_k) + (uint32_t)(x >> 6) * (keys * 128) + (uint32_t)run * rows_box * 128;
            const uint32_t full = tc::smem_u32(v ? s_vfull : s_kfull), empty = tc::smem_u32(v ? s_vempty : s_kempty);
            const auto row_of = [&](int i) { return cache_row(P, b, h, (int64_t)k_lo + (int64_t)i * keys + run * rows_box, rows_box, first, kv_len); };
            int next_row = n_it > 0 ? row_of(0) : 0;                    // a stage's pages are looked up while the one before waits, the first while the queries are fetched
            bool ok = true;
            if (n_it > 0 && !v) {
                if (round > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_out), (uint32_t)(round - 1) & 1u, P.wait_cycles));
                if (ok && !P.hold && lane == 0) {
                    q_issued = round + 1;
                    tc::mbar_expect_tx(tc::smem_u32(&s_q), C::kTiles * C::kPanels * rows_tile * 128);
                    for (int t = 0; t < C::kTiles; ++t)
                        for (int p = 0; p < C::kPanels; ++p)
                            tc::tma_load_3d(tc::smem_u32(smem) + t * C::kQBytes + p * (128 * 128), &tm_q, p * 64, h * P.group,
                                            (int)(q0 + t0 + t * tok_tile), tc::smem_u32(&s_q));
                }
            }
            int s = kSub * it % stages, row = 0;
            uint32_t phase = (uint32_t)(kSub * it / stages) & 1u;
            for (int i = 0; i < kSub * n_it && ok; ++i) {
                const int part_i = v ? 0 : i % kSub, i_row = v ? i : i / kSub;          // keys: the stage's columns; the rows are the step's
                if (part_i == 0) {
                    row = next_row;
                    if (i + (v ? 1 : kSub) < kSub * n_it) next_row = row_of(i_row + 1);
                }
                ok = __all_sync(0xffffffffu, tc::mbar_wait(empty + 8 * s, phase ^ 1u, P.wait_cycles)) && !P.hold;
                if (!ok) break;
                if (lane == 0) tc::mbar_expect_tx(full + 8 * s, C::kKvBytes);   // the phase cannot end before this arrival, whichever copy comes first
                if (lane < boxes) tc::tma_load_2d(dst + (uint32_t)s * C::kKvBytes, tm, x + part_i * (D / kSub), row, full + 8 * s);
                ++issued;
                if (++s == stages) { s = 0; phase ^= 1u; }
            }
            if (!ok) {
                if (lane == 0) *(volatile int*)&s_timeout = 1;
                break;
            }
        } else if (warp >= kWarpMma) {
            // ---------------- tensor cores
            if (n_it > 0) {
                const int who = __shfl_sync(0xffffffffu, warp, 0) - kWarpMma;          // (uniform, and known to be)
                const uint32_t leader = tc::elect_one();
                bool ok = tc::warp_wait(tc::smem_u32(&s_q), (uint32_t)round & 1u, P.wait_cycles);
                // Descriptors and slots are stepped, not computed: a product of 16 keys or columns takes 64 cycles, about what a handful of dependent
                // instructions takes.
                const uint64_t q_desc = tc::sw128_desc(tc::smem_u32(smem)), k_desc = tc::sw128_desc(tc::smem_u32(ring_k)),
                               v_desc = tc::sw128_desc(tc::smem_u32(ring_v), kStageKeys * 128, 1024);
                const uint32_t kfull = tc::smem_u32(s_kfull), kempty = tc::smem_u32(s_kempty), vfull = tc::smem_u32(s_vfull), vempty = tc::smem_u32(s_vempty);
                int ks = kSub * it % C::kStagesK, vs = kSub * it % C::kStagesV;         // slots of the next keys and values
                uint32_t kp = (uint32_t)(kSub * it / C::kStagesK) & 1u, vp = (uint32_t)(kSub * it / C::kStagesV) & 1u;
                const auto next_k = [&] { if (++ks == C::kStagesK) { ks = 0; kp ^= 1u; } };
                const auto next_v = [&] { if (++vs == C::kStagesV) { vs = 0; vp ^= 1u; } };
                const auto scores = [&](int t, int sub) {               // S_t += Q_t K^T for a stage's columns
                    const uint64_t qd = q_desc + (uint64_t)(C::kTiles == 2 ? t * (C::kQBytes >> 4) : 0) + (uint64_t)(sub * (C::kPanels / kSub) * (128 * 128 >> 4));
                    const uint64_t kd = k_desc + (uint64_t)(ks * (C::kKvBytes >> 4));
#pragma unroll
                    for (int x = 0; x < D / kSub / 16; ++x)
                        MATQ_TC_MMA(1, "f16", tmem + t * kKeys, qd + (uint64_t)((x / 4) * (128 * 128 >> 4) + (x & 3) * 2), kd + (uint64_t)((x / 4) * (kKeys * 128 >> 4) + (x & 3) * 2),
                                    idesc_16bit(kKeys, false, HALF), (sub > 0 || x > 0) ? 1u : 0u, leader);
                    if (sub == kSub - 1) tc::tc_commit(tc::smem_u32(&s_score[t]), leader);
                };
                const auto product = [&](int t, int i, int sub) {       // O_t += P_t V for a stage's keys
                    const uint64_t vd = v_desc + (uint64_t)(vs * (C::kKvBytes >> 4));
                    const uint32_t d = tmem + C::kTmemO + (C::kTiles == 2 ? t * D : 0);
#pragma unroll
                    for (int x = 0; x < kStageKeys / 16; ++x)
                        MATQ_TC_MMA_TMEM_A(1, "f16", d, tmem + t * kKeys + sub * (kStageKeys / 2) + x * 8, vd + (uint64_t)(x * (2048 >> 4)), idesc_16bit(D, true, HALF),
                                           (i > 0 || sub > 0 || x > 0) ? 1u : 0u, leader);
                };
                const auto first_read = [&](int i) { return i > 0 || round == 0 || tc::warp_wait(tc::smem_u32(&s_read), (uint32_t)(round - 1) & 1u, P.wait_cycles); };
                const auto keys_there = [&] { return ok = ok && tc::warp_wait(kfull + 8 * ks, kp, P.wait_cycles); };
                const auto free_keys = [&] { tc::tc_commit(kempty + 8 * ks, leader); next_k(); };
                const auto weights_there = [&](int t, uint32_t parity) { return ok = ok && tc::warp_wait(tc::smem_u32(&s_prob[t]), parity, P.wait_cycles); };
                const auto values_there = [&](int i) { return ok = ok && tc::warp_wait(vfull + 8 * vs, vp, P.wait_cycles) && first_read(i); };
                const auto free_values = [&] { tc::tc_commit(vempty + 8 * vs, leader); next_v(); };
                if (C::kTiles == 2) {
                    // The scores that overwrite P are issued behind the product that reads it, by the same thread.
                    if (who == 0 && keys_there()) {
                        tc::fence_after();
                        scores(0, 0);
                        scores(1, 0);
                        free_keys();
                        for (int i = 0; i < n_it; ++i) {
                            const uint32_t parity = (uint32_t)(it + i) & 1u;
                            const bool more = i + 1 < n_it;
                            if (!values_there(i) || (more && !keys_there()) || !weights_there(0, parity)) break;
                            tc::fence_after();
                            product(0, i, 0);
                            if (more) scores(0, 0);
                            if (!weights_there(1, parity)) break;
                            tc::fence_after();
                            product(1, i, 0);
                            free_values();
                            if (more) { scores(1, 0); free_keys(); }
                        }
                    }
                } else if (who == 0) {
                    for (int i = 0; i < n_it && ok; ++i) {
                        // The product that read this buffer's last P is over.  (The first two of a tile: queries arrive after the tile before has ended.)
                        if (i >= 2) ok = tc::warp_wait(tc::smem_u32(&s_pv[(it + i) & 1]), (uint32_t)((it + i - 2) >> 1) & 1u, P.wait_cycles);
                        for (int sub = 0; sub < kSub && keys_there(); ++sub) {
                            tc::fence_after();
                            scores((it + i) & 1, sub);
                            free_keys();
                        }
                    }
                } else {
                    for (int i = 0; i < n_it; ++i) {
                        if (!weights_there((it + i) & 1, (uint32_t)((it + i) >> 1) & 1u)) break;
                        for (int sub = 0; sub < kSub && values_there(i); ++sub) {
                            tc::fence_after();
                            product((it + i) & 1, i, sub);
                            free_values();
                        }
                        if (!ok) break;
                        tc::tc_commit(tc::smem_u32(&s_pv[(it + i) & 1]), leader);
                    }
                }
                if (!ok) { *(volatile int*)&s_timeout = 1; __threadfence_block(); }
                if (who == (C::kTiles == 2 ? 0 : 1)) tc::tc_commit(tc::smem_u32(&s_out), leader);    // also when giving up: nobody waits for longer than its limit
            }
            __syncwarp();
        } else {
            // ---------------- softmax: thread = row of tile t (with one tile: half of the keys of a row, and half of its outputs)
            const int part_of = warp >> 2, t = C::kTiles == 2 ? part_of : 0, r = tid & 127;
            const int col0 = C::kTiles == 2 ? 0 : part_of * C::kCols;
            const int64_t tok = t0 + t * tok_tile + r / P.group;
            const bool live = r < rows_tile && tok < n_new;
            const int see_hi = live ? (int)(ctx + tok) : -1, see_lo = live ? lo(see_hi) : 0;
            const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
            const uint32_t o_addr = lane_addr + C::kTmemO + t * D;
            float score_scale = P.scale, value_scale = 1.f;
            if constexpr (HALF) {
                if (live) score_scale = P.scale * P.q_scale[(q0 + tok) * P.q_heads + h * P.group + r % P.group] * P.k_scale[(int64_t)b * P.kv_heads + h];
                value_scale = P.v_scale[(int64_t)b * P.kv_heads + h];
            }
            constexpr float kUp = HALF ? kFarHalf : kFar;
            const auto room = [](float reference) { return HALF && fabsf(reference) < kLarge ? kRoomHalf : 0.f; };
            const Score sc(score_scale, P.softcap);
            const float tanh1 = kShort1 * sc.cap2, tanh2 = kShort2 * sc.cap2, tanh3 = kShort3 * sc.cap2, t_max = P.softcap <= kShortCap ? kTanhMax : -1.f;   // with the cap
            // The reference is kept as a score; with the cap, as an exponent.  (HALF: the factors of a row of zeros and of keys of zero make products of zero, and a unit of
            // zero would make NaN of a reference of -inf; exponents are the same with the smallest number.)
            const float unit = CAP ? 1.f : HALF ? fmaxf(sc.mul, 0x1p-126f) : sc.mul;
            float m = -INFINITY, l = 0.f;
            bool ok = true;
            int masked_no = 0;
            if (tid == 0) s_any_bad = 0;
            for (int x = tid; x < kMaxMasked * (kKeys / 32); x += C::kSoft) (&s_bad[0][0])[x] = 0;
            asm volatile("bar.sync 1, %0;" ::"n"(C::kSoft) : "memory");
            constexpr int kOCols = D * C::kTiles / 2;                   // outputs of this thread: columns o_col ..
            const int o_col = C::kTiles == 2 ? 0 : part_of * kOCols;
            const auto soft_any = [&](bool mine) {                       // whether some softmax thread says so; a barrier of them all
                int any;
                asm volatile("{ .reg .pred p, q; setp.ne.b32 p, %1, 0; barrier.cta.red.or.pred q, 2, %2, p; selp.b32 %0, 1, 0, q; }"
                             : "=r"(any) : "r"((int)mine), "n"(C::kSoft) : "memory");
                return any != 0;
            };
            const auto rescale = [&](float f) {
#pragma unroll 1
                for (int c = 0; c < kOCols; c += 32) {
                    uint32_t o[32];
                    tc::tmem_ld32(o_addr + o_col + c, o);
                    tc::tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                    tmem_st32(o_addr + o_col + c, o);
                }
            };

            for (int i = 0; i < n_it; ++i) {
                const int gi = it + i, j0 = k_lo + i * kKeys;
                const int which = C::kTiles == 2 ? t : gi & 1;
                const uint32_t par = C::kTiles == 2 ? (uint32_t)gi & 1u : (uint32_t)(gi >> 1) & 1u;
                if (ok) ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_score[which]), par, P.wait_cycles)) && *(volatile int*)&s_timeout == 0;
                ok = __all_sync(0xffffffffu, ok);
                const bool masked = is_masked(j0);
                const uint32_t s_addr = lane_addr + which * kKeys + col0;
                float top = -INFINITY, use, off;
                uint64_t sum2[2];
                uint32_t pk[C::kCols / 2];
                // HALF: the first reference, looked up before the first step's pass (rows that it shows no key get theirs as they move one).
                if (HALF && i == 0) {
                    if (ok) {
                        tc::fence_after();
                        float best = masked ? largest_score<CAP, C::kCols>(s_addr, see_lo - j0 - col0, see_hi - j0 - col0, sc) : largest_of_all<CAP, C::kCols>(s_addr, sc);
                        if (see_hi >= 0) m = best;
                    }
                    if (C::kTiles == 1) {
                        s_half[part_of][r] = m;
                        asm volatile("bar.sync 2, %0;" ::"n"(C::kSoft) : "memory");
                        m = fmaxf(s_half[0][r], s_half[1][r]);
                    }
                }
                // One pass: exponents x = score - reference, their maximum, 2^x, its sum, bf16.  Should x exceed kFar somewhere the reference moves and
                // the pass is done again; otherwise the maximum costs no second look at the scores.
                const auto pass = [&](auto hide) {
                    top = -INFINITY;
                    sum2[0] = sum2[1] = 0;
                    uint32_t sr[2][32];
                    tc::tmem_ld32(s_addr, sr[0]);
                    const uint64_t neg = pair(off, off), mul = pair(sc.mul, sc.mul);
#pragma unroll
                    for (int c = 0; c < C::kCols; c += 32) {
                        uint32_t* v = sr[(c >> 5) & 1];
                        tc::tmem_wait_ld();
                        if (c + 32 < C::kCols) tc::tmem_ld32(s_addr + c + 32, sr[((c >> 5) + 1) & 1]);
                        if constexpr (CAP) {
                            float big = 0.f;
#pragma unroll
                            for (int e = 0; e < 32; e += 2) big = max3(big, fabsf(__uint_as_float(v[e])), fabsf(__uint_as_float(v[e + 1])));
                            if (__any_sync(0xffffffffu, see_hi >= 0 && !(big * sc.tmul <= t_max))) {       // some score of a query is past the polynomial's range
                                if (t_max < 0.f) {
#pragma unroll
                                    for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(capped(__uint_as_float(v[e]), sc) + off);
                                } else {
                                    // Scores in the polynomial's range get what it gives them below: no score depends on its neighbours, nor on what
                                    // the cache holds where nobody looks.
#pragma unroll
                                    for (int e = 0; e < 32; ++e) {
                                        const float s = __uint_as_float(v[e]), t = s * sc.tmul, u = t * t;
                                        v[e] = __float_as_uint(fabsf(t) <= kTanhMax ? fmaf(t, fmaf(fmaf(fmaf(u, tanh3, tanh2), u, tanh1), u, sc.cap2), off) : capped_far(s, sc) + off);
                                    }
                                }
                            } else {
                                const uint64_t tm2 = pair(sc.tmul, sc.tmul);
#pragma unroll
                                for (int e = 0; e < 32; e += 2) {
                                    const uint64_t t2 = mul2(pair(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), tm2), u2 = mul2(t2, t2);
                                    uint64_t p2 = fma2(u2, pair(tanh3, tanh3), pair(tanh2, tanh2));
                                    p2 = fma2(p2, u2, pair(tanh1, tanh1));
                                    p2 = fma2(p2, u2, pair(sc.cap2, sc.cap2));
                                    float x, y;
                                    unpair(fma2(t2, p2, neg), x, y);
                                    v[e] = __float_as_uint(x);
                                    v[e + 1] = __float_as_uint(y);
                                }
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float x, y;
                            if (CAP) {
                                x = __uint_as_float(v[e]);
                                y = __uint_as_float(v[e + 1]);
                            } else {
                                unpair(fma2(pair(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), mul, neg), x, y);
                            }
                            if (hide) {
                                const int j = j0 + col0 + c + e;
                                if (j > see_hi || j < see_lo) x = -INFINITY;
                                if (j + 1 > see_hi || j + 1 < see_lo) y = -INFINITY;
                            }
                            top = max3(top, x, y);
                            x = ex2(x);
                            y = ex2(y);
                            sum2[(e >> 1) & 1] = add2(sum2[(e >> 1) & 1], pair(x, y));
                            pk[(c + e) / 2] = HALF ? pack_f16(x, y) : pack_bf16(x, y);
                        }
                    }
                };
                // A row without a reference (m = -inf) takes 0 for one if its largest score is not far from it, as ordinary scores are not: then its first
                // step is not done twice (but see HALF).  A row with a large one always has its scores looked at once more.
                // (Rows of the tile that stand for no query hold whatever shared memory held: they ask for nothing.)
                bool lifted = false;
                const auto wants = [&] {
                    return ok && see_hi >= 0 && (top > kUp || (m == -INFINITY && (HALF || top < -kFar) && top > -INFINITY) || (!lifted && fabsf(use) >= kLarge));
                };
                if (ok) tc::fence_after();
                for (int attempt = 0; attempt < 3; ++attempt) {         // the second suffices: nothing lies far above a reference that was just moved
                    use = m == -INFINITY ? 0.f : m * unit;
                    off = (!CAP && lifted && fabsf(use) >= kLarge ? 0.f : -use) + room(use);
                    if (ok) {
                        if (masked) pass(std::true_type{});
                        else pass(std::false_type{});
                    }
                    bool raise = wants();
                    if (C::kTiles == 1) {
                        // The two threads of a row move together, and all scores are read before any P is written.  (Every warp passes these barriers, also
                        // one that gave up.)
                        if (!soft_any(raise || (m == -INFINITY && top > -INFINITY))) break;
                        s_half[part_of][r] = top;
                        asm volatile("bar.sync 2, %0;" ::"n"(C::kSoft) : "memory");
                        top = fmaxf(s_half[0][r], s_half[1][r]);
                        raise = wants();
                        if (m == -INFINITY && top > -INFINITY && !raise) m = 0.f;
                        if (__builtin_expect(!soft_any(raise), 1)) break;
                        if (ok && i > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_pv[(gi - 1) & 1]), (uint32_t)((gi - 1) >> 1) & 1u, P.wait_cycles));
                    } else {
                        if (m == -INFINITY && top > -INFINITY && !raise) m = 0.f;
                        if (__builtin_expect(!__any_sync(0xffffffffu, raise), 1)) break;
                    }
                    float ref = (use + (top - room(use))) / unit, next = ref * unit;          // the new reference as it is kept, and as an exponent
                    const bool large = !lifted && raise && (fabsf(use) >= kLarge || fabsf(next) >= kLarge);
                    if (__builtin_expect(C::kTiles == 1 ? soft_any(large) : __any_sync(0xffffffffu, large), 0)) {
                        float best = ok ? largest_score<CAP, C::kCols>(s_addr, see_lo - j0 - col0, see_hi - j0 - col0, sc) : -INFINITY;
                        if (C::kTiles == 1) {
                            s_half[part_of][r] = best;
                            asm volatile("bar.sync 2, %0;" ::"n"(C::kSoft) : "memory");
                            best = fmaxf(s_half[0][r], s_half[1][r]);
                        }
                        if (large) {
                            ref = best;
                            next = best * unit;
                            raise = best > -INFINITY && (m == -INFINITY || next - use > kUp);
                        }
                        if (!CAP && ok) lift_scores<C::kCols>(s_addr, raise ? (fabsf(next) >= kLarge ? ref : 0.f) : fabsf(use) >= kLarge ? m : 0.f);
                        lifted = true;
                    }
                    // O holds the steps before this one.  Their last product is over: with one tile that was waited for, with two the scores' arrival says so.
                    const float f = raise ? ex2(m * unit - next + (room(next) - room(m * unit))) : 1.f;
                    if (raise) m = ref;
                    l *= f;
                    if (ok && i > 0) {
                        tc::fence_after();
                        rescale(f);
                    }
                }
                if (ok) {
                    float a, d;
                    unpair(add2(sum2[0], sum2[1]), a, d);
                    l += a + d;
                    const uint32_t p_addr = lane_addr + which * kKeys + col0 / 2;
#pragma unroll
                    for (int c = 0; c < C::kCols / 2; c += 16) tmem_st16(p_addr + c, pk + c);
                    tc::tmem_wait_st();
                }
                if (masked) {
                    // A weight of zero does not silence a NaN or Inf.  Values that no row sees become zero; non-finite ones that only some rows
                    // see leave the tile, and those rows get them at the end.  Every thread looks at one key, all or half of it.
                    // A slot's use before this one has to be known to be over, or the parity wait could pass a phase early.  With one stage per step that use is
                    // two or more steps back, whose product these scores were issued behind; with two it is the last step's, whose product is waited for.
                    static_assert(C::kStagesV >= 2 && (kSub == 1 || C::kStagesV == kSub), "see above");
                    if (kSub > 1 && ok && i > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_pv[(gi - 1) & 1]), (uint32_t)((gi - 1) >> 1) & 1u, P.wait_cycles));
                    for (int sub = 0; sub < kSub && ok; ++sub) {
                        const int u = kSub * gi + sub;
                        ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_vfull[u % C::kStagesV]), (uint32_t)(u / C::kStagesV) & 1u, P.wait_cycles));
                    }
                    if (ok) {
                        constexpr uint32_t kExponent = HALF ? 0x7c007c00u : 0x7f807f80u;         // of Inf and NaN
                        constexpr int kShare = C::kSoft / kKeys;         // threads per key: 2
                        const int key = tid % kKeys, j = j0 + key;
                        const bool unseen = j > p_hi || j < first, all = j <= p_lo && j >= all_from;
                        const uint32_t vb = tc::smem_u32(ring_v) + (uint32_t)((kSub * gi + key / kStageKeys) % C::kStagesV) * C::kKvBytes + (key % kStageKeys) * 128;
                        bool bad = false;
                        if (!all) {
                            constexpr int kAtOnce = D / 8 / kShare < 8 ? D / 8 / kShare : 8;       // pieces of 16 bytes requested together
                            const auto at = [&](int ch) { return vb + (uint32_t)(ch >> 3) * (kStageKeys * 128) + (((ch & 7) ^ (key & 7)) << 4); };
                            for (int ch0 = tid / kKeys; ch0 < D / 8; ch0 += kAtOnce * kShare) {
                                uint32_t w[kAtOnce][4];
#pragma unroll
                                for (int x = 0; x < kAtOnce; ++x) {
                                    if (unseen) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at(ch0 + x * kShare)), "r"(0) : "memory");
                                    else asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[x][0]), "=r"(w[x][1]), "=r"(w[x][2]), "=r"(w[x][3]) : "r"(at(ch0 + x * kShare)) : "memory");
                                }
                                if (unseen) continue;
#pragma unroll
                                for (int x = 0; x < kAtOnce; ++x) {
                                    uint32_t hit = 0;
#pragma unroll
                                    for (int e = 0; e < 4; ++e) hit |= __vcmpeq2(w[x][e] & kExponent, kExponent);
                                    if (hit) {
#pragma unroll
                                        for (int e = 0; e < 4; ++e) w[x][e] &= ~__vcmpeq2(w[x][e] & kExponent, kExponent);
                                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at(ch0 + x * kShare)), "r"(w[x][0]), "r"(w[x][1]), "r"(w[x][2]), "r"(w[x][3]) : "memory");
                                        bad = true;
                                    }
                                }
                            }
                        }
                        if (bad && masked_no < kMaxMasked) {
                            atomicOr(&s_bad[masked_no][key >> 5], 1u << (key & 31));
                            s_any_bad = 1;
                        }
                        if (tid == 0 && masked_no < kMaxMasked) s_bad_key[masked_no] = j0;
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    ++masked_no;
                    asm volatile("bar.sync 1, %0;" ::"n"(C::kSoft) : "memory");     // both tiles' products read the mended values
                }
                tc::fence_before();
                tc::mbar_arrive(tc::smem_u32(&s_prob[which]));
            }

            // ---------------- outputs
            // (Also after giving up: no product may be in flight when tensor memory is given back.)
            if (n_it > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_out), (uint32_t)round & 1u, P.wait_cycles)) && ok && *(volatile int*)&s_timeout == 0;
            ok = __all_sync(0xffffffffu, ok);
            tc::fence_after();
            const int64_t row = (q0 + tok) * P.q_heads + h * P.group + r % P.group;
            const bool any = see_hi >= 0;
            if (C::kTiles == 1) {
                s_half[part_of][r] = l;
                asm volatile("bar.sync 2, %0;" ::"n"(C::kSoft) : "memory");
                l = s_half[0][r] + s_half[1][r];
            }
            const float inv = any ? 1.f / l : 0.f;
            if (!ok) *(volatile int*)&s_timeout = 1;
            if (ok && live && P.splits > 1 && o_col == 0) P.part_ml[(int64_t)part * (P.T * P.q_heads) + row] = make_float2(m * unit - room(m * unit), l);
            if (ok && !(P.splits > 1 && n_it == 0)) {
#pragma unroll 1
                for (int c = o_col; c < o_col + kOCols; c += 32) {
                    uint32_t o[32];
                    if (n_it > 0) {
                        tc::tmem_ld32(o_addr + c, o);
                        tc::tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0u;
                    }
                    if (s_any_bad && live) {
                        for (int x = 0; x < min(masked_no, kMaxMasked); ++x)
                            for (int key = 0; key < kKeys; ++key) {
                                const int j = s_bad_key[x] + key;
                                if (!((s_bad[x][key >> 5] >> (key & 31)) & 1u) || j > see_hi || j < see_lo) continue;
                                const int64_t at = cache_row(P, b, h, j, 1, 0, kv_len);
                                if (at >= P.n_pages * P.kv_heads * P.page_size) continue;
                                const uint16_t* v = reinterpret_cast<const uint16_t*>(P.v) + at * D + c;
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (HALF ? (v[e] & 0x7c00u) == 0x7c00u : nonfinite_bf16(v[e]))
                                        o[e] = __float_as_uint(__uint_as_float(o[e]) + (HALF ? __half2float(__ushort_as_half(v[e])) : bf16_bits_to_float(v[e])));
                            }
                    }
                    if constexpr (HALF) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * value_scale);
                    }
                    if (!live) continue;
                    if (P.splits > 1) {
                        float* dst = P.part_o + ((int64_t)part * (P.T * P.q_heads) + row) * D + c;
                        const bool wide = (reinterpret_cast<uintptr_t>(P.part_o) & 31u) == 0;       // the workspace is aligned to 16 bytes, or better
#pragma unroll
                        for (int e = 0; e < 4; ++e) store32(dst + 8 * e, o + 8 * e, wide);
                    } else {
                        __nv_bfloat16* dst = P.out + (q0 + tok) * P.ldo + (int64_t)(h * P.group + r % P.group) * D + c;
                        const bool wide = (reinterpret_cast<uintptr_t>(dst) & 31u) == 0;
                        uint32_t w[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) w[x] = any ? pack_bf16(__uint_as_float(o[2 * x]) * inv, __uint_as_float(o[2 * x + 1]) * inv) : 0u;
                        store32(dst, w, wide);
                        store32(dst + 16, w + 8, wide);
                    }
                }
            }
            tc::fence_before();
            if (n_it > 0) tc::mbar_arrive(tc::smem_u32(&s_read));
            asm volatile("bar.sync 1, %0;" ::"n"(C::kSoft) : "memory");             // s_bad is read before the next tile clears it
        }
        it += n_it;
        if (n_it > 0) ++round;
    }
    if (warp == kWarpK || warp == kWarpV) {                             // no copy may be in flight when the CTA ends, whatever became of its consumer
        const int stages = warp == kWarpV ? C::kStagesV : C::kStagesK;
        for (int u = max(0, issued - stages); u < issued; ++u)
            tc::mbar_wait(tc::smem_u32(warp == kWarpV ? s_vfull : s_kfull) + 8 * (u % stages), (uint32_t)(u / stages) & 1u, P.wait_cycles);
        if (q_issued) tc::mbar_wait(tc::smem_u32(&s_q), (uint32_t)(q_issued - 1) & 1u, P.wait_cycles);
    }
    tc::fence_before();
    __syncthreads();
    if (tid == 0 && s_timeout) report(P.dev_status, MATQ_ERR_TIMEOUT);
    if (warp == kWarpMma)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

}  // namespace attn
}  // namespace matq
