// matq_gemm_groups: a linear layer on weights in 4-bit groups for many tokens, on the fifth-generation tensor cores.
//
// y[m,n] = sum_g ( scale_ng sum_{k in g} x_mk (q_nk - 8) + (low_ng + 8 scale_ng) sum_{k in g} x_mk ).  scale (q - 8) has at most 8 + 3 bits, which fp16 holds: with a
// power of two per row of the matrix the weights enter the products as fp16 without a rounding, and so do the tokens' bf16 with a power of two per token.  The second
// term is four more columns of K per group: (low, low, 8 scale, 8 scale) beside (hi, lo, hi, lo) of the tokens' sums in two fp16 (22 bits).  So the whole layer is one
// product with sums in fp32 in tensor memory, and nothing is done per group behind it.  (Sums of codes alone would have to be read back, scaled and added for every group: 128 x 128
// values, as often as every second product with groups of 32.)
//
// A first kernel writes the tokens as fp16, in the order in which masks take codes out of a word, and their sums, and transposes the groups, scaled, so that a thread that
// has a row finds them beside its neighbours'.  In the second, persistent one a thread of the eight converting warps has a row of 128: codes come by TMA, become
// fp16 in registers (13 instructions for eight) and go to tensor memory, from where the products take them; tokens come by TMA into shared memory.  Eight warps add and
// store one tile's sums while the next is multiplied.  Few tiles: the CTAs of a cluster share K.  bf16 outputs of many tiles: pairs of CTAs (cta_group::2) with 256 rows x
// 256 tokens, so that a block that was converted meets twice the tokens (4096 tokens x 14336 x 4096, groups of 128, 388 us or 1.24 PFLOP/s, with single CTAs 481).
//
// Bound: the converting warps, about 1000 cycles for a block of 128 x 128 weights, whose products take 4 cycles a token, and the hand-overs around them (without any
// one of conversion, copies of codes, stores to tensor memory or products a block takes 3 to 13 % less; three sets of four converting warps instead of two are no faster);
// beside that whole rounds: 1024 tokens x 14336 rows are 224 tiles for 74 pairs, of which the fourth round has two.
// 64 tokens x 14336 x 4096 27 us, of which the first kernel, the start and the end take 12 (matq_gemv_groups: 61 us); 1024 tokens 121 us (794).
#include <cuda_fp16.h>

#include "group4.cuh"
#include "tc.cuh"

namespace matq {
namespace grpm {

constexpr int kBM = 128, kBlock = 128;       // rows of a tile; columns of a block of K
constexpr int kMaxNT = 128, kPairNT = 256, kSlots = 4, kCodeStages = 5;
constexpr int kCodeStage = 128 * 128;        // bytes: two blocks of 128 rows
constexpr int kTokenRing = kSlots * kMaxNT * 256;
constexpr int kThreads = 32 * 18;            // warps 0-7 add and store, 8-15 convert, 16 copies, 17 multiplies
// Blocks whose products are summed in tensor memory: these sums are cut off, not rounded, so that their error grows with their length (K = 2304 2.4e-6 of the outputs' norm,
// 14336 1.7e-5); every 1024 columns they are added to sums in registers, beside the next products.
constexpr int kSegment = 8;
constexpr size_t kSmem = 1024 + kCodeStages * kCodeStage + kTokenRing;
constexpr int kPrepThreads = 256, kPrepRows = 32;
constexpr int kTokenExp = 7, kRowExp = 14;   // the largest of a token comes to lie in [2^7, 2^8), so that sums of 128 stay within fp16; of a row in [2^14, 2^15)

struct Prepare {
    const __nv_bfloat16* x;
    const uint32_t* params;
    int64_t M, N, K, ldx, n_pad, width;      // width: columns of a prepared token
    int group, groups, main_width;
    __half* xp;                              // [M][width]
    int *token_exp, *row_exp;                // what was taken off
    uint32_t* scaled;                        // [groups][n_pad]: (scale, low) as two fp16
};

__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__global__ void __launch_bounds__(kPrepThreads) gemm_groups_prepare_kernel(const Prepare P) {
    __shared__ uint32_t s_top[kPrepRows];
    after_previous_kernel();
    let_next_kernel_start();
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid < kPrepRows) s_top[tid] = 0u;
    __syncthreads();
    if (blockIdx.x < P.M) {                  // a token
        const int64_t m = blockIdx.x;
        const __nv_bfloat16* x = P.x + m * P.ldx;
        const int pieces = P.main_width / 8, real = (int)(P.K / 8), lanes = P.group / 8;
        uint32_t top = 0u;
        for (int i = tid; i < real; i += kPrepThreads) top = max(top, top_of_piece(*reinterpret_cast<const uint4*>(x + 8 * (int64_t)i)));
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) atomicMax(&s_top[0], top);
        __syncthreads();
        const int e = max((int)(s_top[0] >> 23) - 127 - kTokenExp, -126);
        const float by = exp2i(-e);
        __half* to = P.xp + m * P.width;
        for (int i0 = 0; i0 < pieces; i0 += kPrepThreads) {
            const int i = i0 + tid;
            const uint4 v = i < real ? *reinterpret_cast<const uint4*>(x + 8 * (int64_t)i) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            float f[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(w[j] << 16) * by; f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u) * by; }
            float sum = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
            for (int s = 1; s < lanes; s <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
            if (i < pieces) *reinterpret_cast<uint4*>(to + 8 * (int64_t)i) = make_uint4(half2_bits(f[0], f[4]), half2_bits(f[1], f[5]), half2_bits(f[2], f[6]), half2_bits(f[3], f[7]));
            if (i < real && i % lanes == 0) {
                const float hi = __half2float(__float2half_rn(sum));
                const uint32_t both = half2_bits(hi, sum - hi);
                *reinterpret_cast<uint2*>(to + P.main_width + 4 * (int64_t)(i / lanes)) = make_uint2(both, both);
            }
        }
        for (int i = P.groups + tid; i < (P.width - P.main_width) / 4; i += kPrepThreads) *reinterpret_cast<uint2*>(to + P.main_width + 4 * (int64_t)i) = make_uint2(0u, 0u);
        if (tid == 0) P.token_exp[m] = e;
        return;
    }
    // 32 rows of the matrix: their largest, four rows a warp, then 32 groups at a time, read along the rows and written across them
    __shared__ uint32_t s_tile[2][kPrepRows][33];
    const int64_t n0 = (blockIdx.x - P.M) * kPrepRows;
    const int warp = tid / 32;
    constexpr int kEach = kPrepRows / (kPrepThreads / 32);
    uint32_t top[kEach] = {};
    for (int i = lane; i < P.groups; i += 32)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int64_t n = n0 + warp * kEach + j;
            const uint32_t g = n < P.N ? P.params[n * P.groups + i] : 0u;
            const float most = fminf(fmaxf(fabsf(low_of(g)), 8.f * fabsf(scale_of(g))), 3.402823466e38f);
            if (scale_of(g) == scale_of(g)) top[j] = max(top[j], __float_as_uint(most));         // not of a group that stands for NaN
        }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t t = __reduce_max_sync(0xffffffffu, top[j]);
        if (lane == 0) s_top[warp * kEach + j] = t;
    }
    __syncthreads();
    const int e = max((int)(s_top[lane] >> 23) - 127 - kRowExp, -126);
    const float by = exp2i(-e);
    for (int i0 = 0, turn = 0; i0 < P.groups; i0 += 32, turn ^= 1) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = warp * kEach + j;
            s_tile[turn][r][lane] = n0 + r < P.N && i0 + lane < P.groups ? P.params[(n0 + r) * P.groups + i0 + lane] : 0u;
        }
        __syncthreads();                                                // (the other tile is written next: one barrier a turn)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int i = warp * kEach + j;
            const uint32_t g = s_tile[turn][lane][i];
            if (i0 + i < P.groups) P.scaled[(int64_t)(i0 + i) * P.n_pad + n0 + lane] = half2_bits(scale_of(g) * by, low_of(g) * by);
        }
    }
    if (tid < kPrepRows && n0 + tid < P.N) P.row_exp[n0 + tid] = e;
}

struct Params {
    const uint32_t* scaled;
    const int *token_exp, *row_exp;
    void* y;
    int64_t M, N, ldy, n_pad;
    int groups;                  // of a row
    int main, extra;             // blocks of codes, and of low ends and scales
    int nt;                      // tokens of a tile
    int splits;                  // CTAs of a cluster, which share K; more than one: a cluster has one tile
    int out_bf16, hold;
    long long wait_cycles;
    int32_t* dev_status;
};

__device__ __forceinline__ float scaled(float sum, int e) {             // in two halves: each is a power of two that fp32 holds
    const int h = e >> 1;
    return sum * exp2i(h) * exp2i(e - h);
}
__device__ __forceinline__ void put(float* y, float v) { *y = v; }
__device__ __forceinline__ void put(__nv_bfloat16* y, float v) { *y = __float2bfloat16_rn(v); }
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned; barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
                   "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
                   "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
// Eight codes as fp16 times scale: (code - 8) scale, exact.  1024 + n is the number with the bits of n below 1024's (a published way from integers to fp16: Kim et al. 2022,
// "Who Says Elephants Can't Run").
__device__ __forceinline__ void weights_of(uint32_t w, __half2 scale, uint32_t* o) {
    const auto number = [](uint32_t bits) { return *reinterpret_cast<const __half2*>(&bits); };
    const __half2 up = __floats2half2_rn(-1032.f, -1032.f), part = __floats2half2_rn(0.0625f, 0.0625f), less = __floats2half2_rn(-72.f, -72.f);
    const uint32_t w8 = w >> 8;
    const __half2 v[4] = {__hadd2(number((w & 0x000f000fu) | 0x64006400u), up), __hfma2(number((w & 0x00f000f0u) | 0x64006400u), part, less),
                          __hadd2(number((w8 & 0x000f000fu) | 0x64006400u), up), __hfma2(number((w8 & 0x00f000f0u) | 0x64006400u), part, less)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 p = __hmul2(v[i], scale);
        o[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
}

__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
// A copy of a block of tokens into this CTA, whose bytes are counted by a barrier of either CTA of a pair
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t cluster_bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(cluster_bar) : "memory");
}
// arrives on a barrier of this CTA, or on the same barrier of both CTAs of a pair, when every product issued so far has ended
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar, uint32_t leader) {
    if constexpr (PAIR)
        asm volatile("{ .reg .pred e; setp.ne.b32 e, %2, 0; @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1; }"
                     ::"r"(bar), "h"((uint16_t)3), "r"(leader) : "memory");
    else tc::tc_commit(bar, leader);
}
// Arrives on a barrier of this CTA, or on that of a pair's first CTA.  What is handed over stands in tensor memory, whose accesses tcgen05.wait and the fences around
// the barrier order: a release at the cluster's scope would wait for everything else too (1200 cycles, measured, as long as two blocks' products take).
template <bool PAIR>
__device__ __forceinline__ void arrive(uint32_t bar) {
    if constexpr (PAIR) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_cta(bar, 0)) : "memory");
    else tc::mbar_arrive(bar);
}

// S: groups of a block.  PAIR: two CTAs of 128 rows share the tokens, half of which each of them brings, and the first issues the products of both.
template <int S, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) gemm_groups_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Params P) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_cfull[kCodeStages], s_cempty[kCodeStages], s_full[kSlots], s_empty[kSlots], s_acc[2], s_read[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_timeout;
    __shared__ int s_exp[2][PAIR ? kPairNT : kMaxNT];
    constexpr int kTokens = PAIR ? kPairNT : kMaxNT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char* codes = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);
    const uint32_t code_ring = tc::smem_u32(codes), token_ring = code_ring + kCodeStages * kCodeStage;
    if (tid == 0) {
        for (int s = 0; s < kCodeStages; ++s) { tc::mbar_init(tc::smem_u32(&s_cfull[s]), 1); tc::mbar_init(tc::smem_u32(&s_cempty[s]), 8); }
        for (int s = 0; s < kSlots; ++s) { tc::mbar_init(tc::smem_u32(&s_full[s]), PAIR ? 9 : 5); tc::mbar_init(tc::smem_u32(&s_empty[s]), 1); }
        for (int a = 0; a < 2; ++a) { tc::mbar_init(tc::smem_u32(&s_acc[a]), 1); tc::mbar_init(tc::smem_u32(&s_read[a]), PAIR ? 16 : 8); }
        tc::mbar_init_fence();
        s_timeout = 0;
    }
    if (warp == 17) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&s_tmem)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&s_tmem)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc::fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();                                           // the other CTA's barriers are there
    tc::fence_after();
    const uint32_t tmem = s_tmem, slots = tmem + 256;
    after_previous_kernel();
    let_next_kernel_start();

    // A cluster is consecutive CTAs: a pair, which shares a tile of 256 rows, or the CTAs that share K.
    const int shared = PAIR ? 2 : P.splits, rank = (int)blockIdx.x % shared, first_tile = (int)blockIdx.x / shared, step = (int)gridDim.x / shared;
    const int splits = PAIR ? 1 : P.splits, part = PAIR ? 0 : rank, row_part = PAIR ? rank : 0;
    const int m_tiles = (int)((P.M + P.nt - 1) / P.nt), tiles = m_tiles * (int)((P.N + (PAIR ? 2 : 1) * kBM - 1) / ((PAIR ? 2 : 1) * kBM));
    const auto rows_from = [&](int tile) { return (tile / m_tiles * (PAIR ? 2 : 1) + row_part) * kBM; };
    // this CTA's blocks, in pairs: two blocks of codes come by one copy
    const int all_pairs = (P.main + P.extra + 1) / 2, p_lo = (int)((int64_t)all_pairs * part / splits), p_hi = (int)((int64_t)all_pairs * (part + 1) / splits);
    const int b_lo = 2 * p_lo, b_hi = min(2 * p_hi, P.main + P.extra), blocks = b_hi - b_lo, code_pairs = min(p_hi, (P.main + 1) / 2);
    const uint32_t token_bytes = (uint32_t)P.nt * (PAIR ? 128 : 256);    // of a block, in this CTA: two columns of 64 elements, 128 bytes a token
    // The sums of a cluster's CTAs, [token][row], where the tokens were: a cluster has one tile, whose products are over by then.
    float* parts = reinterpret_cast<float*>(codes + kCodeStages * kCodeStage);
    bool ok = true;

    if (warp == 16) {
        // ---------------- copies
        if (lane == 0 && !P.hold) {
            int cs = 0, xs = 0;
            uint32_t cphase = 1, xphase = 1;
            for (int tile = first_tile; tile < tiles && ok; tile += step) {
                const int m0 = tile % m_tiles * P.nt + row_part * (P.nt / 2), n0 = rows_from(tile);
                for (int i = b_lo; i < b_hi; ++i) {
                    if (i < P.main && (i & 1) == 0) {
                        if (!(ok = tc::mbar_wait(tc::smem_u32(&s_cempty[cs]), cphase, P.wait_cycles))) break;
                        tc::mbar_expect_tx(tc::smem_u32(&s_cfull[cs]), kCodeStage);
                        tc::tma_load_2d(code_ring + cs * kCodeStage, &tm_w, i * (kBlock / 2), n0, tc::smem_u32(&s_cfull[cs]));
                        if (++cs == kCodeStages) { cs = 0; cphase ^= 1u; }
                    }
                    if (!(ok = tc::mbar_wait(tc::smem_u32(&s_empty[xs]), xphase, P.wait_cycles))) break;
                    if (row_part == 0) tc::mbar_expect_tx(tc::smem_u32(&s_full[xs]), (PAIR ? 2 : 1) * token_bytes);
                    if constexpr (PAIR) tma_load_3d_pair(token_ring + xs * token_bytes, &tm_x, 0, m0, 2 * i, in_cta(tc::smem_u32(&s_full[xs]), 0));
                    else tc::tma_load_3d(token_ring + xs * token_bytes, &tm_x, 0, m0, 2 * i, tc::smem_u32(&s_full[xs]));
                    if (++xs == kSlots) { xs = 0; xphase ^= 1u; }
                }
            }
            // What frees the last slots is waited for: no copy and no product may be in flight when the CTA ends, whatever became of the warps that wait for them, and in a
            // pair it arrives from the other CTA.  (A wait that ran out above or here lasted longer than any copy takes.)
            for (int i = 0; i < kSlots && ok; ++i) {
                ok = tc::mbar_wait(tc::smem_u32(&s_empty[xs]), xphase, P.wait_cycles);
                if (++xs == kSlots) { xs = 0; xphase ^= 1u; }
            }
            if (!ok) *(volatile int*)&s_timeout = 1;
        }
    } else if (warp == 17) {
        // ---------------- products
        const uint32_t leader = tc::elect_one(), idesc = (1u << 4) | ((uint32_t)(P.nt >> 3) << 17) | ((PAIR ? 16u : 8u) << 24);       // D = fp32, A = B = fp16
        const uint64_t desc0 = tc::sw128_desc(token_ring);
        int slot = 0, round = 0;
        uint32_t phase = 0;
        for (int tile = first_tile; tile < tiles && ok && row_part == 0; tile += step)
            for (int i0 = 0; i0 < blocks && ok; i0 += PAIR ? blocks : kSegment, ++round) {
                const int a = PAIR ? 0 : round & 1, n = PAIR ? blocks : min(kSegment, blocks - i0);
                ok = tc::warp_wait(tc::smem_u32(&s_read[a]), ((uint32_t)(PAIR ? round : round >> 1) & 1u) ^ 1u, P.wait_cycles);
                tc::fence_after();
                for (int i = 0; i < n && ok; ++i) {
                    if (!(ok = tc::warp_wait(tc::smem_u32(&s_full[slot]), phase, P.wait_cycles))) break;
                    tc::fence_after();
                    const uint64_t at = desc0 + (uint64_t)(slot * (token_bytes >> 4));
                    // tensor memory is this CTA's as a whole: its first column is column 0, and the addresses need no register that differs between threads
#pragma unroll
                    for (int x = 0; x < kBlock / 16; ++x) {
                        const uint32_t w = 256 + slot * 64 + x * 8, d = a * kMaxNT, more = i > 0 || x > 0;
                        const uint64_t t = at + (uint64_t)((x / 4) * (token_bytes >> 5) + (x & 3) * 2);
                        if constexpr (PAIR) MATQ_TC_MMA_TMEM_A(2, "f16", d, w, t, idesc, more, leader);
                        else MATQ_TC_MMA_TMEM_A(1, "f16", d, w, t, idesc, more, leader);
                    }
                    commit<PAIR>(tc::smem_u32(&s_empty[slot]), leader);
                    if (++slot == kSlots) { slot = 0; phase ^= 1u; }
                }
                if (ok) commit<PAIR>(tc::smem_u32(&s_acc[a]), leader);
            }
        if (!ok) *(volatile int*)&s_timeout = 1;
    } else if (warp >= 8) {
        // ---------------- weights: two sets of four warps take every second block
        const int set = (warp - 8) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        int cs = 0, u0 = 0;                                             // u0: blocks before this tile
        uint32_t cphase = 0;
        for (int tile = first_tile; tile < tiles && ok; tile += step, u0 += blocks) {
            const uint32_t* groups = P.scaled + rows_from(tile) + row;
            const auto group = [&](int i) { return i < P.groups ? groups[(int64_t)i * P.n_pad] : 0u; };
            const auto put = [&](int i, int part, const uint32_t* v) { tmem_st32(slots + lanes + ((u0 + i - b_lo) % kSlots) * 64 + part * 32, v); };
            const auto slot_free = [&](int i) {
                const int u = u0 + i - b_lo;
                const bool f = tc::warp_wait(tc::smem_u32(&s_empty[u % kSlots]), ((uint32_t)(u / kSlots) & 1u) ^ 1u, P.wait_cycles);
                tc::fence_after();
                return f;
            };
            const auto slot_full = [&](int i) {
                tc::tmem_wait_st();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) arrive<PAIR>(tc::smem_u32(&s_full[(u0 + i - b_lo) % kSlots]));
            };
            uint32_t next[S];
#pragma unroll
            for (int s = 0; s < S; ++s) next[s] = group((b_lo + set) * S + s);
            for (int p = p_lo; p < code_pairs && ok; ++p) {
                const int i = 2 * p + set;
                uint32_t now[S];
#pragma unroll
                for (int s = 0; s < S; ++s) { now[s] = next[s]; next[s] = group((i + 2) * S + s); }
                if (!(ok = tc::warp_wait(tc::smem_u32(&s_cfull[cs]), cphase, P.wait_cycles))) break;
                uint4 w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const uint4*>(codes + cs * kCodeStage + row * 128 + (((set * 4 + k) ^ (row & 7)) * 16));
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&s_cempty[cs]));
                if (++cs == kCodeStages) { cs = 0; cphase ^= 1u; }
                if (i >= P.main) continue;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t o[32];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint4 v = w[2 * part + k];
                        const uint32_t c[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t g = now[((2 * part + k) * 4 + j) * S / 16], twice = __byte_perm(g, g, 0x1010);
                            weights_of(c[j], *reinterpret_cast<const __half2*>(&twice), o + (k * 4 + j) * 4);
                        }
                    }
                    if (part == 0 && !(ok = slot_free(i))) break;
                    put(i, part, o);
                }
                if (!ok) break;
                slot_full(i);
            }
            for (int i = max(P.main, b_lo); i < b_hi && ok; ++i) {
                if ((i & 1) != set) continue;
                const int e = i - P.main;
                uint32_t g[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) g[j] = group(e * 32 + j);
                if (!(ok = slot_free(i))) break;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t o[32];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const __half2 v = *reinterpret_cast<const __half2*>(&g[part * 16 + j]);
                        const __half2 low = __half2half2(__high2half(v)), up = __hmul2(__half2half2(__low2half(v)), __floats2half2_rn(8.f, 8.f));
                        o[2 * j] = *reinterpret_cast<const uint32_t*>(&low);
                        o[2 * j + 1] = *reinterpret_cast<const uint32_t*>(&up);
                    }
                    put(i, part, o);
                }
                slot_full(i);
            }
        }
        if (!ok) *(volatile int*)&s_timeout = 1;
    } else {
        // ---------------- sums: thread = row of the matrix, half of the tokens
        // (all warps walk all tiles, whatever became of their waits: they meet at a barrier)
        const int quad = warp & 3, half = (P.nt / 16 + 1) / 2 * 16, c_lo = warp < 4 ? 0 : half, pieces = ((warp < 4 ? half : P.nt) - c_lo) / 16;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        int round = 0, turn = 0;
        for (int tile = first_tile; tile < tiles; tile += step, turn ^= 1) {
            const int64_t m0 = (int64_t)(tile % m_tiles) * P.nt, n = (int64_t)rows_from(tile) + quad * 32 + lane;
            const int cols = (int)min((int64_t)P.nt, P.M - m0), row_exp = n < P.N ? P.row_exp[n] : 0;
            if (tid < kTokens) s_exp[turn][tid] = tid < cols ? P.token_exp[m0 + tid] : 0;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if constexpr (PAIR) {                                       // bf16 outputs, straight from tensor memory
                if (ok) ok = tc::warp_wait(tc::smem_u32(&s_acc[0]), (uint32_t)round & 1u, P.wait_cycles);
                ++round;
                if (ok) {
                    tc::fence_after();
                    __nv_bfloat16* y = static_cast<__nv_bfloat16*>(P.y) + m0 * P.ldy + n;
                    for (int p = 0; p < pieces; ++p) {
                        uint32_t v[16];
                        tc::tmem_ld16(tmem + lanes + c_lo + 16 * p, v);
                        tc::tmem_wait_ld();
                        if (n >= P.N) continue;
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            const int at = c_lo + 16 * p + c;
                            const float out = scaled(__uint_as_float(v[c]), row_exp + s_exp[turn][at]);
                            if (at < cols) put(y + at * P.ldy, out);
                        }
                    }
                    tc::fence_before();
                }
                __syncwarp();
                if (lane == 0) arrive<PAIR>(tc::smem_u32(&s_read[0]));
            } else {
                float sum[kMaxNT / 32][16];
#pragma unroll
                for (int p = 0; p < kMaxNT / 32; ++p)
#pragma unroll
                    for (int c = 0; c < 16; ++c) sum[p][c] = 0.f;
                for (int i0 = 0; i0 < blocks; i0 += kSegment, ++round) {
                    const int a = round & 1;
                    if (ok) ok = tc::warp_wait(tc::smem_u32(&s_acc[a]), (uint32_t)(round >> 1) & 1u, P.wait_cycles);
                    if (ok) {
                        tc::fence_after();
#pragma unroll
                        for (int p = 0; p < kMaxNT / 32; ++p)
                            if (p < pieces) {
                                uint32_t v[16];
                                tc::tmem_ld16(tmem + lanes + a * kMaxNT + c_lo + 16 * p, v);
                                tc::tmem_wait_ld();
#pragma unroll
                                for (int c = 0; c < 16; ++c) sum[p][c] += __uint_as_float(v[c]);
                            }
                        tc::fence_before();
                    }
                    __syncwarp();
                    if (lane == 0) arrive<PAIR>(tc::smem_u32(&s_read[a]));
                }
                const auto each = [&](auto f) {                             // f(the token, its sum)
#pragma unroll
                    for (int p = 0; p < kMaxNT / 32; ++p)
                        if (p < pieces) {
#pragma unroll
                            for (int c = 0; c < 16; ++c) f(c_lo + 16 * p + c, sum[p][c]);
                        }
                };
                const auto stored = [&](auto* y) {
                    y += m0 * P.ldy + n;
                    each([&](int at, float v) {
                        const float out = scaled(v, row_exp + s_exp[turn][at]);
                        if (at < cols) put(y + at * P.ldy, out);
                    });
                };
                if (splits > 1) each([&](int at, float v) { parts[at * kBM + quad * 32 + lane] = v; });
                else if (ok && n < P.N) {
                    if (P.out_bf16) stored(static_cast<__nv_bfloat16*>(P.y));
                    else stored(static_cast<float*>(P.y));
                }
            }
        }
        if (!ok) *(volatile int*)&s_timeout = 1;
    }
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();                                           // nobody leaves while the other may still write into its barriers or read its tokens
    if (splits > 1) {
        cluster_sync();
        const int64_t m0 = (int64_t)(first_tile % m_tiles) * P.nt, n0 = rows_from(first_tile);
        const int cols = (int)min((int64_t)P.nt, P.M - m0);
        for (int i = rank * kThreads + tid; i < cols * kBM; i += P.splits * kThreads) {
            float of[8], sum = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                uint32_t at;
                of[c] = 0.f;
                if (c < P.splits) {
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(parts + i)), "r"(c));
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(of[c]) : "r"(at) : "memory");
                }
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) sum += of[c];
            const int64_t m = m0 + i / kBM, n = n0 + i % kBM;
            if (n >= P.N) continue;
            const float v = scaled(sum, P.row_exp[n] + P.token_exp[m]);
            if (P.out_bf16) put(static_cast<__nv_bfloat16*>(P.y) + m * P.ldy + n, v);
            else put(static_cast<float*>(P.y) + m * P.ldy + n, v);
        }
        cluster_sync();                                                 // nobody leaves while another reads its sums
    }
    if (tid == 0 && s_timeout) report(P.dev_status, MATQ_ERR_TIMEOUT);
    if (warp == 17) {
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

struct Plan {
    int main, extra;
    int64_t width, n_pad, groups;
    size_t x_bytes, exp_bytes, scaled_bytes;
    size_t total() const { return x_bytes + exp_bytes + scaled_bytes; }
};
inline size_t padded(size_t n) { return (n + 255) / 256 * 256; }
inline Plan plan(int64_t M, int64_t N, int64_t K, int group) {
    Plan p;
    p.groups = K / group;
    p.main = (int)((K + kBlock - 1) / kBlock);
    p.extra = (int)((4 * p.groups + kBlock - 1) / kBlock);
    p.width = (int64_t)(p.main + p.extra) * kBlock;
    p.n_pad = (N + 2 * kBM - 1) / (2 * kBM) * (2 * kBM);
    p.x_bytes = padded((size_t)M * p.width * 2);
    p.exp_bytes = padded((size_t)(M + N) * 4);
    p.scaled_bytes = padded((size_t)p.groups * p.n_pad * 4);
    return p;
}
inline bool sizes_ok(int64_t M, int64_t N, int64_t K, int group) {
    return M > 0 && N > 0 && K > 0 && (group == 32 || group == 64 || group == 128) && K % group == 0 && K <= 65536 && N < (1ll << 31) - 2 * kBM && M < (1ll << 31) - kPairNT &&
           ((M + 15) / 16) * ((N + kBM - 1) / kBM) < (1ll << 30) && M + N / kPrepRows + 4 < (1ll << 31);
}

// Tokens of a tile, shared out evenly; as many CTAs to a tile as leave no tile waiting (clusters of eight find about 128 of 148 SMs, of four about 136, and each
// CTA takes two pairs of blocks or more), or, for bf16 outputs, pairs where they take less time.  Cycles, measured: a block of a CTA 550 and 3.7 a token, of a pair 1050;
// a tile's end, which a pair does not overlap, 20 a token.  The products of a CTA take tokens in steps of 16, those of a pair in steps of 32.
struct Shape {
    bool pair;
    int nt, splits;              // tokens of a tile; CTAs that share K
    int64_t tiles;
};
inline Shape choose(int64_t M, int64_t N, const Plan& p, int out_type, int sms) {
    const auto tokens_of = [&](int most, int step) { const int64_t t = (M + most - 1) / most; return (int)(((M + t - 1) / t + step - 1) / step * step); };
    const auto tiles_of = [&](int nt, int rows) { return ((M + nt - 1) / nt) * ((N + rows - 1) / rows); };
    const int blocks = p.main + p.extra, nt_one = tokens_of(kMaxNT, 16), nt_pair = tokens_of(kPairNT, 32);
    const int64_t tiles = tiles_of(nt_one, kBM), tiles_pair = tiles_of(nt_pair, 2 * kBM);
    const double one = (double)((tiles + sms - 1) / sms) * blocks * (550 + 3.7 * nt_one), two = (double)((tiles_pair + sms / 2 - 1) / (sms / 2)) * (blocks * 1050.0 + 20.0 * nt_pair);
    if (out_type == MATQ_OUT_BF16 && tiles > sms && two < one) return {true, nt_pair, 1, tiles_pair};
    int splits = 1;
    for (int n = 2; n <= 8; n *= 2)
        if (tiles * n <= (n == 8 ? sms * 7 / 8 : n == 4 ? sms * 9 / 10 : sms) && blocks >= 4 * n) splits = n;
    return {false, nt_one, splits, tiles};
}

template <int S, bool PAIR>
int launch(const CUtensorMap& tw, const CUtensorMap& tx, const Params& P, unsigned grid, cudaStream_t s) {
    static std::atomic<unsigned long long> smem_ok{0};
    if (!opt_in_max_smem(gemm_groups_kernel<S, PAIR>, smem_ok)) return MATQ_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PAIR ? 2u : (unsigned)P.splits;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, gemm_groups_kernel<S, PAIR>, tw, tx, P) != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}

}  // namespace grpm
}  // namespace matq

// From 33 tokens on, with large matrices from 17 on, where its two launches weigh less.  us, and matq_gemv_groups', groups of 128: 14336 x 4096, 24 tokens 26.1 and 28.5, 64
// tokens 27.5 and 61.3; 4096 x 4096, 48 tokens 18.0 and 22.6; 2304 x 2304, 256 tokens 18.6 and 18.7.  The rule weighs tokens before the matrix: small matrices and few rows
// take less time with matq_gemv_groups for up to 256 tokens (1024 x 1024, 48 tokens 11.0 and 4.8, 256 tokens 14.8 and 7.4; 2304 x 2304, 48 tokens 11.2 and 9.5; 300 x 14336,
// 64 tokens 18.9 and 12.4; 4096 x 1024, 128 tokens 15.2 and 10.3).
extern "C" int matq_gemm_groups_pays(int64_t M, int64_t N, int64_t K, int group) {
    using namespace matq::grpm;
    return sizes_ok(M, N, K, group) && (M > 32 || (M > 16 && (double)N * K >= (double)(1 << 25)));
}

extern "C" size_t matq_gemm_groups_workspace_bytes(int64_t M, int64_t N, int64_t K, int group) {
    using namespace matq::grpm;
    return sizes_ok(M, N, K, group) ? plan(M, N, K, group).total() : 0;
}

extern "C" int matq_gemm_groups_plan(int64_t M, int64_t N, int64_t K, int group, int out_type, int* pairs, int* tokens, int* parts) {
    using namespace matq;
    using namespace matq::grpm;
    if (M < 1 || N < 1 || K < 0 || (out_type != MATQ_OUT_F32 && out_type != MATQ_OUT_BF16)) return MATQ_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return MATQ_ERR_UNSUPPORTED;
    if (!sizes_ok(M, N, K, group)) return MATQ_ERR_SHAPE;
    const Shape s = choose(M, N, plan(M, N, K, group), out_type, sm_count());
    if (pairs) *pairs = s.pair ? 1 : 0;
    if (tokens) *tokens = s.nt;
    if (parts) *parts = s.splits;
    return MATQ_OK;
}

extern "C" int matq_gemm_groups(const uint8_t* packed, int64_t N, int64_t K, int group, const void* params, const void* x, int64_t M, int64_t ldx, int out_type, void* y,
                                int64_t ldy, void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    using namespace matq;
    using namespace matq::grpm;
    if (N < 0 || K < 0 || M < 0 || (out_type != MATQ_OUT_F32 && out_type != MATQ_OUT_BF16)) return MATQ_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return MATQ_ERR_UNSUPPORTED;
    if (K == 0 || K % group != 0 || K > 65536 || ldx < K || ldx % 8 != 0 || ldy < N) return MATQ_ERR_SHAPE;
    if (M == 0 || N == 0) return MATQ_OK;
    if (!sizes_ok(M, N, K, group)) return MATQ_ERR_SHAPE;
    if (!packed || !params || !x || !y) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(packed) || !aligned16(params) || !aligned16(x) || !aligned16(workspace)) return MATQ_ERR_ALIGNMENT;
    const Plan p = plan(M, N, K, group);
    if (p.total() > workspace_bytes || !workspace) return MATQ_ERR_WORKSPACE;
    unsigned char* at = static_cast<unsigned char*>(workspace);
    Prepare A;
    A.x = static_cast<const __nv_bfloat16*>(x); A.params = static_cast<const uint32_t*>(params);
    A.M = M; A.N = N; A.K = K; A.ldx = ldx; A.n_pad = p.n_pad; A.width = p.width; A.group = group; A.groups = (int)p.groups; A.main_width = p.main * kBlock;
    A.xp = reinterpret_cast<__half*>(at);
    A.token_exp = reinterpret_cast<int*>(at + p.x_bytes);
    A.row_exp = A.token_exp + M;
    A.scaled = reinterpret_cast<uint32_t*>(at + p.x_bytes + p.exp_bytes);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int sms = sm_count();
    const Shape shape = choose(M, N, p, out_type, sms);
    const bool pair = shape.pair;
    const int nt = shape.nt, splits = shape.splits;
    const cuuint64_t wd[2] = {(cuuint64_t)(K / 2), (cuuint64_t)N}, ws[1] = {(cuuint64_t)(K / 2)};
    const cuuint64_t xd[3] = {64, (cuuint64_t)M, (cuuint64_t)(p.width / 64)}, xs[2] = {(cuuint64_t)p.width * 2, 128};
    const cuuint32_t wb[2] = {128, kBM}, xb[3] = {64, (cuuint32_t)(pair ? nt / 2 : nt), 2};
    CUtensorMap tw, tx;
    if (!tc::make_map(&tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, packed, wd, ws, wb) || !tc::make_map(&tx, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, A.xp, xd, xs, xb)) return MATQ_ERR_CUDA;
    if (launch_overlapped(gemm_groups_prepare_kernel, dim3((unsigned)(M + p.n_pad / kPrepRows)), dim3(kPrepThreads), 0, s, A) != cudaSuccess) {
        cudaGetLastError();
        return MATQ_ERR_CUDA;
    }
    Params P;
    P.scaled = A.scaled; P.token_exp = A.token_exp; P.row_exp = A.row_exp; P.y = y; P.M = M; P.N = N; P.ldy = ldy; P.n_pad = p.n_pad;
    P.groups = (int)p.groups; P.main = p.main; P.extra = p.extra; P.nt = nt;
    P.out_bf16 = out_type == MATQ_OUT_BF16; P.hold = tc::test_stall() ? 1 : 0; P.wait_cycles = P.hold ? tc::kStallWaitCycles : tc::kWaitCycles; P.dev_status = dev_status;
    P.splits = splits;
    const unsigned grid = (unsigned)(pair ? 2 * (shape.tiles < sms / 2 ? shape.tiles : sms / 2) : shape.tiles * splits < sms ? shape.tiles * splits : sms);
    if (pair) return group == 128 ? launch<1, true>(tw, tx, P, grid, s) : group == 64 ? launch<2, true>(tw, tx, P, grid, s) : launch<4, true>(tw, tx, P, grid, s);
    return group == 128 ? launch<1, false>(tw, tx, P, grid, s) : group == 64 ? launch<2, false>(tw, tx, P, grid, s) : launch<4, false>(tw, tx, P, grid, s);
}
