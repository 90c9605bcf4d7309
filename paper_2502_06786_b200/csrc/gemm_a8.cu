// matq_gemm_a8: Y[m,n] = xscale_m alpha_n ( sum_k xq[m,k] q[n,k] - z_n sum_k xq[m,k] ), the sums in 8-bit integers on the tensor cores.
#include "tc.cuh"

namespace matq {
namespace a8 {

constexpr int kBM = 128;             // channels of a CTA of the pair kernel: the rows of its accumulator (tensor-memory lanes)
constexpr int kBK = 128;             // bytes of K per block: one 128-byte swizzle row
constexpr int kMaxNT = 256;

struct Params {
    const float *alpha, *zero, *xscale;
    const int32_t* xsum;
    void* Y;
    int64_t M, N, K, ldy;
    int nkb, nt, splits, stages, tmem_cols, bf16_out, early;
    int32_t* dev_status;
    long long wait_cycles;
    int hold;
};

// kind::i8, D = s32, A = u8 (codes), B = s8 (activations), both K-major
__device__ __forceinline__ uint32_t idesc_i8(int m, int n) {
    return (2u << 4) | (0u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// What an output needs of its token, prepared once per tile: one 16-byte read per output of the pair kernel's epilogue.
struct __align__(16) Token {
    float xs, sum;       // scale; sum of its codes
    int off;             // 128 times that sum
    int pad;
};
__device__ __forceinline__ Token token(const Params& P, int64_t m) {
    Token t = {0.f, 0.f, 0, 0};
    if (m < P.M) {
        const int sum = P.xsum[m];
        t.xs = P.xscale[m];
        t.sum = (float)sum;
        t.off = 128 * sum;
    }
    return t;
}
__device__ __forceinline__ float finish(int acc, const Token& t, float al, float zc) { return (t.xs * al) * ((float)(acc - t.off) - zc * t.sum); }
__device__ __forceinline__ void put(float* y, float v) { *y = v; }
__device__ __forceinline__ void put(__nv_bfloat16* y, float v) { *y = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_y(const Params& P, int64_t m, int64_t n, float y) {
    if (P.bf16_out) put(static_cast<__nv_bfloat16*>(P.Y) + m * P.ldy + n, y);
    else put(static_cast<float*>(P.Y) + m * P.ldy + n, y);
}
// columns c_lo .. cols - 1 of an accumulator to the outputs of one channel
template <typename T>
__device__ __forceinline__ void store_columns(uint32_t addr, const Token* tok, int c_lo, int cols, bool live, T* y, int64_t ldy, float al, float zc) {
    for (int c0 = c_lo; c0 < cols; c0 += 16) {
        uint32_t d[16];
        tc::tmem_ld16(addr + c0, d);
        tc::tmem_wait_ld();
        T* p = y + (int64_t)c0 * ldy;
        if (!live) continue;
        if (c0 + 16 <= cols) {
#pragma unroll
            for (int j = 0; j < 16; ++j, p += ldy) put(p, finish((int)d[j], tok[c0 + j], al, zc));
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j, p += ldy)
                if (c0 + j < cols) put(p, finish((int)d[j], tok[c0 + j], al, zc));
        }
    }
}

// ---------------------------------------------------------------- few tokens: warp-level integer MMA
//
// Up to 8 tokens and a few megabytes of codes the product is mostly latency: no tensor memory, no tensor maps, no cluster (5 tokens, 544 x 4064: 3.0 us, the
// split kernel below 4.2; 8 tokens, 14336 x 4096 from HBM: 15.0 and 12.3, so that those go there).  A CTA takes 16 MT
// channels; its warps take 64-byte pieces of K in turn.  A thread loads 16 bytes of its row's piece: the four bytes per register that mma.sync
// m16n8k32 wants need not be neighbours in K as long as codes and activations agree, so the 16 bytes are two products' worth of fragments as they
// are, for codes and activations alike.  The warps' sums meet in shared memory (integers: the order is free).
constexpr int kFewWarps = 8, kFewThreads = 32 * kFewWarps, kFewMaxM = 8;

__device__ __forceinline__ void mma_u8s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// MT tiles of 16 channels; UNROLL pieces of K in flight per warp
template <int MT, int UNROLL>
__global__ void __launch_bounds__(kFewThreads)
gemm_a8_few_kernel(const uint8_t* __restrict__ q, int64_t ldw, const int8_t* xq, int64_t ldx, const Params P) {
    __shared__ int s_sum[8][16 * MT + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, kq = (lane & 3) * 16;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * MT);
    if (!P.early) { after_previous_kernel(); let_next_kernel_start(); }
    for (int i = tid; i < 8 * (16 * MT + 1); i += kFewThreads) (&s_sum[0][0])[i] = 0;
    const int K = (int)P.K, pieces = (K + 63) / 64;
    const uint8_t* wrow[2 * MT];
    bool wlive[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
        wlive[i] = n0 + g + 8 * i < P.N;
        wrow[i] = q + (wlive[i] ? n0 + g + 8 * i : 0) * ldw + kq;
    }
    int acc[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] = 0;
    bool waited = !P.early;
    for (int c0 = warp; c0 < pieces; c0 += kFewWarps * UNROLL) {
        uint4 w[UNROLL][2 * MT], x[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int k = (c0 + u * kFewWarps) * 64;
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) w[u][i] = wlive[i] && k + kq < K ? ld_stream_u4(wrow[i] + k) : make_uint4(0u, 0u, 0u, 0u);
        }
        if (!waited) { after_previous_kernel(); let_next_kernel_start(); waited = true; }         // the first codes are on their way before the activations are known to be there
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int k = (c0 + u * kFewWarps) * 64;
            x[u] = g < P.M && k + kq < K ? *reinterpret_cast<const uint4*>(xq + (int64_t)g * ldx + k + kq) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                mma_u8s8(acc[i], w[u][2 * i].x, w[u][2 * i + 1].x, w[u][2 * i].y, w[u][2 * i + 1].y, x[u].x, x[u].y);
                mma_u8s8(acc[i], w[u][2 * i].z, w[u][2 * i + 1].z, w[u][2 * i].w, w[u][2 * i + 1].w, x[u].z, x[u].w);
            }
    }
    if (!waited) { after_previous_kernel(); let_next_kernel_start(); }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) atomicAdd(&s_sum[2 * (lane & 3) + (e & 1)][16 * i + g + 8 * (e >> 1)], acc[i][e]);
    __syncthreads();
    for (int i = tid; i < 8 * 16 * MT; i += kFewThreads) {
        const int m = i / (16 * MT), c = i % (16 * MT);
        const int64_t n = n0 + c;
        if (m < P.M && n < P.N) store_y(P, m, n, finish(s_sum[m][c], token(P, m), P.alpha[n], P.zero[n] - 128.f));
    }
}

inline cudaError_t launch_few(const uint8_t* q, int64_t ldw, const int8_t* xq, int64_t ldx, const Params& P, int sms, cudaStream_t s) {
    // 32 channels per CTA halve the reads of the activations from the L2; 16 where 32 would leave SMs without work
    if ((P.N + 31) / 32 >= 2 * sms)
        return launch_overlapped(gemm_a8_few_kernel<2, 4>, dim3((unsigned)((P.N + 31) / 32)), dim3(kFewThreads), 0, s, q, ldw, xq, ldx, P);
    return launch_overlapped(gemm_a8_few_kernel<1, 8>, dim3((unsigned)((P.N + 15) / 16)), dim3(kFewThreads), 0, s, q, ldw, xq, ldx, P);
}

// ---------------------------------------------------------------- some tokens, or too few tiles for the pairs: K split inside a cluster
//
// A CTA sums 128 channels x nt tokens over a part of K in tensor memory; the CTAs of a cluster hold the same tile for different parts, put their sums into
// shared memory and finish every splits-th token each, reading the others' sums from there.  Tiles of up to 64 tokens leave room for two CTAs per SM.
// Eight warps store, as in the pair kernel (with four, one token tile of 128 took 6 us to store).
// From HBM, with MATQ_GEMV_PDL and without: 64 x 14336 x 4096 12.4 and 13.6 us (4.7 and 4.3 TB/s of codes), 37 x 2304 x 9216 8.7 and 9.3 us, of which the copies
// take 3.3; the rest is the start of a launch, the join and the stores.
constexpr int kSplitWarps = 8, kSplitThreads = 32 * (2 + kSplitWarps);
// A stage is 256 bytes of K here too (with 128, 600 tokens through 2304 x 9216 took 23 us instead of 19, 17 through 10587 x 11072 24 instead of 23).
constexpr int kMaxStages = 8, kMaxSplitsK = 8, kSplitBlocks = 2;

// Every splits-th token of the tile, from `split` on, every second of them for this warp: sums the parts that the cluster's CTAs hold ([token][channel], this thread's channel
// at `mine`) and stores the outputs.  All parts of four tokens are requested before the first is added: a load from another SM takes some hundred cycles.
template <typename T>
__device__ __forceinline__ void join_tokens(uint32_t mine, const Token* tok, int split, int splits, int odd, int cols, bool live, T* y, int64_t ldy, float al, float zc) {
    uint32_t from[kMaxSplitsK];
#pragma unroll
    for (int r = 0; r < kMaxSplitsK; ++r) asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from[r]) : "r"(mine), "r"(min(r, splits - 1)));
    const int step = 2 * splits;
    for (int c0 = split + odd * splits; c0 < cols; c0 += 4 * step) {
        int v[4][kMaxSplitsK];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < kMaxSplitsK; ++r) {
                const int c = c0 + i * step;
                v[i][r] = 0;
                if (r < splits && c < cols) asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v[i][r]) : "r"(from[r] + c * kBM * 4));
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = c0 + i * step;
            int sum = 0;
#pragma unroll
            for (int r = 0; r < kMaxSplitsK; ++r) sum += v[i][r];
            if (c < cols && live) put(y + (int64_t)c * ldy, finish(sum, tok[c], al, zc));
        }
    }
}

__global__ void __launch_bounds__(kSplitThreads)
gemm_a8_split_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Params P) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_acc;
    __shared__ uint32_t s_tmem;
    __shared__ int s_timeout;
    __shared__ Token s_tok[128];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int split = (int)(blockIdx.x % (unsigned)P.splits);            // rank in the cluster
    const int64_t n0 = (int64_t)(blockIdx.x / (unsigned)P.splits) * kBM, m0 = (int64_t)blockIdx.y * P.nt;
    const int nst = (P.nkb + kSplitBlocks - 1) / kSplitBlocks;                 // stages of the whole K; past K the copies bring zeros
    const int st0 = (int)((int64_t)nst * split / P.splits), st1 = (int)((int64_t)nst * (split + 1) / P.splits);
    const int block_bytes = (kBM + P.nt) * kBK, stage_bytes = kSplitBlocks * block_bytes;
    unsigned char* ring = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);

    if (!P.early) { after_previous_kernel(); let_next_kernel_start(); }
    if (tid == 0) {
        for (int s = 0; s < P.stages; ++s) { tc::mbar_init(tc::smem_u32(&s_full[s]), 1); tc::mbar_init(tc::smem_u32(&s_empty[s]), 1); }
        tc::mbar_init(tc::smem_u32(&s_acc), 1);
        tc::mbar_init_fence();
        s_timeout = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&s_tmem)), "r"(P.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = s_tmem;

    const int64_t n = n0 + (warp & 3) * 32 + lane;                      // epilogue warps: this thread's channel
    float al = 0.f, zc = 0.f;

    if (warp == 0) {
        if (lane == 0) {
            // the weights of the first stages are fetched before the activations are known to be there
            // (each of the two loops over K is one thread's chain of instructions: slots and descriptors are stepped, not computed)
            const int ahead = min(P.stages, st1 - st0);
            const uint32_t full = tc::smem_u32(s_full), empty = tc::smem_u32(s_empty), base = tc::smem_u32(ring);
            const auto weights = [&](uint32_t dst, int st, uint32_t bar) {
                tc::mbar_expect_tx(bar, stage_bytes);
#pragma unroll
                for (int i = 0; i < kSplitBlocks; ++i) tc::tma_load_2d(dst + i * block_bytes, &tm_w, (st * kSplitBlocks + i) * kBK, (int)n0, bar);
            };
            if (!P.hold)
                for (int i = 0; i < ahead; ++i) weights(base + (uint32_t)(i * stage_bytes), st0 + i, full + 8 * i);
            if (P.early) { after_previous_kernel(); let_next_kernel_start(); }
            int s = 0, issued = 0;
            uint32_t phase = 1;
            for (int st = st0; st < st1 && !P.hold; ++st) {
                const uint32_t dst = base + (uint32_t)(s * stage_bytes);
                if (issued >= ahead) {
                    if (!tc::mbar_wait(empty + 8 * s, phase, P.wait_cycles)) { s_timeout = 1; break; }
                    weights(dst, st, full + 8 * s);
                }
#pragma unroll
                for (int i = 0; i < kSplitBlocks; ++i) tc::tma_load_2d(dst + i * block_bytes + kBM * kBK, &tm_x, (st * kSplitBlocks + i) * kBK, (int)m0, full + 8 * s);
                ++issued;
                if (++s == P.stages) { s = 0; phase ^= 1u; }
            }
            // no copy may be in flight when the CTA ends, whatever became of its consumer
            for (int i = max(0, issued - P.stages); i < issued; ++i)
                tc::mbar_wait(full + 8 * (i % P.stages), (uint32_t)(i / P.stages) & 1u, P.wait_cycles);
        }
    } else if (warp == 1) {
        const uint32_t leader = tc::elect_one(), idesc = idesc_i8(kBM, P.nt), full = tc::smem_u32(s_full), empty = tc::smem_u32(s_empty);
        const uint64_t desc0 = tc::sw128_desc(tc::smem_u32(ring));
        int s = 0;
        uint32_t phase = 0, more = 0;
        for (int st = st0; st < st1; ++st) {
            if (!tc::warp_wait(full + 8 * s, phase, P.wait_cycles)) {
                *(volatile int*)&s_timeout = 1;
                __threadfence_block();
                break;
            }
            tc::fence_after();
            const uint64_t w = desc0 + (uint64_t)(s * (stage_bytes >> 4));
#pragma unroll
            for (int kk = 0; kk < kSplitBlocks * kBK / 32; ++kk) {
                const uint64_t at = w + (uint64_t)((kk / 4) * (block_bytes >> 4) + (kk & 3) * 2);
                MATQ_TC_MMA(1, "i8", tmem, at, at + (uint64_t)(kBM * kBK >> 4), idesc, more, leader);
                more = 1;
            }
            tc::tc_commit(empty + 8 * s, leader);
            if (++s == P.stages) { s = 0; phase ^= 1u; }
        }
        tc::tc_commit(tc::smem_u32(&s_acc), leader);
    } else {
        if (n < P.N) { al = P.alpha[n]; zc = P.zero[n] - 128.f; }
        if (P.early) after_previous_kernel();
        for (int c = tid - 64; c < P.nt; c += 32 * kSplitWarps) s_tok[c] = token(P, m0 + c);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const bool done = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_acc), 0, P.wait_cycles)) && *(volatile int*)&s_timeout == 0;
        if (!done) *(volatile int*)&s_timeout = 1;
        tc::fence_after();
        const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const int c_lo = ((warp - 2) >> 2) * (P.nt / 2), cols = (int)min((int64_t)(c_lo + P.nt / 2), P.M - m0);      // the two warps of a lane quarter
        if (done && P.splits == 1) {
            if (P.bf16_out) store_columns(lane_addr, s_tok, c_lo, cols, n < P.N, static_cast<__nv_bfloat16*>(P.Y) + m0 * P.ldy + n, P.ldy, al, zc);
            else store_columns(lane_addr, s_tok, c_lo, cols, n < P.N, static_cast<float*>(P.Y) + m0 * P.ldy + n, P.ldy, al, zc);
        } else if (done) {
            int* part = reinterpret_cast<int*>(ring) + (warp & 3) * 32 + lane;      // partial sums go where the stages were: [token][channel]
            for (int c0 = c_lo; c0 < cols; c0 += 16) {
                uint32_t d[16];
                tc::tmem_ld16(lane_addr + c0, d);
                tc::tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (c0 + j < cols) part[(c0 + j) * kBM] = (int)d[j];
            }
        }
    }
    if (P.splits > 1) {
        // The CTAs of a cluster hold the same tile for different parts of K.  Integer sums: the order is free.
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned; barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (warp >= 2) {
            bool ok = true;
            for (int r = 0; r < P.splits; ++r) {
                uint32_t a, t;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(&s_timeout)), "r"(r));
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(t) : "r"(a) : "memory");
                ok &= t == 0;
            }
            const uint32_t mine = tc::smem_u32(ring) + ((warp & 3) * 32 + lane) * 4;
            const int cols = (int)min((int64_t)P.nt, P.M - m0), odd = (warp - 2) >> 2;
            if (ok && P.bf16_out) join_tokens(mine, s_tok, split, P.splits, odd, cols, n < P.N, static_cast<__nv_bfloat16*>(P.Y) + m0 * P.ldy + n, P.ldy, al, zc);
            else if (ok) join_tokens(mine, s_tok, split, P.splits, odd, cols, n < P.N, static_cast<float*>(P.Y) + m0 * P.ldy + n, P.ldy, al, zc);
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned; barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    tc::fence_before();
    __syncthreads();
    if (tid == 0 && s_timeout) report(P.dev_status, MATQ_ERR_TIMEOUT);
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(P.tmem_cols) : "memory");
}

// ---------------------------------------------------------------- many tokens: pairs of SMs
//
// Two CTAs of a cluster share a tile of 256 channels x nt tokens (tcgen05.mma with cta_group::2): each holds its 128 channels and half of the
// tokens in shared memory and its 128 channels x nt sums in tensor memory, so that a byte brought into an SM meets twice the products of
// a CTA by itself.  The even CTA issues the products for both; a stage's barrier lives in it and collects both CTAs' copies, and one commit frees
// the stage in both.  The kernel is persistent: a pair takes every (number of pairs)-th tile, two accumulators take turns, and eight
// warps store one tile while the next is summed.  Channels are the accumulator's rows, so a thread keeps its channel's alpha and z in registers and a
// warp's stores run along a token's outputs.
// A stage is 256 bytes of K, two blocks of 128: waiting for a stage, issuing and committing cost the issuing thread about 500 cycles whatever the
// stage holds, and the products of one block take no more than that (4096 x 14336 x 4096: 770 cycles a block with one block per stage).
// 4096 x 14336 x 4096: 164 us = 2.93 POP/s (about 190 us in a long run, at the power cap).  What bounds it is the tensor pipe.
constexpr int kPairWarps = 8, kPairThreads = 32 * (2 + kPairWarps), kPairStages = 3, kPairBlocks = 2;
constexpr int kPairBlockBytes = 2 * kBM * kBK;       // 128 channels and up to 128 tokens
constexpr int kPairStageBytes = kPairBlocks * kPairBlockBytes;

__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
// a copy into this CTA whose bytes are counted by a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t cluster_bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(cluster_bar) : "memory");
}
// arrives on the same barrier of both CTAs when every product issued so far has ended
__device__ __forceinline__ void commit_pair(uint32_t bar, uint32_t leader) {
    asm volatile("{ .reg .pred e; setp.ne.b32 e, %2, 0; @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1; }"
                 ::"r"(bar), "h"((uint16_t)3), "r"(leader) : "memory");
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
gemm_a8_pair_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Params P) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t s_full[kPairStages], s_empty[kPairStages], s_acc[2], s_read[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_timeout;
    __shared__ Token s_tok[2][kMaxNT];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = blockIdx.x & 1u;
    unsigned char* ring = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);      // the same offset in both CTAs

    if (tid == 0) {
        for (int s = 0; s < kPairStages; ++s) { tc::mbar_init(tc::smem_u32(&s_full[s]), 1); tc::mbar_init(tc::smem_u32(&s_empty[s]), 1); }
        for (int a = 0; a < 2; ++a) { tc::mbar_init(tc::smem_u32(&s_acc[a]), 1); tc::mbar_init(tc::smem_u32(&s_read[a]), 2 * kPairWarps); }
        tc::mbar_init_fence();
        s_timeout = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&s_tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc::fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned; barrier.cluster.wait.acquire.aligned;" ::: "memory");     // the other CTA's barriers are there
    tc::fence_after();
    const uint32_t tmem = s_tmem;
    after_previous_kernel();
    let_next_kernel_start();

    const int m_tiles = (int)((P.M + P.nt - 1) / P.nt), n_tiles = (int)((P.N + 2 * kBM - 1) / (2 * kBM)), tiles = m_tiles * n_tiles;
    const int pairs = (int)(gridDim.x >> 1), pair = (int)(blockIdx.x >> 1), half = P.nt / 2;
    int round = 0;                                                      // tiles so far

    // The two loops over K are each one thread's chain of instructions, and a stage's products take 512 cycles: everything that does not change
    // with the stage stays out of them (with slot numbers by division and descriptors put together in place they took a thousand).
    if (warp == 0) {
        if (lane == 0 && !P.hold) {
            bool ok = true;
            int s = 0;
            uint32_t phase = 1;
            const uint32_t full = tc::smem_u32(s_full), empty = tc::smem_u32(s_empty), lead = in_cta(full, 0), base = tc::smem_u32(ring);
            const uint32_t bytes = 2 * kPairBlocks * (kBM + half) * kBK;
            for (int tile = pair; tile < tiles && ok; tile += pairs) {
                const int m0 = (int)min((int64_t)(tile % m_tiles) * P.nt + rank * half, P.M), n0 = tile / m_tiles * (2 * kBM) + (int)rank * kBM;
                for (int x = 0; x < P.nkb * kBK; x += kPairBlocks * kBK) {             // past K the copies bring zeros
                    if (!tc::mbar_wait(empty + 8 * s, phase, P.wait_cycles)) { *(volatile int*)&s_timeout = 1; ok = false; break; }
                    if (rank == 0) tc::mbar_expect_tx(full + 8 * s, bytes);
                    const uint32_t dst = base + s * kPairStageBytes;
#pragma unroll
                    for (int i = 0; i < kPairBlocks; ++i) {
                        tma_load_pair(dst + i * kPairBlockBytes, &tm_w, x + i * kBK, n0, lead + 8 * s);
                        tma_load_pair(dst + i * kPairBlockBytes + kBM * kBK, &tm_x, x + i * kBK, m0, lead + 8 * s);
                    }
                    if (++s == kPairStages) { s = 0; phase ^= 1u; }
                }
            }
            // the commits that free the last stages arrive here from the even CTA: they are waited for, so that none meets a CTA that has ended
            for (int i = 0; i < kPairStages && ok; ++i) {
                ok = tc::mbar_wait(empty + 8 * s, phase, P.wait_cycles);
                if (++s == kPairStages) { s = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t leader = tc::elect_one(), idesc = idesc_i8(2 * kBM, P.nt);
            bool ok = true;
            int s = 0;
            uint32_t phase = 0;
            const uint32_t full = tc::smem_u32(s_full), empty = tc::smem_u32(s_empty);
            const uint64_t desc0 = tc::sw128_desc(tc::smem_u32(ring));
            for (int tile = pair; tile < tiles; tile += pairs, ++round) {
                const int a = round & 1;
                ok = tc::warp_wait(tc::smem_u32(&s_read[a]), ((uint32_t)(round >> 1) & 1u) ^ 1u, P.wait_cycles);
                tc::fence_after();
                const uint32_t d = tmem + a * 256;
                uint32_t more = 0;
                for (int kb = 0; kb < P.nkb && ok; kb += kPairBlocks) {
                    if (!(ok = tc::warp_wait(full + 8 * s, phase, P.wait_cycles))) break;
                    tc::fence_after();
                    const uint64_t w = desc0 + (uint64_t)(s * (kPairStageBytes >> 4));
#pragma unroll
                    for (int kk = 0; kk < kPairBlocks * kBK / 32; ++kk) {
                        const uint64_t at = w + (uint64_t)((kk / 4) * (kPairBlockBytes >> 4) + (kk & 3) * 2);
                        MATQ_TC_MMA(2, "i8", d, at, at + (uint64_t)(kBM * kBK >> 4), idesc, more, leader);
                        more = 1;
                    }
                    commit_pair(empty + 8 * s, leader);
                    if (++s == kPairStages) { s = 0; phase ^= 1u; }
                }
                if (!ok) { *(volatile int*)&s_timeout = 1; __threadfence_block(); break; }
                commit_pair(tc::smem_u32(&s_acc[a]), leader);
            }
        }
    } else {
        // ---------------- outputs: thread = channel; the two warps of a lane quarter take half of the tokens each
        const int quad = warp & 3, part = (warp - 2) >> 2;
        const int c_lo = part * half, c_hi = part ? P.nt : half;
        bool ok = true;
        for (int tile = pair; tile < tiles; tile += pairs, ++round) {
            const int64_t m0 = (int64_t)(tile % m_tiles) * P.nt, n = (int64_t)(tile / m_tiles) * (2 * kBM) + rank * kBM + quad * 32 + lane;
            const int a = round & 1;
            for (int c = tid - 64; c < P.nt; c += 32 * kPairWarps) s_tok[a][c] = token(P, m0 + c);
            float al = 0.f, zc = 0.f;
            if (n < P.N) { al = P.alpha[n]; zc = P.zero[n] - 128.f; }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (ok) ok = __all_sync(0xffffffffu, tc::mbar_wait(tc::smem_u32(&s_acc[a]), (uint32_t)(round >> 1) & 1u, P.wait_cycles));
            if (ok) {
                tc::fence_after();
                const uint32_t addr = tmem + ((uint32_t)(quad * 32) << 16) + a * 256;
                const int cols = (int)min((int64_t)c_hi, P.M - m0);
                if (P.bf16_out) store_columns(addr, s_tok[a], c_lo, cols, n < P.N, static_cast<__nv_bfloat16*>(P.Y) + m0 * P.ldy + n, P.ldy, al, zc);
                else store_columns(addr, s_tok[a], c_lo, cols, n < P.N, static_cast<float*>(P.Y) + m0 * P.ldy + n, P.ldy, al, zc);
                tc::fence_before();
            } else {
                *(volatile int*)&s_timeout = 1;
            }
            __syncwarp();
            if (lane == 0)
                asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_cta(tc::smem_u32(&s_read[a]), 0)) : "memory");
        }
    }
    // Nobody leaves while the other may still write into its barriers or read its stages.  The pair's copies are over by then: the even CTA consumed
    // them all, or its waits for them ran out first.
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned; barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (tid == 0 && s_timeout) report(P.dev_status, MATQ_ERR_TIMEOUT);
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

inline bool byte_map(CUtensorMap* tm, const void* base, int64_t rows, int64_t K, int64_t ld, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)box_rows};
    return tc::make_map(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box);
}

enum Kind { kNone = -1, kFew = MATQ_GEMM_A8_FEW, kSplit = MATQ_GEMM_A8_SPLIT, kPairs = MATQ_GEMM_A8_PAIRS };
struct Shape {
    int kind, nt, splits;        // nt: token width of a tile; splits: CTAs that share K
    int64_t cost;
};

// Kernel and tile: the shape whose estimated time is least.  Measured, ns: the start 2000 (pairs 2500); 256 bytes of K 350 (pairs 420,
// above 168 tokens 2.5 a token); storing a tile 14 a token (pairs 800 and 18, while the next tile is summed); a cluster's join 1200 and 20 a token; an SM's
// copies 85 GB/s, HBM 6300.  A cluster's CTAs share a GPC, which leaves clusters of eight about 128 of 148 SMs and clusters of four about 136.
// The few-token kernel: 2200, and its copies at 45 GB/s per SM, 5000 in all.
// Sizes that no kernel's grid holds have no shape.
inline Shape choose(int64_t M, int64_t N, int64_t K, int sms) {
    Shape s = {kNone, 0, 0, 0};
    const auto offer = [&s](int kind, int nt, int splits, int64_t cost) {
        if (s.kind == kNone || cost < s.cost) s = {kind, nt, splits, cost};
    };
    const int pairs = sms / 2;
    const int64_t nst = ((K + kBK - 1) / kBK + 1) / 2, n_pair = (N + 2 * kBM - 1) / (2 * kBM), tiles_n = (N + kBM - 1) / kBM, hbm = N * K / 6300;
    if (M <= kFewMaxM) {
        const int64_t sm = ((N + 15) / 16 + sms - 1) / sms * 16 * K / 45, all = N * K / 5000;
        offer(kFew, 0, 1, 2200 + (sm > all ? sm : all));
    }
    for (int nt = 16; nt <= 128; nt *= 2) {
        const int64_t tiles_m = (M + nt - 1) / nt;
        if ((nt < 128 && tiles_m > 8) || tiles_m > 65535) continue;
        for (int sp = 1; sp <= kMaxSplitsK && sp <= nst; sp *= 2) {
            const int64_t ctas = tiles_n * tiles_m * sp, stages = (nst + sp - 1) / sp, usable = sp == 8 ? sms * 128 / 148 : sp == 4 ? sms * 136 / 148 : sms;
            const int64_t slots = usable * (nt <= 64 ? 2 : 1), rounds = (ctas + slots - 1) / slots, copies = (ctas + usable - 1) / usable * stages * (kBM + nt) * 256 / 85;
            int64_t work = rounds * stages * 350;
            if (work < copies) work = copies;
            if (work < hbm) work = hbm;
            offer(kSplit, nt, sp, work + rounds * (2000 + (sp > 1 ? 1200 + 20 * nt : 14 * nt)));
        }
    }
    for (int nt = 256; nt >= 64 && M > 32; nt -= 32) {
        const int64_t tiles = n_pair * ((M + nt - 1) / nt), rounds = (tiles + pairs - 1) / pairs;
        if (tiles >= (1ll << 30)) continue;
        const int64_t sum = nst * (nt > 168 ? 5 * nt / 2 : 420), store = 800 + 18 * nt;
        int64_t work = (rounds - 1) * (sum > store ? sum : store) + sum;
        if (work < hbm) work = hbm;
        offer(kPairs, nt, 1, 2500 + work + store);
    }
    return s;
}

inline int size_error(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 0 || K <= 0) return MATQ_ERR_INVALID_ARG;
    if (K % 16 != 0 || K > 65536 || M >= (1ll << 31) || N >= (1ll << 31)) return MATQ_ERR_SHAPE;
    return MATQ_OK;
}

}  // namespace a8
}  // namespace matq

extern "C" int matq_gemm_a8_plan(int64_t M, int64_t N, int64_t K, int* kernel, int* tokens, int* parts) {
    using namespace matq;
    using namespace matq::a8;
    const int st = size_error(M, N, K);
    if (st != MATQ_OK) return st;
    if (M == 0 || N == 0) return MATQ_ERR_INVALID_ARG;
    const Shape s = choose(M, N, K, sm_count());
    if (s.kind == kNone) return MATQ_ERR_SHAPE;
    if (kernel) *kernel = s.kind;
    if (tokens) *tokens = s.kind == kFew ? kFewMaxM : s.nt;
    if (parts) *parts = s.splits;
    return MATQ_OK;
}

extern "C" int matq_gemm_a8(const int8_t* xq, int64_t M, int64_t K, int64_t ldxq, const float* xscale, const int32_t* xsum,
                            const uint8_t* q, int64_t N, int64_t ldw, int c, const float* alpha, const float* zero,
                            int out_type, void* Y, int64_t ldy, unsigned flags, int32_t* dev_status, void* stream) {
    using namespace matq;
    using namespace matq::a8;
    if (M < 0 || N < 0 || K <= 0 || (out_type != MATQ_OUT_F32 && out_type != MATQ_OUT_BF16) || (flags & ~(unsigned)MATQ_GEMV_PDL)) return MATQ_ERR_INVALID_ARG;
    if (c != kCodeBits) return MATQ_ERR_UNSUPPORTED;
    if (size_error(M, N, K) != MATQ_OK || ldxq < K || ldxq % 16 != 0 || ldw < K || ldw % 16 != 0 || ldy < N) return MATQ_ERR_SHAPE;
    if (M == 0 || N == 0) return MATQ_OK;
    if (!xq || !xscale || !xsum || !q || !alpha || !zero || !Y) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(xq) || !aligned16(q)) return MATQ_ERR_ALIGNMENT;
    cudaStream_t s = static_cast<cudaStream_t>(stream);

    Params P;
    P.alpha = alpha; P.zero = zero; P.xscale = xscale; P.xsum = xsum; P.Y = Y; P.M = M; P.N = N; P.ldy = ldy;
    P.bf16_out = out_type == MATQ_OUT_BF16;
    P.early = (flags & MATQ_GEMV_PDL) ? 1 : 0;
    P.dev_status = dev_status;
    P.hold = tc::test_stall() ? 1 : 0;
    P.wait_cycles = P.hold ? tc::kStallWaitCycles : tc::kWaitCycles;
    P.K = K;
    P.nkb = (int)((K + kBK - 1) / kBK);
    const int sms = sm_count();
    const Shape shape = choose(M, N, K, sms);
    if (shape.kind == kNone) return MATQ_ERR_SHAPE;
    P.nt = shape.nt; P.splits = shape.splits;
    cudaError_t e;
    if (shape.kind == kFew) {
        e = launch_few(q, ldw, xq, ldxq, P, sms, s);
    } else if (shape.kind == kSplit) {
        P.tmem_cols = P.nt < 32 ? 32 : P.nt;
        const int64_t tiles_n = (N + kBM - 1) / kBM, tiles_m = (M + P.nt - 1) / P.nt;
        const int stage_bytes = kSplitBlocks * (kBM + P.nt) * kBK;
        P.stages = (P.nt <= 64 && tiles_n * tiles_m * P.splits > sms ? 104 * 1024 : 200 * 1024) / stage_bytes;      // two CTAs share an SM, or one has it
        if (P.stages > kMaxStages) P.stages = kMaxStages;
        size_t smem = (size_t)P.stages * stage_bytes;
        if (P.splits > 1 && smem < (size_t)P.nt * kBM * 4) smem = (size_t)P.nt * kBM * 4;
        CUtensorMap tm_w, tm_x;
        if (!byte_map(&tm_w, q, N, K, ldw, kBM) || !byte_map(&tm_x, xq, M, K, ldxq, P.nt)) return MATQ_ERR_CUDA;
        static std::atomic<unsigned long long> split_ok{0};
        if (!opt_in_max_smem(gemm_a8_split_kernel, split_ok)) return MATQ_ERR_CUDA;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(tiles_n * P.splits), (unsigned)tiles_m);
        cfg.blockDim = dim3(kSplitThreads);
        cfg.dynamicSmemBytes = smem + 1024;
        cfg.stream = s;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)P.splits;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        e = cudaLaunchKernelEx(&cfg, gemm_a8_split_kernel, tm_w, tm_x, P);
    } else {
        const int64_t tiles = (N + 2 * kBM - 1) / (2 * kBM) * ((M + P.nt - 1) / P.nt), pairs = sms / 2;
        CUtensorMap tm_w, tm_x;
        if (!byte_map(&tm_w, q, N, K, ldw, kBM) || !byte_map(&tm_x, xq, M, K, ldxq, P.nt / 2)) return MATQ_ERR_CUDA;
        static std::atomic<unsigned long long> pair_ok{0};
        if (!opt_in_max_smem(gemm_a8_pair_kernel, pair_ok)) return MATQ_ERR_CUDA;
        const unsigned grid = 2u * (unsigned)(tiles < pairs ? tiles : pairs);
        e = launch_overlapped(gemm_a8_pair_kernel, dim3(grid), dim3(kPairThreads), (size_t)kPairStages * kPairStageBytes + 1024, s, tm_w, tm_x, P);
    }
    if (e != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}
