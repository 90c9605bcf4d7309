// 4-bit weights with a scale and a low end per group of 32, 64 or 128 weights of a row: matq_quantize_groups and matq_gemv_groups.
#include <type_traits>

#include "group4.cuh"

namespace matq {
namespace grp {

// ---------------------------------------------------------------- quantiser
// A thread takes eight weights, the threads of a group are neighbours in a warp and exchange its two ends by shuffles.  Groups follow one another without
// a gap, across the ends of rows too, so that codes and groups have one running index each.  Every weight is read once: HBM, and beside it the instructions of a
// weight (correctly rounded operations one by one; two weights in one instruction where there is one): 9216 x 2304, groups of 64, 12.1 us (4.5 TB/s), 14336 x 4096,
// groups of 128, 27.2 us (5.5 TB/s).  Four pieces a thread, requested together.
constexpr int kQuantThreads = 256, kQuantPieces = 4;

template <int GROUP, bool DENSE>
__global__ void __launch_bounds__(kQuantThreads) quantize_groups_kernel(const __nv_bfloat16* W, int64_t total, int64_t row_pieces, int64_t ldw,
                                                                        uint32_t* packed, uint32_t* params, int32_t* dev_status) {
    after_previous_kernel();
    let_next_kernel_start();
    const int64_t first = (int64_t)blockIdx.x * (kQuantThreads * kQuantPieces) + threadIdx.x;
    uint4 w[kQuantPieces];
#pragma unroll
    for (int i = 0; i < kQuantPieces; ++i) {
        const int64_t f = first + i * kQuantThreads;
        const __nv_bfloat16* src = W + f * 8;
        if (!DENSE) {
            const int64_t row = total <= 0xffffffffll ? (int64_t)((uint32_t)f / (uint32_t)row_pieces) : f / row_pieces;
            src = W + row * ldw + (f - row * row_pieces) * 8;
        }
        w[i] = f < total ? ld_stream_u4(src) : make_uint4(0u, 0u, 0u, 0u);
    }
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kQuantPieces; ++i) {
        const int64_t f = first + i * kQuantThreads;
        uint32_t codes;
        const uint32_t sl = quantise_piece<GROUP / 8>(w[i], codes);
        if (f < total) {
            packed[f] = codes;
            if ((threadIdx.x & (GROUP / 8 - 1)) == 0) {
                params[f / (GROUP / 8)] = sl;
                bad |= sl == kNoGroup;
            }
        }
    }
    if (__any_sync(0xffffffffu, bad) && (threadIdx.x & 31) == 0) report(dev_status, MATQ_ERR_NONFINITE);
}

template <int GROUP>
cudaError_t launch_quantize(const void* W, int64_t N, int64_t K, int64_t ldw, void* packed, void* params, int32_t* dev_status, cudaStream_t s) {
    const int64_t total = N * (K / 8), per = kQuantThreads * kQuantPieces;
    const dim3 grid((unsigned)((total + per - 1) / per));
    const auto w = static_cast<const __nv_bfloat16*>(W);
    const auto p = static_cast<uint32_t*>(packed), g = static_cast<uint32_t*>(params);
    if (ldw == K || N == 1) return launch_overlapped(quantize_groups_kernel<GROUP, true>, grid, dim3(kQuantThreads), 0, s, w, total, K / 8, ldw, p, g, dev_status);
    return launch_overlapped(quantize_groups_kernel<GROUP, false>, grid, dim3(kQuantThreads), 0, s, w, total, K / 8, ldw, p, g, dev_status);
}

// ---------------------------------------------------------------- product of a few tokens
// y[m,n] = sum_g ( scale_ng sum_{k in g} x_mk q_nk + low_ng sum_{k in g} x_mk ): the inner sums on the tensor cores (mma.sync m16n8k16: 16 rows of the matrix,
// 8 columns of tokens), what surrounds them in fp32 once per group.
//
// Codes enter the products as they are masked out of a word, without a conversion: the bf16 number with the bits of an integer i below 256 is i * 2^-133, also
// through bit 7, where the subnormal numbers end, and the tensor cores take it exactly.  Five instructions make operands of eight codes: (w & 0x000f000f) holds
// codes 0 and 4, (w & 0x00f000f0) 16 times codes 1 and 5, and w >> 8 the other four likewise.  The tokens stand in shared memory in that order of pairs, scaled
// by a power of two (and by 2^-4 where the code is 16 times too large), so that no product leaves fp32's range (group4.cuh).
//
// The sixteen elements of a product's row, four lanes' words, have to lie in one group.  With S = 2 or 4 groups in a block of 128 there are two forms.  C = S: the lanes
// read the block as if it were one group, and a token has a column for each group, zero in the lanes of the others; its eight columns hold 8 / S tokens.  C = 1: the lanes
// read the block group by group, eight or four bytes each at a time, and add each group's sums on its own.  The first is taken while it needs no second block of columns:
// 65536 x 2304, groups of 64, one token 19.9 against 21.5 us, four tokens x 4096 x 4096 6.5 against 7.5; beyond that its products double: 64 tokens, 14336 x 4096,
// groups of 32, 140 against 73 us.
//
// A CTA takes a part of K, staged in shared memory for its tokens, and walks the matrix in steps of 16 RW rows; its warps are RW row tiles times SK parts of
// that part, block by block of 128.  Each warp brings its own blocks into its own ring by cp.async, across the ends of steps, so that the ring never drains.
// The CTAs of a cluster share K and add their sums through distributed shared memory.  All sums are taken in a fixed order.
//
// Bound: one token, the chain of a launch (start, tokens' trip to memory, staging, the last blocks' trip, sums): 9216 x 2304 5.2 us, 14336 x 4096 10.5, 65536 x 2304 (a second
// step for 216 of 296 CTAs) 18.9 us or 4.5 TB/s.  16 tokens: latencies of 16 warps (1.9 instructions a cycle) and the cluster's sums: 3584 x 14336 18.0 us.
constexpr int kBlock = 128;
// Warps of a CTA: eight, and two CTAs on an SM, as long as a CTA has one block of columns; sixteen beside tokens that take more shared memory.
__host__ __device__ constexpr int warps_of(int nt) { return nt == 1 ? 8 : 16; }
// Bytes from row to row in a ring: four lanes that read a block in four passes take 16 bytes of a row at a time, which eight rows 64 bytes apart would have on the same banks.
__host__ __device__ constexpr int row_bytes_of(int passes) { return passes == 4 ? 80 : 64; }
__host__ __device__ constexpr int ctas_of(int nt) { return nt > 1 ? 1 : 2; }
__host__ __device__ constexpr int depth_of(int nt, int mt) { return nt > 1 && mt > 1 ? 3 : nt == 1 && mt == 1 ? 6 : 4; }

struct GemvParams {
    const uint8_t* packed;
    const uint32_t* params;      // (scale, low) as two bf16, [N, K / group]
    const __nv_bfloat16* x;
    void* y;
    int64_t N, K, M, ldx, ldy, groups;       // groups of a row
    int tokens;                  // per CTA (a multiple goes to gridDim.z)
    int sk, rw;                  // sk * rw = the CTA's warps
    int slice;                   // most blocks of a CTA's part of K
    int steps;                   // of 16 rw rows
    int early;                   // codes and groups may be fetched before the wait
    int out_bf16;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool in) {
    // a warp's next block is the next 64 bytes of the same rows: HBM is asked for more of a row at a time
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool in) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float ld_cluster(const float* p, unsigned rank) {
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void store(const GemvParams& P, int64_t m, int64_t row, float v) {
    if (row >= P.N) return;
    if (P.out_bf16) static_cast<__nv_bfloat16*>(P.y)[m * P.ldy + row] = __float2bfloat16_rn(v);
    else static_cast<float*>(P.y)[m * P.ldy + row] = v;
}

// The exponent of the factor that tokens get as long as each of their elements is zero or lies between 2^-92 and 2^24, so that nothing else has to be known of them.
constexpr int kUsualExp = 99;
__device__ __forceinline__ bool unusual(uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t most = 0u, least = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t m = w[i] & 0x7fff7fffu;
        most = __vmaxu2(most, m);
        least = __vminu2(least, __vsub2(m, 0x00010001u));               // zero becomes the largest
    }
    return max(most & 0xffffu, most >> 16) >= 0x4b80u || min(least & 0xffffu, least >> 16) < 0x1180u - 1u;
}

// NT blocks of eight columns, S groups in a block of K, C columns of a token (1 or S), MT tiles of 16 rows of a warp
template <int NT, int S, int C, int MT>
__global__ void __launch_bounds__(32 * warps_of(NT), ctas_of(NT)) gemv_groups_kernel(const GemvParams P) {
    constexpr int kWarps = warps_of(NT), kThreads = 32 * kWarps, kDepth = depth_of(NT, MT);
    constexpr int kPasses = S / C, kRow = row_bytes_of(kPasses), kCodes = 16 * MT * kRow;          // a block's codes of a row, and of 16 MT rows
    constexpr int kSlot = kCodes + 64 * S * MT, kWarpRing = kDepth * kSlot;              // and their groups
    constexpr int kWords = 4 / kPasses;      // of eight codes of a row that a lane takes in a pass
    constexpr int kCols = NT * 8, kTile = 16 * MT, kGroupCopies = (kTile * S + 31) / 32;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint32_t s_top[32];           // largest magnitude per token (bits of a float)
    __shared__ __align__(16) uint4 s_zero[16];      // a block of no token
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
    const int rt = warp % P.rw, kw = warp / P.rw, rows = kTile * P.rw, rows_shift = 31 - __clz(rows);
    const unsigned cl = gridDim.x, rank = blockIdx.x;                   // the cluster is the grid's x
    const int blocks = (int)((P.K + kBlock - 1) / kBlock), b_lo = (int)((int64_t)blocks * rank / cl);
    const int n_blocks = (int)((int64_t)blocks * (rank + 1) / cl) - b_lo;
    const int64_t m0 = (int64_t)blockIdx.z * P.tokens;
    const int tokens = (int)min((int64_t)P.tokens, P.M - m0);

    // shared memory: the warps' rings; tokens [tokens][slice][256 bytes] (+ 64 bytes a token); sums of groups [slice passes][columns]; results
    const int x_stride = P.slice * 256 + 64;
    unsigned char* s_x = smem + kWarps * kWarpRing;
    float* s_sum = reinterpret_cast<float*>(s_x + (size_t)P.tokens * x_stride);
    float* s_red = s_sum + (size_t)P.slice * kPasses * kCols;

    // ---- this warp's blocks, fetched kDepth - 1 ahead: a lane brings 16 bytes of rows g, g + 8, .., and some of the tile's groups
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + (uint32_t)warp * kWarpRing;
    int f_step = kw < n_blocks ? (int)blockIdx.y : P.steps, f_block = kw, f_at = 0;
    const uint8_t* f_w[2 * MT];
    const uint32_t* f_g[kGroupCopies];
    int f_has[kGroupCopies];                                            // blocks that have this group
    const int f_in = (int)(P.K / kBlock) + (q < (int)(P.K % kBlock) / 32) - b_lo;         // blocks that have this lane's 32 columns
#pragma unroll
    for (int e = 0; e < kGroupCopies; ++e) f_has[e] = lane + 32 * e < kTile * S ? (int)((P.groups - (lane + 32 * e) % S + S - 1) / S) - b_lo : 0;
    const auto rows_of_step = [&] {                                     // past the end: the last row, whose sums are not stored
        const int64_t row0 = (int64_t)f_step * rows + rt * kTile;
#pragma unroll
        for (int e = 0; e < 2 * MT; ++e) f_w[e] = P.packed + min(row0 + g + 8 * e, P.N - 1) * (P.K / 2) + (int64_t)b_lo * (kBlock / 2) + 16 * q;
#pragma unroll
        for (int e = 0; e < kGroupCopies; ++e) f_g[e] = P.params + min(row0 + (lane + 32 * e) / S, P.N - 1) * P.groups + (int64_t)b_lo * S + (lane + 32 * e) % S;
    };
    if (f_step < P.steps) rows_of_step();
    const auto fetch = [&] {
        if (f_step < P.steps) {
#pragma unroll
            for (int e = 0; e < 2 * MT; ++e) copy16(ring + f_at + (g + 8 * e) * kRow + q * 16, f_w[e] + f_block * 64, f_block < f_in);
#pragma unroll
            for (int e = 0; e < kGroupCopies; ++e)
                if (kTile * S % 32 == 0 || lane < kTile * S) copy4(ring + f_at + kCodes + (lane + 32 * e) * 4, f_g[e] + f_block * S, f_block < f_has[e]);
            f_block += P.sk;
            if (f_block >= n_blocks) {
                f_block = kw;
                f_step += gridDim.y;
                if (f_step < P.steps) rows_of_step();
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        f_at = f_at == (kDepth - 1) * kSlot ? 0 : f_at + kSlot;
    };
    if (tid < 32) s_top[tid] = 0u;
    if (tid < 16) s_zero[tid] = make_uint4(0u, 0u, 0u, 0u);
    for (int i = tid; i < P.slice * kPasses * kCols; i += kThreads) s_sum[i] = 0.f;
    if (!P.early) after_previous_kernel();
#pragma unroll 1
    for (int d = 0; d < kDepth - 1; ++d) fetch();
    after_previous_kernel();                                            // (at once if it has waited above)

    // ---- the tokens, four pieces of eight elements a thread at a time, scaled and in the order of pairs, and the sums of their groups
    // The four lanes of a row read 64 bytes side by side: a pass's pieces stand word by word, lane by lane.  The pieces of all tokens have one running index; those
    // of a group are neighbours in a warp.
    const int pieces = n_blocks * 16, all = pieces * tokens, last_piece = (int)min((int64_t)pieces, (P.K - (int64_t)b_lo * kBlock) / 8);
    const auto each_piece = [&](auto f) {                               // f(the piece, its token, its place in the token's row, whether there is one)
        int v = 0, i = tid;
        const __nv_bfloat16* src = P.x + m0 * P.ldx + (int64_t)b_lo * kBlock + tid * 8;
        const auto settle = [&] {
            while (i >= pieces && v < tokens) { i -= pieces; src += P.ldx - pieces * 8; ++v; }
        };
        for (int f0 = 0; f0 < all; f0 += 4 * kThreads) {
            uint4 x[4];
            int pv[4], pi[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                settle();
                x[n] = v < tokens && i < last_piece ? *reinterpret_cast<const uint4*>(src) : make_uint4(0u, 0u, 0u, 0u);
                pv[n] = v;
                pi[n] = i;
                i += kThreads;
                src += kThreads * 8;
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) f(x[n], pv[n], pi[n], pv[n] < tokens);
        }
    };
    const auto put = [&](uint4 x, int v, int i, bool in, int e) {
        float sum;
        const uint4 o = operand_of_piece(x, e, sum);
#pragma unroll
        for (int w = 1; w < 16 / S; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        if (in) {
            const int pass = i / (16 / kPasses), lane_of = i % (16 / kPasses) / kWords, word = i % kWords;
            *reinterpret_cast<uint4*>(s_x + (size_t)v * x_stride + ((pass * kWords + word) * 4 + lane_of) * 16) = o;
            if (i % (16 / S) == 0) s_sum[pass * kCols + v * C + (C == 1 ? 0 : i % 16 / (16 / S))] = sum;
        }
    };
    __syncthreads();
    bool odd = false;
    each_piece([&](uint4 x, int v, int i, bool in) {
        odd |= unusual(x);
        put(x, v, i, in, kUsualExp);
    });
    const bool odd_sizes = __syncthreads_or(odd);
    if (odd_sizes) {                                                    // then each token by its largest magnitude
        each_piece([&](uint4 x, int v, int, bool in) {
            const uint32_t top = top_of_piece(x);
            if (in && top) atomicMax(&s_top[v], top);
        });
        __syncthreads();
        each_piece([&](uint4 x, int v, int i, bool in) { put(x, v, i, in, in ? scale_exponent(s_top[v]) : kUsualExp); });
        __syncthreads();
    }

    // Not before the tokens are here: what the next kernel fetches early would be in their way.
    let_next_kernel_start();

    // Column 8 nt + g of this lane's operands: a token's, in the lanes that have the column's group, or zero.
    const unsigned char* x_from[NT];
    int x_step[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int v = (8 * nt + g) / C;
        const bool some = v < tokens && (C == 1 || q * S / 4 == g % S);
        x_from[nt] = some ? s_x + (size_t)v * x_stride + kw * 256 + q * 16 : reinterpret_cast<const unsigned char*>(s_zero);
        x_step[nt] = some ? 256 * P.sk : 0;
    }
    const int part_floats = kWarps * kTile * (kCols + 1), buffer_floats = part_floats + rows * P.tokens;
    int at = 0, turn = 0, before = -1;                                  // before: the step whose sums are still with the CTAs of the cluster
    const auto gather = [&](int step, const float* part) {
        for (int i = (int)rank * kThreads + tid; i < rows * tokens; i += (int)cl * kThreads) {
            const int v = i >> rows_shift;
            float of[8], sum = 0.f;
#pragma unroll
            for (unsigned c = 0; c < 8; ++c) of[c] = c < cl ? ld_cluster(part + i, c) : 0.f;
#pragma unroll
            for (unsigned c = 0; c < 8; ++c) sum += of[c];
            store(P, m0 + v, (int64_t)step * rows + (i & (rows - 1)), sum);
        }
    };
    for (int step = blockIdx.y; step < P.steps; step += gridDim.y, turn ^= 1) {
        float y[MT][NT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[mt][nt][e] = 0.f;
        const unsigned char* x_at[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) x_at[nt] = x_from[nt];
        const float* sum_at = s_sum + kw * kPasses * kCols + 2 * q;
#pragma unroll 1
        for (int i = kw; i < n_blocks; i += P.sk) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
            __syncwarp();
            const unsigned char* slot = smem + (size_t)warp * kWarpRing + at;
            uint32_t w[2 * MT][4], gr[2 * MT][C == 1 ? S : 2];          // groups of the passes, or of columns 2 q and 2 q + 1
#pragma unroll
            for (int e = 0; e < 2 * MT; ++e) {
                const unsigned char* row = slot + (g + 8 * e) * kRow + q * (16 / kPasses);
                if constexpr (kPasses == 1) {
                    const uint4 v = *reinterpret_cast<const uint4*>(row);
                    w[e][0] = v.x; w[e][1] = v.y; w[e][2] = v.z; w[e][3] = v.w;
                } else if constexpr (kPasses == 2) {
                    const uint2 v = *reinterpret_cast<const uint2*>(row), u = *reinterpret_cast<const uint2*>(row + 32);
                    w[e][0] = v.x; w[e][1] = v.y; w[e][2] = u.x; w[e][3] = u.y;
                } else {
#pragma unroll
                    for (int s = 0; s < 4; ++s) w[e][s] = *reinterpret_cast<const uint32_t*>(row + 16 * s);
                }
                const unsigned char* of_row = slot + kCodes + (g + 8 * e) * (4 * S);
                if constexpr (C == 1) {
#pragma unroll
                    for (int s = 0; s < S; ++s) gr[e][s] = *reinterpret_cast<const uint32_t*>(of_row + 4 * s);
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(of_row + (S == 4 ? 8 * (q & 1) : 0));
                    gr[e][0] = v.x; gr[e][1] = v.y;
                }
            }
            at = at == (kDepth - 1) * kSlot ? 0 : at + kSlot;
            fetch();                                                    // into the slot that was read one block ago
#pragma unroll
            for (int s = 0; s < kPasses; ++s) {
                constexpr int kChains = MT * NT * kPasses == 1 ? 2 : 1;       // sums that do not wait for one another
                float acc[kChains][MT][NT][4];
#pragma unroll
                for (int j = 0; j < kWords; ++j) {
                    uint4 xv[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) xv[nt] = *reinterpret_cast<const uint4*>(x_at[nt] + 64 * (s * kWords + j));
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const uint32_t a = w[2 * mt][s * kWords + j], b = w[2 * mt + 1][s * kWords + j], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if (j == 0) mma_bf16_first(acc[0][mt][nt], a & 0x000f000fu, b & 0x000f000fu, a & 0x00f000f0u, b & 0x00f000f0u, xv[nt].x, xv[nt].y);
                            else mma_bf16(acc[0][mt][nt], a & 0x000f000fu, b & 0x000f000fu, a & 0x00f000f0u, b & 0x00f000f0u, xv[nt].x, xv[nt].y);
                            if (j == 0 && kChains == 2) mma_bf16_first(acc[kChains - 1][mt][nt], a8 & 0x000f000fu, b8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x00f000f0u, xv[nt].z, xv[nt].w);
                            else mma_bf16(acc[kChains - 1][mt][nt], a8 & 0x000f000fu, b8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x00f000f0u, xv[nt].z, xv[nt].w);
                        }
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float2 sum = *reinterpret_cast<const float2*>(sum_at + s * kCols + 8 * nt);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t group = gr[2 * mt + (e >> 1)][C == 1 ? s : e & 1];
                            const float v = kChains == 2 ? acc[0][mt][nt][e] + acc[kChains - 1][mt][nt][e] : acc[0][mt][nt][e];
                            y[mt][nt][e] = fmaf(scale_of(group), v, fmaf(low_of(group), (e & 1) ? sum.y : sum.x, y[mt][nt][e]));
                        }
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) x_at[nt] += x_step[nt];
            sum_at += P.sk * kPasses * kCols;
        }
        // ---- sums over the warps that share a row tile, the columns of a token and the CTAs of the cluster, each in a fixed order
        float* red = s_red + turn * buffer_floats;                      // [kw][row][columns]; then [token][row]
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = 8 * nt + 2 * q + (e & 1);
                    if (c < tokens * C) red[(kw * rows + rt * kTile + 16 * mt + g + 8 * (e >> 1)) * (kCols + 1) + c] = from_units(y[mt][nt][e], odd_sizes ? scale_exponent(s_top[c / C]) : kUsualExp);
                }
        __syncthreads();
        float* part = red + part_floats;
        // The CTAs of the cluster meet a step late, so that none waits for another while it has blocks to multiply.  That all of them have come this far says that they
        // have gathered the sums of the step before the last, whose place these take.
        if (cl > 1 && before >= 0) cluster_wait();
        for (int i = tid; i < rows * tokens; i += kThreads) {
            const int v = i >> rows_shift, r = i & (rows - 1);
            float sum = 0.f;
            for (int w = 0; w < P.sk; ++w)
#pragma unroll
                for (int s = 0; s < C; ++s) sum += red[(w * rows + r) * (kCols + 1) + v * C + s];
            if (cl > 1) part[i] = sum;
            else store(P, m0 + v, (int64_t)step * rows + r, sum);
        }
        if (cl > 1) {
            if (before >= 0) gather(before, s_red + (turn ^ 1) * buffer_floats + part_floats);
            cluster_arrive();
            before = step;
        }
    }
    if (cl > 1) {
        if (before >= 0) {
            cluster_wait();
            gather(before, s_red + (turn ^ 1) * buffer_floats + part_floats);
        }
        cluster_arrive();                                               // no CTA leaves while another reads its sums
        cluster_wait();
    }
}

struct GemvPlan {
    int nt, mt, cl, sk, rw, slice;
    int64_t tokens, steps, row_ctas, token_blocks;
    size_t smem;
    double cost;
};

inline int columns_of(int64_t M, int S) { return M * S <= 8 ? S : 1; }

inline size_t gemv_smem(int64_t tokens, int64_t slice, int S, int passes, int nt, int mt, int rw) {
    const size_t warps = warps_of(nt), ring = warps * depth_of(nt, mt) * mt * (16 * row_bytes_of(passes) + 64 * S), stage = (size_t)tokens * (slice * 256 + 64) + (size_t)slice * passes * nt * 8 * 4;
    const size_t join = 2 * (warps * 16 * mt * (nt * 8 + 1) + (size_t)tokens * 16 * mt * rw) * 4;
    return ring + stage + join;
}

constexpr size_t kSmemOne = 224 * 1024;
// CTAs on an SM
inline int on_an_sm(int nt, size_t smem) { return ctas_of(nt) == 2 && 2 * (smem + 1536) <= 227 * 1024 ? 2 : 1; }

// Shape of one choice of columns, cluster, warps per row tile and row tiles per warp, and what it costs (ns); false: it does not fit.  The constants are measurements:
// 3 us for a dependent launch and its end; the tokens' trip to memory and their staging; a block of 128 of a warp, which takes its chain of latencies, its share of
// the SM or its share of HBM, whichever is longest; the sums at the end of a step, and those of a cluster.
inline bool plan_shape(GemvPlan& p, int64_t M, int64_t N, int64_t K, int S, int sms) {
    const int64_t blocks = (K + kBlock - 1) / kBlock;
    const int warps = warps_of(p.nt), passes = S / columns_of(M, S);
    p.rw = warps / p.sk;
    p.slice = (int)((blocks + p.cl - 1) / p.cl);
    p.smem = gemv_smem(p.tokens, p.slice, S, passes, p.nt, p.mt, p.rw);
    if (p.smem > kSmemOne || p.cl > blocks) return false;
    p.token_blocks = (M + p.tokens - 1) / p.tokens;
    const int rows = 16 * p.mt * p.rw, per_sm = on_an_sm(p.nt, p.smem);
    p.steps = (N + rows - 1) / rows;
    const int64_t slots = (int64_t)sms * per_sm / p.cl;
    p.row_ctas = slots / p.token_blocks < 1 ? 1 : slots / p.token_blocks;
    if (p.row_ctas > p.steps) p.row_ctas = p.steps;
    const double busy = (double)p.row_ctas * p.token_blocks * p.cl, most = (double)slots * p.cl, at_work = busy < most ? busy : most;
    const double rounds = (double)((p.steps + p.row_ctas - 1) / p.row_ctas) * (busy / at_work);
    const double on_sm = at_work <= sms ? 1 : per_sm, tile = p.mt * p.nt * (S == 1 ? 1.0 : passes == 1 ? 1.15 : 1.0 + 0.1 * passes * p.mt);
    const double alone = 85 + 150 * tile, shared = (100 + 260 * tile) * warps * on_sm / 16, hbm = (double)p.mt * (1024 + 64 * S) * warps * at_work / 6300.0 * (p.mt == 2 && p.sk == 1 && per_sm == 2 ? 1.6 : 1.0);
    // (32 rows of 64 bytes at a time and nobody at the rows' next bytes: 65536 x 2304 in 26 us, with two warps to a row 20.5)
    double block = alone > shared ? alone : shared;
    if (hbm > block) block = hbm;
    const int64_t trips = (p.tokens * p.slice + 8 * warps - 1) / (8 * warps);          // a thread has four of a block's sixteen pieces on their way at a time
    const double stage = 200 + 600.0 * trips + (at_work > sms ? 700 * (at_work - sms) / sms : 0), sums = 500 + 60.0 * rows * p.tokens / (32 * warps) + 50 * p.sk * (S / passes) + (p.cl > 1 ? 500 + 200 * p.cl : 0);
    p.cost = 2000 + stage + rounds * ((double)((p.slice + p.sk - 1) / p.sk) * block + sums);
    return true;
}

inline GemvPlan plan_gemv(int64_t M, int64_t N, int64_t K, int S, int sms) {
    GemvPlan best, p;
    best.cost = -1;
    for (p.nt = 1; p.nt <= 4; p.nt *= 2) {
        if (p.nt > 1 && M <= 4 * p.nt) break;                        // half as many columns would do
        p.tokens = p.nt * 8 < M ? p.nt * 8 : M;
        for (p.mt = 1; p.mt <= (p.nt < 4 ? 2 : 1); ++p.mt)
            for (p.cl = 1; p.cl <= 8; p.cl *= 2)
                for (p.sk = 1; p.sk <= warps_of(p.nt); p.sk *= 2)
                    if (plan_shape(p, M, N, K, S, sms) && (best.cost < 0 || p.cost < best.cost)) best = p;
    }
    return best;
}

inline bool has_grid(const GemvPlan& p) { return p.cost >= 0 && p.token_blocks <= 65535; }
inline int size_error(int64_t N, int64_t K, int group) {
    if (N < 0 || K < 0) return MATQ_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return MATQ_ERR_UNSUPPORTED;
    return K == 0 || K % group != 0 || K > 65536 || N >= (1ll << 31) ? MATQ_ERR_SHAPE : MATQ_OK;
}

template <int NT, int S, int C, int MT>
int launch_gemv(const GemvPlan& p, const GemvParams& P, cudaStream_t s) {
    static std::atomic<unsigned long long> smem_ok{0};
    if (!opt_in_max_smem(gemv_groups_kernel<NT, S, C, MT>, smem_ok)) return MATQ_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.cl, (unsigned)p.row_ctas, (unsigned)p.token_blocks);
    cfg.blockDim = dim3(32 * warps_of(NT));
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.cl;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, gemv_groups_kernel<NT, S, C, MT>, P) != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}

template <int S>
int launch_gemv_s(const GemvPlan& p, const GemvParams& P, cudaStream_t s) {
    if (S > 1 && columns_of(P.M, S) == S) return p.mt == 1 ? launch_gemv<1, S, S, 1>(p, P, s) : launch_gemv<1, S, S, 2>(p, P, s);
    if (p.nt == 4) return launch_gemv<4, S, 1, 1>(p, P, s);
    if (p.mt == 1) return p.nt == 1 ? launch_gemv<1, S, 1, 1>(p, P, s) : launch_gemv<2, S, 1, 1>(p, P, s);
    return p.nt == 1 ? launch_gemv<1, S, 1, 2>(p, P, s) : launch_gemv<2, S, 1, 2>(p, P, s);
}

}  // namespace grp
}  // namespace matq

extern "C" int matq_quantize_groups(const void* W, int64_t N, int64_t K, int64_t ldw, int group, uint8_t* packed, void* params, int32_t* dev_status, void* stream) {
    using namespace matq;
    using namespace matq::grp;
    if (N < 0 || K < 0) return MATQ_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return MATQ_ERR_UNSUPPORTED;
    if (K == 0 || K % group != 0 || ldw < K || ldw % 8 != 0 || K >= (1ll << 31) || N >= (1ll << 31) || N * (K / 8) >= (1ll << 41)) return MATQ_ERR_SHAPE;
    if (N == 0) return MATQ_OK;
    if (!W || !packed || !params) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(W) || !aligned16(packed) || !aligned16(params)) return MATQ_ERR_ALIGNMENT;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = group == 32 ? launch_quantize<32>(W, N, K, ldw, packed, params, dev_status, s)
                          : group == 64 ? launch_quantize<64>(W, N, K, ldw, packed, params, dev_status, s) : launch_quantize<128>(W, N, K, ldw, packed, params, dev_status, s);
    if (e != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}

extern "C" int matq_gemv_groups_plan(int64_t M, int64_t N, int64_t K, int group, int* tokens, int* parts, int* steps) {
    using namespace matq;
    using namespace matq::grp;
    const int st = size_error(N, K, group);
    if (st != MATQ_OK) return st;
    if (M < 1 || N < 1) return MATQ_ERR_INVALID_ARG;
    const GemvPlan p = plan_gemv(M, N, K, kBlock / group, sm_count());
    if (!has_grid(p)) return MATQ_ERR_SHAPE;
    if (tokens) *tokens = (int)p.tokens;
    if (parts) *parts = p.cl;
    if (steps) *steps = (int)((p.steps + p.row_ctas - 1) / p.row_ctas);
    return MATQ_OK;
}

extern "C" int matq_gemv_groups(const uint8_t* packed, int64_t N, int64_t K, int group, const void* params, const void* x, int64_t M, int64_t ldx,
                                int out_type, void* y, int64_t ldy, unsigned flags, void* stream) {
    using namespace matq;
    using namespace matq::grp;
    if (M < 0 || (out_type != MATQ_OUT_F32 && out_type != MATQ_OUT_BF16) || (flags & ~(unsigned)MATQ_GEMV_PDL)) return MATQ_ERR_INVALID_ARG;
    const int st = size_error(N, K, group);
    if (st != MATQ_OK) return st;
    if (ldx < K || ldx % 8 != 0 || ldy < N) return MATQ_ERR_SHAPE;
    if (M == 0 || N == 0) return MATQ_OK;
    if (!packed || !params || !x || !y) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(packed) || !aligned16(params) || !aligned16(x)) return MATQ_ERR_ALIGNMENT;
    const int S = kBlock / group;
    static thread_local Recent<GemvPlan, 5> recent;
    const int sms = sm_count();
    const GemvPlan& p = recent.of({M, N, K, S, sms}, [&] { return plan_gemv(M, N, K, S, sms); });
    if (!has_grid(p)) return MATQ_ERR_SHAPE;
    GemvParams P;
    P.packed = packed; P.params = static_cast<const uint32_t*>(params); P.x = static_cast<const __nv_bfloat16*>(x); P.y = y;
    P.N = N; P.K = K; P.M = M; P.ldx = ldx; P.ldy = ldy; P.groups = K / group;
    P.tokens = (int)p.tokens; P.sk = p.sk; P.rw = p.rw; P.slice = p.slice; P.steps = (int)p.steps;
    P.early = (flags & MATQ_GEMV_PDL) != 0; P.out_bf16 = out_type == MATQ_OUT_BF16;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return S == 1 ? launch_gemv_s<1>(p, P, s) : S == 2 ? launch_gemv_s<2>(p, P, s) : launch_gemv_s<4>(p, P, s);
}
