// 4-bit weights with a scale and a low end per group of 32, 64 or 128 weights of a row: matq_quantize_groups and matq_gemv_groups.
#include "group4.cuh"

namespace matq {
namespace grp {

// ---------------------------------------------------------------- quantiser
// A thread takes eight weights, the threads of a group are neighbours in a warp and exchange its two ends by shuffles.  Groups follow one another without
// a gap, across the ends of rows too, so that codes and groups have one running index each.  Every weight is read once: HBM.
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
// With groups of 32 or 64 the four lanes that share a row hold 4 or 2 groups at a time.  Each group gets columns of its own: token m of group slot s is column
// m S + s, whose operand is zero in the lanes of the other slots (S = 128 / group).
//
// A CTA takes 16 RW rows and a part of K, staged in shared memory for its tokens; its warps are RW row tiles times SK parts of that part, block by block of 128;
// the CTAs of a cluster share K and add their sums through distributed shared memory, in rank order.  Bound: HBM (and the start of a launch).
constexpr int kBlock = 128, kWarps = 16, kThreads = 32 * kWarps;

struct GemvParams {
    const uint8_t* packed;
    const uint32_t* params;      // (scale, low) as two bf16, [N, K / group]
    const __nv_bfloat16* x;
    void* y;
    int64_t N, K, M, ldx, ldy, groups;       // groups of a row
    int tokens;                  // per CTA (a multiple goes to gridDim.z)
    int sk, rw;                  // sk * rw = kWarps
    int pass_blocks;             // blocks of 128 staged at a time, a multiple of the ring's turn
    int early;                   // codes and groups may be fetched before the wait
    int out_bf16;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(const float* p, unsigned rank) {
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

template <int NT, int S>
__global__ void __launch_bounds__(kThreads, 1) gemv_groups_kernel(const GemvParams P) {
    constexpr int kDepth = NT >= 4 ? 2 : 4, kSlots = S == 1 ? 1 : 2;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t s_top[32];           // largest magnitude per token (bits of a float)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
    const int rt = warp % P.rw, kw = warp / P.rw;
    const unsigned cl = gridDim.x, rank = blockIdx.x;                   // the cluster is the grid's x
    const int64_t blocks = (P.K + kBlock - 1) / kBlock;
    const int64_t b_lo = blocks * rank / cl, b_hi = blocks * (rank + 1) / cl;
    const int n_blocks = (int)(b_hi - b_lo);
    const int64_t row0 = (int64_t)blockIdx.y * (16 * P.rw), m0 = (int64_t)blockIdx.z * P.tokens;
    const int tokens = (int)min((int64_t)P.tokens, P.M - m0);
    const int64_t row_bytes = P.K / 2;

    // ---- this lane's rows: g and g + 8 of the warp's tile (past the end: the last row, whose sums are not stored)
    const int64_t r_a = min(row0 + rt * 16 + g, P.N - 1), r_b = min(row0 + rt * 16 + g + 8, P.N - 1);
    const uint8_t *w_a = P.packed + r_a * row_bytes + 16 * q, *w_b = P.packed + r_b * row_bytes + 16 * q;
    const uint32_t *p_a = P.params + r_a * P.groups, *p_b = P.params + r_b * P.groups;
    uint4 wa[kDepth], wb[kDepth];
    uint32_t pa[kDepth][kSlots], pb[kDepth][kSlots];
    const auto fetch = [&](int d, int i) {                              // block i of this CTA's part; past the end nothing is read
        const int64_t blk = b_lo + i;
        const bool in = i < n_blocks && blk * kBlock + 32 * q < P.K;
        wa[d] = in ? ld_stream_u4(w_a + blk * (kBlock / 2)) : make_uint4(0u, 0u, 0u, 0u);
        wb[d] = in ? ld_stream_u4(w_b + blk * (kBlock / 2)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int e = 0; e < kSlots; ++e) {
            // column 2 q + e belongs to slot (2 q + e) % S
            const int64_t at = blk * S + (S == 1 ? 0 : (2 * q + e) % S);
            const bool has = i < n_blocks && at < P.groups;
            pa[d][e] = has ? __ldg(p_a + at) : 0u;
            pb[d][e] = has ? __ldg(p_b + at) : 0u;
        }
    };
    if (!P.early) after_previous_kernel();
#pragma unroll
    for (int d = 0; d < kDepth; ++d) fetch(d, kw + d * P.sk);
    if (P.early) after_previous_kernel();
    let_next_kernel_start();

    // ---- shared memory: tokens [tokens][pass_blocks][256 bytes] (+ 64 bytes a token), sums per group [tokens][pass_blocks S], then the warps' results
    const int x_stride = P.pass_blocks * 256 + 64;
    float* s_sum = reinterpret_cast<float*>(smem + (size_t)P.tokens * x_stride);
    const int sum_stride = P.pass_blocks * S;
    float y[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[nt][e] = 0.f;
    // this lane's operand columns 8 nt + g, and whether its quarter of a block belongs to their slot
    const bool mine = (q * S) / 4 == g % S;

    for (int p0 = 0; p0 < n_blocks; p0 += P.pass_blocks) {
        const int here = min(P.pass_blocks, n_blocks - p0);             // blocks of this pass
        const int64_t k0 = (b_lo + p0) * kBlock;
        __syncthreads();                                                // the last pass is done with the stage
        if (tid < 32) s_top[tid] = 0u;
        __syncthreads();
        const int pieces = here * 16;                                   // of eight elements, per token
        for (int v = 0; v < tokens; ++v) {
            uint32_t top = 0u;
            for (int i = tid; i < pieces; i += kThreads) {
                const int64_t k = k0 + i * 8;
                if (k < P.K) top = max(top, top_of_piece(*reinterpret_cast<const uint4*>(P.x + (m0 + v) * P.ldx + k)));
            }
            top = __reduce_max_sync(0xffffffffu, top);
            if (lane == 0 && top) atomicMax(&s_top[v], top);
        }
        __syncthreads();
        for (int v = 0; v < tokens; ++v) {
            const int e = scale_exponent(s_top[v]);
            for (int base = 0; base < pieces; base += kThreads) {       // whole warps: the sums of a group go through shuffles
                const int i = base + tid;
                const int64_t k = k0 + (int64_t)i * 8;
                const bool in = i < pieces && k < P.K;
                const uint4 x = in ? *reinterpret_cast<const uint4*>(P.x + (m0 + v) * P.ldx + k) : make_uint4(0u, 0u, 0u, 0u);
                float sum;
                const uint4 o = operand_of_piece(x, e, sum);
#pragma unroll
                for (int w = 1; w < 16 / S; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
                if (i < pieces) {
                    // piece 4 q + j of a block goes to place 4 j + q: the four lanes of a row read 64 bytes side by side
                    const int at = (i & ~15) | ((i & 3) << 2) | ((i >> 2) & 3);
                    *reinterpret_cast<uint4*>(smem + (size_t)v * x_stride + at * 16) = o;
                    if ((i & (16 / S - 1)) == 0) s_sum[v * sum_stride + i / (16 / S)] = sum;
                }
            }
        }
        __syncthreads();

        float yp[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) yp[nt][e] = 0.f;
        for (int i0 = kw; i0 < here; i0 += kDepth * P.sk)
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            const int i = i0 + d * P.sk;
            if (i >= here) break;
            float acc[NT][2][4] = {};
            const uint32_t wra[4] = {wa[d].x, wa[d].y, wa[d].z, wa[d].w}, wrb[4] = {wb[d].x, wb[d].y, wb[d].z, wb[d].w};
            uint32_t gpa[kSlots], gpb[kSlots];
#pragma unroll
            for (int e = 0; e < kSlots; ++e) { gpa[e] = pa[d][e]; gpb[e] = pb[d][e]; }
            fetch(d, p0 + i + kDepth * P.sk);
            const unsigned char* xs = smem + i * 256 + q * 16;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = wra[j], b = wrb[j], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int v = (8 * nt + g) / S;
                    uint4 xv = make_uint4(0u, 0u, 0u, 0u);
                    if (mine && v < tokens) xv = *reinterpret_cast<const uint4*>(xs + (size_t)v * x_stride + j * 64);
                    mma_bf16(acc[nt][j & 1], a & 0x000f000fu, b & 0x000f000fu, a & 0x00f000f0u, b & 0x00f000f0u, xv.x, xv.y);
                    mma_bf16(acc[nt][j & 1], a8 & 0x000f000fu, b8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x00f000f0u, xv.z, xv.w);
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int c = 8 * nt + 2 * q + e, v = c / S;
                    const float sum = v < tokens ? s_sum[v * sum_stride + i * S + c % S] : 0.f;
                    const uint32_t ga = gpa[S == 1 ? 0 : e], gb = gpb[S == 1 ? 0 : e];
                    const float ra = (acc[nt][0][e] + acc[nt][1][e]) , rb = (acc[nt][0][2 + e] + acc[nt][1][2 + e]) ;
                    yp[nt][e] = fmaf(scale_of(ga), ra, fmaf(low_of(ga), sum, yp[nt][e]));
                    yp[nt][2 + e] = fmaf(scale_of(gb), rb, fmaf(low_of(gb), sum, yp[nt][2 + e]));
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = (8 * nt + 2 * q + (e & 1)) / S;
                y[nt][e] = v < tokens ? y[nt][e] + from_units(yp[nt][e], scale_exponent(s_top[v])) : 0.f;
            }
    }

    // ---- sums over the slots, the warps that share a row tile, and the CTAs of the cluster, each in a fixed order
    const int rows = 16 * P.rw, cols = NT * 8 + 1;
    float* red = reinterpret_cast<float*>(smem);                        // [kw][row][columns]
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) red[(size_t)(kw * rows + rt * 16 + g + 8 * (e >> 1)) * cols + 8 * nt + 2 * q + (e & 1)] = y[nt][e];
    __syncthreads();
    float* mine_sum = red + (size_t)P.sk * rows * cols;                 // [token][row]
    for (int i = tid; i < rows * tokens; i += kThreads) {
        const int v = i / rows, r = i - v * rows;
        float sum = 0.f;
        for (int w = 0; w < P.sk; ++w)
#pragma unroll
            for (int s = 0; s < S; ++s) sum += red[(size_t)(w * rows + r) * cols + v * S + s];
        mine_sum[i] = sum;
    }
    if (cl > 1) cluster_sync();
    else __syncthreads();
    for (int i = (int)rank * kThreads + tid; i < rows * tokens; i += (int)cl * kThreads) {
        const int v = i / rows;
        const int64_t r = row0 + i - v * rows;
        float sum = 0.f;
        if (cl == 1) sum = mine_sum[i];
        else
            for (unsigned c = 0; c < cl; ++c) sum += ld_cluster(mine_sum + i, c);
        if (r < P.N) {
            if (P.out_bf16) static_cast<__nv_bfloat16*>(P.y)[(m0 + v) * P.ldy + r] = __float2bfloat16_rn(sum);
            else static_cast<float*>(P.y)[(m0 + v) * P.ldy + r] = sum;
        }
    }
    if (cl > 1) cluster_sync();                                         // no CTA leaves while another reads its sums
}

struct GemvPlan {
    int nt, cl, sk, rw, pass_blocks;
    int64_t tokens, row_blocks, token_blocks;
    size_t smem;
};

inline size_t gemv_smem(int tokens, int pass_blocks, int S, int sk, int rw, int nt) {
    const size_t stage = (size_t)tokens * (pass_blocks * 256 + 64) + (size_t)tokens * pass_blocks * S * 4;
    const size_t join = ((size_t)sk * 16 * rw * (nt * 8 + 1) + (size_t)16 * rw * tokens) * 4;
    return stage > join ? stage : join;
}

inline GemvPlan plan_gemv(int64_t M, int64_t N, int64_t K, int S, int sms) {
    GemvPlan p;
    const int64_t blocks = (K + kBlock - 1) / kBlock, tiles = (N + 15) / 16;
    p.nt = M * S <= 8 ? 1 : M * S <= 16 ? 2 : 4;
    p.tokens = p.nt * 8 / S < M ? p.nt * 8 / S : M;
    p.token_blocks = (M + p.tokens - 1) / p.tokens;
    p.cl = 1;
    p.sk = 1;
    while (p.sk < kWarps && tiles * p.sk * p.token_blocks < (int64_t)sms * kWarps && blocks >= 2 * p.sk) p.sk *= 2;
    while (p.cl < 8 && ((tiles * p.sk + kWarps - 1) / kWarps) * p.cl * p.token_blocks < sms && blocks >= 4 * p.sk * p.cl) p.cl *= 2;
    int64_t most = (160 * 1024) / (p.tokens * (256 + 4 * S) + 1);        // blocks that fit
    const int64_t per = (blocks + p.cl - 1) / p.cl;
    if (most >= per) {
        most = per;
    } else {                                                            // a pass takes whole turns of the ring of prefetched blocks
        const int depth = p.nt >= 4 ? 2 : 4;
        while (p.sk > 1 && depth * p.sk > most) p.sk /= 2;
        most = most / (depth * p.sk) * (depth * p.sk);
    }
    p.rw = kWarps / p.sk;
    p.row_blocks = (tiles + p.rw - 1) / p.rw;
    p.pass_blocks = (int)most;
    p.smem = gemv_smem((int)p.tokens, p.pass_blocks, S, p.sk, p.rw, p.nt);
    return p;
}

template <int NT, int S>
int launch_gemv(const GemvPlan& p, const GemvParams& P, cudaStream_t s) {
    static std::atomic<unsigned long long> smem_ok{0};
    if (!opt_in_max_smem(gemv_groups_kernel<NT, S>, smem_ok)) return MATQ_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.cl, (unsigned)p.row_blocks, (unsigned)p.token_blocks);
    cfg.blockDim = dim3(kThreads);
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
    if (cudaLaunchKernelEx(&cfg, gemv_groups_kernel<NT, S>, P) != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}

template <int S>
int launch_gemv_s(const GemvPlan& p, const GemvParams& P, cudaStream_t s) {
    return p.nt == 1 ? launch_gemv<1, S>(p, P, s) : p.nt == 2 ? launch_gemv<2, S>(p, P, s) : launch_gemv<4, S>(p, P, s);
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

extern "C" int matq_gemv_groups(const uint8_t* packed, int64_t N, int64_t K, int group, const void* params, const void* x, int64_t M, int64_t ldx,
                                int out_type, void* y, int64_t ldy, unsigned flags, void* stream) {
    using namespace matq;
    using namespace matq::grp;
    if (N < 0 || K < 0 || M < 0 || (out_type != MATQ_OUT_F32 && out_type != MATQ_OUT_BF16) || (flags & ~(unsigned)MATQ_GEMV_PDL)) return MATQ_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && group != 128) return MATQ_ERR_UNSUPPORTED;
    if (K == 0 || K % group != 0 || K > 65536 || ldx < K || ldx % 8 != 0 || ldy < N || N >= (1ll << 31)) return MATQ_ERR_SHAPE;
    if (M == 0 || N == 0) return MATQ_OK;
    if (!packed || !params || !x || !y) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(packed) || !aligned16(params) || !aligned16(x)) return MATQ_ERR_ALIGNMENT;
    const int S = kBlock / group;
    const GemvPlan p = plan_gemv(M, N, K, S, sm_count());
    if (p.row_blocks > 65535 * 16ll || p.token_blocks > 65535) return MATQ_ERR_SHAPE;
    GemvParams P;
    P.packed = packed; P.params = static_cast<const uint32_t*>(params); P.x = static_cast<const __nv_bfloat16*>(x); P.y = y;
    P.N = N; P.K = K; P.M = M; P.ldx = ldx; P.ldy = ldy; P.groups = K / group;
    P.tokens = (int)p.tokens; P.sk = p.sk; P.rw = p.rw; P.pass_blocks = p.pass_blocks;
    P.early = (flags & MATQ_GEMV_PDL) != 0; P.out_bf16 = out_type == MATQ_OUT_BF16;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return S == 1 ? launch_gemv_s<1>(p, P, s) : S == 2 ? launch_gemv_s<2>(p, P, s) : launch_gemv_s<4>(p, P, s);
}
