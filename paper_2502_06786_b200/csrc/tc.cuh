// Barrier, bulk-copy and tensor-core helpers shared by the serving kernels (gemm_a8.cu, attn_*.cuh).
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace matq {
namespace tc {

constexpr long long kWaitCycles = 4000000000ll;     // SM clock cycles after which a wait gives up: about two seconds
constexpr long long kStallWaitCycles = 2000000ll;   // the same under matq_serving_test_stall: about a millisecond

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Bounded in SM clock cycles (the clock is read once per 64 polls; the first reading starts the count).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, long long limit) {
    uint32_t done = 0;
    long long t0 = 0;
    for (uint32_t it = 0; !done; ++it) {
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (!done && (it & 63u) == 63u) {
            const long long now = clock64();
            if (t0 == 0) t0 = now;
            else if (now - t0 > limit) break;
        }
    }
    return done != 0;
}

// A two-dimensional tile; x (elements along the contiguous axis) must start on a 16-byte boundary, y may lie outside (reads as zero).
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// Shared-memory operand descriptor of a tile with 128-byte swizzle: rows of 128 bytes, atoms of 8 rows 1024 bytes apart (K-major operands;
// for an MN-major operand `lead` is the distance of neighbouring 128-byte columns of atoms).
__device__ __forceinline__ uint64_t sw128_desc(uint32_t smem_addr, uint32_t lead = 16, uint32_t stride = 1024) {
    return (uint64_t)((smem_addr >> 4) & 0x3fffu) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(stride >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 consecutive 32-bit columns of this thread's tensor-memory lane
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* d) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]), "=r"(d[4]), "=r"(d[5]), "=r"(d[6]), "=r"(d[7]),
                   "=r"(d[8]), "=r"(d[9]), "=r"(d[10]), "=r"(d[11]), "=r"(d[12]), "=r"(d[13]), "=r"(d[14]), "=r"(d[15]),
                   "=r"(d[16]), "=r"(d[17]), "=r"(d[18]), "=r"(d[19]), "=r"(d[20]), "=r"(d[21]), "=r"(d[22]), "=r"(d[23]),
                   "=r"(d[24]), "=r"(d[25]), "=r"(d[26]), "=r"(d[27]), "=r"(d[28]), "=r"(d[29]), "=r"(d[30]), "=r"(d[31])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* d) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]), "=r"(d[4]), "=r"(d[5]), "=r"(d[6]), "=r"(d[7]),
                   "=r"(d[8]), "=r"(d[9]), "=r"(d[10]), "=r"(d[11]), "=r"(d[12]), "=r"(d[13]), "=r"(d[14]), "=r"(d[15])
                 : "r"(addr) : "memory");
}
// The whole warp runs the loops that issue products, and one lane of it issues them: with the loop under `if (lane == 0)` slots and descriptors are
// computed per thread and moved to the uniform registers that tcgen05.mma reads, which takes about 120 cycles per product (64 is what one of 128 x 128 x 32 bytes takes).
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t e;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(e));
    return e;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, long long limit) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, limit)); }
// A from shared memory, or (TMEM_A) from tensor memory
#define MATQ_TC_MMA(GROUP, KIND, D, A, B, IDESC, ACCUMULATE, LEADER)                                                                       \
    asm volatile("{ .reg .pred p, e; setp.ne.b32 p, %4, 0; setp.ne.b32 e, %5, 0; @e tcgen05.mma.cta_group::" #GROUP ".kind::" KIND " [%0], %1, %2, %3, p; }" \
                 ::"r"(D), "l"(A), "l"(B), "r"(IDESC), "r"(ACCUMULATE), "r"(LEADER) : "memory")
#define MATQ_TC_MMA_TMEM_A(GROUP, KIND, D, A, B, IDESC, ACCUMULATE, LEADER)                                                                \
    asm volatile("{ .reg .pred p, e; setp.ne.b32 p, %4, 0; setp.ne.b32 e, %5, 0; @e tcgen05.mma.cta_group::" #GROUP ".kind::" KIND " [%0], [%1], %2, %3, p; }" \
                 ::"r"(D), "r"(A), "l"(B), "r"(IDESC), "r"(ACCUMULATE), "r"(LEADER) : "memory")
// arrives on a barrier of this CTA when every tcgen05.mma issued so far by this thread has ended
__device__ __forceinline__ void tc_commit(uint32_t bar, uint32_t leader) {
    asm volatile("{ .reg .pred e; setp.ne.b32 e, %1, 0; @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(bar), "r"(leader) : "memory");
}

// ---------------------------------------------------------------- host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

// Tile map with 128-byte swizzle: dims / box innermost first, strides (bytes) of the dimensions above the first; out of range reads as zero.
inline bool make_map(CUtensorMap* tm, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims,
                     const cuuint64_t* strides, const cuuint32_t* box) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(tm, type, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// matq_serving_test_stall (api.cu)
bool test_stall();

}  // namespace tc
}  // namespace matq
