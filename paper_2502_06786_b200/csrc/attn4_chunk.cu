// The 128-row attention kernels on fp16, for matq_attn_paged4 (a translation unit of its own: they take a minute to compile).
#include "attn_chunk.cuh"

namespace matq {
namespace attn {

template <int D, int TILES, bool CAP>
int launch_half(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const Params& P, unsigned grid, cudaStream_t s) {
    using C = ChunkCfg<D, TILES>;
    static std::atomic<unsigned long long> smem_ok{0};
    if (!opt_in_max_smem(attn_chunk_kernel<D, TILES, CAP, true>, smem_ok)) return MATQ_ERR_CUDA;
    if (launch_overlapped(attn_chunk_kernel<D, TILES, CAP, true>, dim3(grid), dim3(C::kThreads), C::kSmem, s, tq, tk, tv, P) != cudaSuccess) {
        cudaGetLastError();
        return MATQ_ERR_CUDA;
    }
    return MATQ_OK;
}

template <int D>
int launch_half_d(int tiles, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const Params& P, unsigned grid, cudaStream_t s) {
    if (tiles == 1) return P.softcap > 0.f ? launch_half<D, 1, true>(tq, tk, tv, P, grid, s) : launch_half<D, 1, false>(tq, tk, tv, P, grid, s);
    if constexpr (D <= 128) return P.softcap > 0.f ? launch_half<D, 2, true>(tq, tk, tv, P, grid, s) : launch_half<D, 2, false>(tq, tk, tv, P, grid, s);
    return MATQ_ERR_UNSUPPORTED;
}

int launch_chunk_half(int D, int tiles, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const Params& P, unsigned grid, cudaStream_t s) {
    return D == 64 ? launch_half_d<64>(tiles, tq, tk, tv, P, grid, s) : D == 128 ? launch_half_d<128>(tiles, tq, tk, tv, P, grid, s) : launch_half_d<256>(tiles, tq, tk, tv, P, grid, s);
}

}  // namespace attn
}  // namespace matq
