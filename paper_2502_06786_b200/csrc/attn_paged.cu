// matq_attn_paged: attention of new tokens over a paged cache (argument checks, choice of kernel and split).
#include "attn_chunk.cuh"
#include "attn_decode.cuh"

namespace matq {
namespace attn {

constexpr int64_t kMaxKeys = (1ll << 31) - 1;                           // lengths are 32-bit numbers

struct Plan {
    int kind;                    // 1, 2: attn_chunk with so many query tiles of 128 rows per CTA; 8, 16: attn_decode with so many rows
    int keys, value_keys;        // keys of a step (the parts of the key range are multiples of it) and of a ring stage of values
    int64_t tiles_per_seq, splits, split_keys;
    double cost;
};

// Kernel and split of one kind from sizes that the host knows, and what they cost (ns).
inline Plan plan_kind(int kind, int batch, int kv_heads, int group, int D, int64_t max_q, int64_t max_kv, int64_t window, int sms) {
    Plan p;
    const int64_t rows = max_q * group;
    p.kind = kind;
    const bool decode = kind >= 8;
    const int keys = p.keys = decode ? (D == 256 ? 32 : 64) : 128;
    p.value_keys = !decode && D == 256 ? ChunkCfg<256, 1>::kStageKeys : keys;
    const int64_t tok = decode ? 0 : (int64_t)(128 / group) * kind;     // tokens per CTA
    p.tiles_per_seq = decode ? (rows + kind - 1) / kind : (max_q + tok - 1) / tok;
    if (p.tiles_per_seq < 1) p.tiles_per_seq = 1;
    int64_t range = max_kv;                                             // keys that a tile can see
    if (window > 0 && window < range && window + tok + 16 < range) range = window + tok + 16;
    range = (range + keys - 1) / keys + 1;                              // steps; one more when the window starts inside one
    // Parts of the key range: the number whose rounds over the SMs cost least.  Measured, ns: a step of the 128-row kernels; a stage of the few-row kernels
    // takes its bytes' time at 45 GB/s per SM or at the share of HBM that the CTAs at work leave each other (and with 16 rows no less than 500), but 250 while
    // the ring is filled for the first time;
    // about 2 us until the first step and after the last (6 for the 128-row kernels); 3 us for the join, and its bytes.  Sequences of a batch differ: without a
    // window their lengths are taken to average 0.6 of the longest.  More CTAs at work than SMs end half a part after the even share, on average.
    const double ctas = (double)p.tiles_per_seq * batch * kv_heads, row_bytes = ctas * (decode ? kind : 128 * kind) * D * 8;
    const int64_t bytes = (int64_t)keys * D * 4, ring = decode ? 192 * 1024 / bytes : 0;
    int64_t splits = 1;
    p.cost = -1;
    const double mean = batch > 1 ? (window > 0 && window < max_kv ? 0.9 : 0.6) : 1.0;
    for (int64_t n = 1; n <= kMaxSplits && n <= range; ++n) {
        const double busy = ctas * (n * mean > 1.0 ? n * mean : 1.0), at_work = busy < sms ? busy : sms;      // CTAs with keys
        const double share = bytes * at_work / 6300.0, first = share > 250 ? share : 250;
        const double alone = kind == 16 && bytes / 45.0 < 500 ? 500 : bytes / 45.0, later = share > alone ? share : alone;
        const int64_t steps = (range + n - 1) / n;                      // of the longest part
        const double step_ns = kind == 2 ? 1900 : D == 256 ? 2400 : 1400;
        const double part = decode ? (steps < ring ? steps : ring) * first + (steps > ring ? steps - ring : 0) * later + 2000 : steps * step_ns + 6000;
        const double all = part * busy / sms * (n * mean > 1.0 ? 1.0 : mean);        // the even share (unsplit: of parts of mean length)
        const double cost = (busy <= sms ? part : all + part / 2) + (n > 1 ? 3000 + row_bytes * n / 5000.0 : 0);
        if (p.cost < 0 || cost < p.cost) { p.cost = cost; splits = n; }
        if (ctas * n >= 6 * sms) break;
    }
    const int64_t per = (range + splits - 1) / splits;
    p.splits = (range + per - 1) / per;
    p.split_keys = per * keys;
    return p;
}

// Up to 16 rows per sequence and key head: the few-row kernel (16 sequences of 4 drafted tokens, 32/8 heads, windows of 4096 keys, D = 64, 128, 256: 34, 46, 82
// us; the 128-row kernel 48, 51, 87).  More: one or two query tiles of 128 rows per CTA, or tiles of 16 rows as long as all of them are at work at once,
// whichever costs less.  Tiles of 16 read the keys more often, but a CTA of theirs starts and ends 3 us sooner (300 tokens over 600, 6 heads of 64 on one key head:
// 9.0 us, in tiles of 128 rows 13.1; over 2800 20.3 and 22.1; 240 rows over 2560 keys of 4 heads of 128: 18.7 and 15.4).  With D = 256 they do not (32 rows over
// 600 keys: 13.8 and 13.9 us; 64 rows of 4 sequences 24.3 and 14.7).
inline Plan plan(int64_t T, int batch, int kv_heads, int group, int D, int64_t max_q, int64_t max_kv, int64_t window, int sms, bool half) {
    if (max_q > T) max_q = T;
    if (max_kv > kMaxKeys) max_kv = kMaxKeys;
    window = window_of(window);
    const int64_t rows = max_q * group;
    if (rows <= 16 && !half) return plan_kind(rows <= 8 ? 8 : 16, batch, kv_heads, group, D, max_q, max_kv, window, sms);
    const Plan one = plan_kind(1, batch, kv_heads, group, D, max_q, max_kv, window, sms);
    if (D == 256) return one;
    Plan best = one;
    if (rows > 128) {
        const Plan two = plan_kind(2, batch, kv_heads, group, D, max_q, max_kv, window, sms);
        if (two.cost <= best.cost) best = two;
    }
    if (half) return best;                                              // only the 128-row kernels take fp16
    const Plan few = plan_kind(16, batch, kv_heads, group, D, max_q, max_kv, window, sms);
    if ((double)few.tiles_per_seq * batch * kv_heads <= sms && few.cost < best.cost) best = few;
    return best;
}

inline size_t part_bytes(int64_t T, int q_heads, int D, int64_t splits) {
    return splits > 1 ? (size_t)splits * T * q_heads * (D + 2) * sizeof(float) : 0;
}

inline bool cache_map(CUtensorMap* tm, const void* base, int64_t rows, int D, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)D * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    return tc::make_map(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box);
}

// queries as [token][head][D]: a box is 64 columns of the heads of a group for the tokens of a tile
inline bool query_map(CUtensorMap* tm, const void* q, int64_t T, int q_heads, int D, int64_t ldq, int group) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)q_heads, (cuuint64_t)T};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)ldq * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)(128 / group)};
    return tc::make_map(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, q, dims, strides, box);
}

template <int D, int NT>
int launch_decode(const CUtensorMap& tk, const CUtensorMap& tv, const Params& P, unsigned grid, cudaStream_t s) {
    using C = DecCfg<D, NT>;
    static std::atomic<unsigned long long> smem_ok{0};
    if (!opt_in_max_smem(attn_decode_kernel<D, NT>, smem_ok)) return MATQ_ERR_CUDA;
    if (launch_overlapped(attn_decode_kernel<D, NT>, dim3(grid), dim3(C::kThreads), C::kSmem, s, tk, tv, P) != cudaSuccess) {
        cudaGetLastError();
        return MATQ_ERR_CUDA;
    }
    return MATQ_OK;
}

template <int D, int TILES, bool CAP>
int launch_chunk(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const Params& P, unsigned grid, cudaStream_t s) {
    using C = ChunkCfg<D, TILES>;
    static std::atomic<unsigned long long> smem_ok{0};
    if (!opt_in_max_smem(attn_chunk_kernel<D, TILES, CAP>, smem_ok)) return MATQ_ERR_CUDA;
    if (launch_overlapped(attn_chunk_kernel<D, TILES, CAP>, dim3(grid), dim3(C::kThreads), C::kSmem, s, tq, tk, tv, P) != cudaSuccess) {
        cudaGetLastError();
        return MATQ_ERR_CUDA;
    }
    return MATQ_OK;
}

template <int D>
int launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const Params& P, int kind, unsigned grid, cudaStream_t s) {
    int st;
    if (kind == 8) {
        st = launch_decode<D, 1>(tk, tv, P, grid, s);
    } else if (kind == 16) {
        st = launch_decode<D, 2>(tk, tv, P, grid, s);
    } else if (kind == 1) {
        st = P.softcap > 0.f ? launch_chunk<D, 1, true>(tq, tk, tv, P, grid, s) : launch_chunk<D, 1, false>(tq, tk, tv, P, grid, s);
    } else {
        if constexpr (D <= 128) st = P.softcap > 0.f ? launch_chunk<D, 2, true>(tq, tk, tv, P, grid, s) : launch_chunk<D, 2, false>(tq, tk, tv, P, grid, s);
        else st = MATQ_ERR_UNSUPPORTED;
    }
    if (st != MATQ_OK) return st;
    if (P.splits > 1 && (st = launch_join<D>(P, s)) != MATQ_OK) return st;
    return launch_status();
}

}  // namespace attn
}  // namespace matq

size_t matq::attn::paged_workspace_bytes(int64_t T, int batch, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv, int64_t window, bool half) {
    if (T <= 0 || batch <= 0 || q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads != 0 || q_heads / kv_heads > 64 || head_dim <= 0 || max_q < 0 || max_kv < 0) return 0;
    const Plan p = plan(T, batch, kv_heads, q_heads / kv_heads, head_dim, max_q, max_kv, window, matq::sm_count(), half);
    return part_bytes(T, q_heads, head_dim, p.splits);
}

double matq::attn::paged_cost(int64_t T, int batch, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv, int64_t window, int* tiles, int* parts) {
    const Plan p = plan(T, batch, kv_heads, q_heads / kv_heads, head_dim, max_q, max_kv, window, matq::sm_count(), true);
    if (tiles) *tiles = p.kind;
    if (parts) *parts = (int)p.splits;
    return p.cost;
}

extern "C" size_t matq_attn_paged_workspace_bytes(int64_t T, int batch, int q_heads, int kv_heads, int head_dim,
                                                  int64_t max_q, int64_t max_kv, int64_t window) {
    return matq::attn::paged_workspace_bytes(T, batch, q_heads, kv_heads, head_dim, max_q, max_kv, window, false);
}

int matq::attn::paged(const matq_paged_kv* cache, int64_t T, const void* q, int q_heads, int64_t ldq, float scale, float softcap, int64_t window, int64_t max_q,
                      int64_t max_kv, void* out, int64_t ldo, void* workspace, size_t workspace_bytes, const Half* half, int32_t* dev_status, void* stream) {
    if (!cache || T < 0 || q_heads < 1 || cache->batch < 0 || cache->n_pages < 0 || cache->kv_heads < 1 || cache->table_width < 0 || (cache->batch > 1 && cache->table_stride < cache->table_width) ||
        window < 0 || max_q < 0 || max_kv < 0 || !(softcap >= 0.f) || !(scale > 0.f))
        return MATQ_ERR_INVALID_ARG;
    const int D = cache->head_dim, ps = cache->page_size;
    if (D != 64 && D != 128 && D != 256) return MATQ_ERR_UNSUPPORTED;
    if (ps != 16 && ps != 32 && ps != 64 && ps != 128 && ps != 256) return MATQ_ERR_UNSUPPORTED;
    if (q_heads % cache->kv_heads != 0 || q_heads / cache->kv_heads > 64) return MATQ_ERR_UNSUPPORTED;
    const int64_t w = (int64_t)q_heads * D;
    if (ldq < w || ldq % 8 != 0 || ldo < w || ldo % 8 != 0 || T >= (1ll << 31) || cache->n_pages > kMaxKeys / ((int64_t)cache->kv_heads * ps)) return MATQ_ERR_SHAPE;
    const int64_t rows = cache->n_pages * cache->kv_heads * ps;
    if (T == 0 || cache->batch == 0) return MATQ_OK;
    if (!q || !out || !cache->k || !cache->v || !cache->page_table || !cache->cu_q || !cache->kv_len || cache->n_pages == 0) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !aligned16(cache->k) || !aligned16(cache->v) || !aligned16(workspace)) return MATQ_ERR_ALIGNMENT;
    const int group = q_heads / cache->kv_heads;
    const Plan p = plan(T, cache->batch, cache->kv_heads, group, D, max_q, max_kv, window, sm_count(), half != nullptr);
    const double ctas = (double)p.splits * cache->kv_heads * cache->batch * p.tiles_per_seq;
    if (ctas >= 2147483648.0 || (p.splits > 1 && T * q_heads >= (1ll << 31))) return MATQ_ERR_SHAPE;
    if (part_bytes(T, q_heads, D, p.splits) > workspace_bytes || (p.splits > 1 && !workspace)) return MATQ_ERR_WORKSPACE;

    Params P;
    P.q = static_cast<const __nv_bfloat16*>(q); P.v = static_cast<const __nv_bfloat16*>(cache->v); P.out = static_cast<__nv_bfloat16*>(out);
    P.table = cache->page_table; P.cu_q = cache->cu_q; P.kv_len = cache->kv_len;
    P.ldq = ldq; P.ldo = ldo; P.table_stride = cache->table_stride; P.table_width = cache->table_width; P.n_pages = cache->n_pages; P.T = T; P.window = window_of(window); P.above_rows = half ? half->above_rows : 0;
    P.batch = cache->batch; P.q_heads = q_heads; P.kv_heads = cache->kv_heads; P.group = group;
    P.page_size = ps; P.page_shift = ps == 16 ? 4 : ps == 32 ? 5 : ps == 64 ? 6 : ps == 128 ? 7 : 8;
    P.tiles_per_seq = (int)p.tiles_per_seq; P.splits = (int)p.splits; P.split_keys = p.split_keys;
    // From 2^100 on a cap is none: it leaves scores below 2^88 as they are in fp32, and larger ones are further apart than any weight reaches either way.
    P.scale = scale; P.softcap = softcap < 0x1p100f ? softcap : 0.f;
    P.part_o = static_cast<float*>(workspace);
    P.part_ml = reinterpret_cast<float2*>(P.part_o + (size_t)p.splits * T * q_heads * D);
    P.dev_status = dev_status;
    P.filter = P.above_rows > 0 ? 1 : 0;
    P.join_above = 1;
    P.q_scale = half ? half->q_scale : nullptr; P.k_scale = half ? half->k_scale : nullptr; P.v_scale = half ? half->v_scale : nullptr;
    P.hold = tc::test_stall() ? 1 : 0;
    P.wait_cycles = P.hold ? tc::kStallWaitCycles : tc::kWaitCycles;
    const unsigned grid = (unsigned)ctas;
    CUtensorMap tq, tk, tv;
    const int box_k = ps < p.keys ? ps : p.keys, box_v = ps < p.value_keys ? ps : p.value_keys;
    if (!cache_map(&tk, cache->k, rows, D, box_k) || !cache_map(&tv, cache->v, rows, D, box_v) || !query_map(&tq, q, T, q_heads, D, ldq, group)) return MATQ_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (half) {
        int st = launch_chunk_half(D, p.kind, tq, tk, tv, P, grid, s);
        if (st == MATQ_OK && P.splits > 1) st = D == 64 ? launch_join<64>(P, s) : D == 128 ? launch_join<128>(P, s) : launch_join<256>(P, s);
        return st == MATQ_OK ? launch_status() : st;
    }
    if (D == 64) return launch<64>(tq, tk, tv, P, p.kind, grid, s);
    if (D == 128) return launch<128>(tq, tk, tv, P, p.kind, grid, s);
    return launch<256>(tq, tk, tv, P, p.kind, grid, s);
}

extern "C" int matq_attn_paged(const matq_paged_kv* cache, int64_t T, const void* q, int q_heads, int64_t ldq, float scale, float softcap,
                               int64_t window, int64_t max_q, int64_t max_kv, void* out, int64_t ldo, void* workspace,
                               size_t workspace_bytes, int32_t* dev_status, void* stream) {
    return matq::attn::paged(cache, T, q, q_heads, ldq, scale, softcap, window, max_q, max_kv, out, ldo, workspace, workspace_bytes, nullptr, dev_status, stream);
}
