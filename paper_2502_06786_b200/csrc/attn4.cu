// matq_attn_paged4: attention of new tokens over a paged cache in 4-bit groups (argument checks, choice of kernels and split).
//
// Few rows per sequence and key head (single tokens, drafts) go to attn4_decode_kernel, which reads the cache as it is.  Sequences with more rows (chunks) are bound
// by their products: their keys and values are unpacked once, into the workspace, and the 128-row kernels of matq_attn_paged take them from there.  That is one
// more pass over what a chunk sees (read 9/16 of a byte an element, written and read 2), where unpacking inside the product kernel would be repeated by every query
// tile and compete with the softmax for the SM's issue slots.
//
// Unpacked to bf16 a key would be rounded to 8 bits once more, and scores with it (with a few large channels outputs were off by 4.6e-3 of their norm, 2.7 times
// what rounding them alone is).  fp16 keeps 11 bits.  Its range is made to suffice by powers of two: a query row is scaled by its largest element, the keys and the
// values of a sequence and head by the largest that their groups can stand for; scores and outputs are scaled back in fp32.
#include <cuda_fp16.h>

#include "attn4_decode.cuh"

namespace matq {
namespace attn {

constexpr int64_t kMost = (1ll << 31) - 1;                              // lengths are 32-bit numbers
constexpr int kUnpackPage = 256, kUnpackThreads = 256, kUnpackKeys = 64;
// Up to kDirectRows rows a call is served by the few-row kernel alone; above, sequences with more than kMixedRows are unpacked (a batch of one whatever it has).
constexpr int64_t kDirectRows = 64, kMixedRows = 16;
// Bytes of unpacked keys and values that a call's workspace holds at a time: sequences that do not fit together are served one round after another.
constexpr int64_t kUnpackBytes = 512ll << 20;
// Most bytes of partial outputs: they are indexed by the call's tokens, of which few may be of sequences that are split.
constexpr double kPartBytes = 256.0 * (1 << 20);

constexpr int kHalfExp = 14;             // the largest magnitudes come to lie in [2^14, 2^15)

struct Unpack {
    const uint8_t* tiles;
    const int32_t *table, *cu_q, *kv_len;
    int64_t table_stride, table_width, n_pages, window, above_rows;
    int batch, kv_heads, group, page_size;
    int64_t new_width;           // entries of a row of the new table
    int new_pages;               // pages of kUnpackPage keys per sequence
    int32_t* new_table;
    __half *k, *v;               // [batch * new_pages][kv_heads][kUnpackPage][D]
    uint32_t* top;               // [2][all sequences][kv_heads]: largest magnitudes, as the bits of floats
    float* scale;                // likewise: what to multiply with afterwards
    int64_t all, first_seq;      // sequences of the call; the first of this launch
    int32_t* dev_status;
};
// The keys that some new token of sequence b sees: [first, kv_len); false: the sequence is not for this call's unpacking.
struct Seen {
    int64_t first, kv_len;
};
__device__ __forceinline__ bool seen_keys(const Unpack& P, int b, Seen& s) {
    const int64_t n_new = (int64_t)P.cu_q[b + 1] - P.cu_q[b];
    s.kv_len = max(P.kv_len[b], 0);
    if (n_new <= 0 || n_new <= P.above_rows / P.group) return false;
    const int64_t ctx = s.kv_len - n_new;
    s.first = P.window && ctx - P.window + 1 > 0 ? ctx - P.window + 1 : 0;
    return s.kv_len > s.first;
}
__device__ __forceinline__ int half_exponent(uint32_t top) { return max((int)(top >> 23) - 127 - kHalfExp, -126); }        // what was taken off: 2^-126 .. 2^114

// Queries to fp16: a warp per token and head.  The kernel also clears the maxima for those that follow.  Bound: HBM.
template <int D>
__global__ void __launch_bounds__(kUnpackThreads) attn4_queries_kernel(const __nv_bfloat16* q, int64_t ldq, int64_t T, int q_heads, __half* to, float* scale, uint32_t* top, int64_t n_top) {
    after_previous_kernel();
    let_next_kernel_start();
    const int lane = threadIdx.x & 31;
    for (int64_t i = (int64_t)blockIdx.x * kUnpackThreads + threadIdx.x; i < n_top; i += (int64_t)gridDim.x * kUnpackThreads) top[i] = 0u;
    const int64_t row = (int64_t)blockIdx.x * (kUnpackThreads / 32) + (threadIdx.x >> 5);
    if (row >= T * q_heads) return;
    const int64_t t = row / q_heads;
    constexpr int kEach = D / 32;                                        // elements of a lane: 2, 4 or 8
    const __nv_bfloat16* src = q + t * ldq + (row - t * q_heads) * D + lane * kEach;
    uint32_t w[kEach / 2], m = 0u;
    if constexpr (kEach == 2) {
        w[0] = *reinterpret_cast<const uint32_t*>(src);
    } else if constexpr (kEach == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(src);
        w[0] = v.x; w[1] = v.y;
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(src);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
#pragma unroll
    for (int i = 0; i < kEach / 2; ++i) m = max(m, max(w[i] << 16 & 0x7fff0000u, w[i] & 0x7fff0000u));
    const int e = half_exponent(__reduce_max_sync(0xffffffffu, m));
    const float f = exp2i(-e);
#pragma unroll
    for (int i = 0; i < kEach / 2; ++i) {
        const __half2 h = __floats2half2_rn(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    uint32_t* dst = reinterpret_cast<uint32_t*>(to + row * D + lane * kEach);
    if constexpr (kEach == 2) *dst = w[0];
    else if constexpr (kEach == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    if (lane == 0) scale[row] = exp2i(e);
}

// The largest magnitudes that the groups of a sequence's keys and values can stand for, per head.  A CTA takes kTopTiles tiles, a thread 16 bytes of groups at a time.
constexpr int kTopTiles = 32;
template <int D>
__global__ void __launch_bounds__(kUnpackThreads) attn4_top_kernel(const Unpack P) {
    after_previous_kernel();
    let_next_kernel_start();
    const int b = blockIdx.y, h = blockIdx.x % P.kv_heads, tid = threadIdx.x;
    Seen s;
    if (!seen_keys(P, b, s)) return;
    const int64_t tile0 = s.first / kv4::kTileKeys + (int64_t)(blockIdx.x / P.kv_heads) * kTopTiles;
    constexpr int kPieces = D / 16;                                      // of 16 bytes, of a tile's keys' (or values') groups
    uint32_t most[2] = {0u, 0u};
    for (int i = tid; i < kTopTiles * kPieces * 2; i += kUnpackThreads) {
        const int value = i / (kTopTiles * kPieces), r = i % (kTopTiles * kPieces), piece = r % kPieces;
        const int64_t key = (tile0 + r / kPieces) * kv4::kTileKeys;
        if (key >= s.kv_len) continue;
        const int64_t pg = key / P.page_size;
        const int64_t page = pg < P.table_width ? P.table[(int64_t)b * P.table_stride + pg] : -1;
        if (page < 0 || page >= P.n_pages) continue;                     // reported by the unpacking
        const int slot = (int)(key - pg * P.page_size);
        const uint8_t* half = P.tiles + ((page * P.kv_heads + h) * (P.page_size / kv4::kTileKeys) + slot / kv4::kTileKeys) * kv4::tile_bytes(D) + (value ? kv4::half_bytes(D) : 0);
        const uint4 v = *reinterpret_cast<const uint4*>(half + kv4::groups_at(D) + piece * 16);
        const uint32_t g[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t at = key + (piece % 4) * 4 + e;                // the key that the group belongs to
            const float low = fabsf(low_of(g[e])), high = fabsf(fmaf(15.f, scale_of(g[e]), low_of(g[e])));
            const float top = fminf(fmaxf(low, high), 3.402823466e38f);
            if (at >= s.first && at < s.kv_len && scale_of(g[e]) == scale_of(g[e])) {        // not of a group that stands for NaN
                if (value) most[1] = max(most[1], __float_as_uint(top));
                else most[0] = max(most[0], __float_as_uint(top));
            }
        }
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const uint32_t m = __reduce_max_sync(0xffffffffu, most[v]);
        if ((tid & 31) == 0 && m) atomicMax(P.top + v * P.all * P.kv_heads + (P.first_seq + b) * P.kv_heads + h, m);
    }
}

// Keys and values to fp16.  A CTA takes 64 keys of a sequence and key head, a thread eight elements of a key at a time.  Bound: HBM, or the L2 that holds what it writes.
template <int D>
__global__ void __launch_bounds__(kUnpackThreads) attn4_unpack_kernel(const Unpack P) {
    after_previous_kernel();
    let_next_kernel_start();
    const int b = blockIdx.y, h = blockIdx.x % P.kv_heads, tid = threadIdx.x;
    Seen s;
    const bool any = seen_keys(P, b, s);
    const int64_t first_page = any ? s.first / kUnpackPage : 0;
    float f[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const int64_t at = v * P.all * P.kv_heads + (P.first_seq + b) * P.kv_heads + h;
        const int e = half_exponent(P.top[at]);
        f[v] = exp2i(-e);
        if (tid == 0 && blockIdx.x / P.kv_heads == 0) P.scale[at] = exp2i(e);
    }
    if (h == 0 && blockIdx.x / P.kv_heads == 0)
        for (int64_t i = tid; i < P.new_width; i += kUnpackThreads) {
            const int64_t at = i - first_page;
            P.new_table[b * P.new_width + i] = at >= 0 && at < P.new_pages ? (int)(b * P.new_pages + at) : -1;
        }
    if (!any) return;
    const int64_t key0 = first_page * kUnpackPage + (int64_t)(blockIdx.x / P.kv_heads) * kUnpackKeys;
    if (key0 >= s.kv_len || key0 + kUnpackKeys <= s.first) return;
    const int64_t at = key0 / kUnpackPage - first_page;
    if (at >= P.new_pages) return;                                      // more keys than the call was told of: the new table has no page for them either
    const int64_t row0 = ((b * (int64_t)P.new_pages + at) * P.kv_heads + h) * kUnpackPage + key0 % kUnpackPage;
    constexpr int kPieces = D / 8;                                      // of a key (and as many of its value)
    for (int i = tid; i < kUnpackKeys * kPieces * 2; i += kUnpackThreads) {
        const int value = i / (kUnpackKeys * kPieces), r = i % (kUnpackKeys * kPieces), j = r / kPieces, piece = r % kPieces;
        const int64_t key = key0 + j;
        if (key >= s.kv_len || key < s.first) continue;
        const int64_t pg = key / P.page_size;
        const int64_t page = pg < P.table_width ? P.table[(int64_t)b * P.table_stride + pg] : -1;
        if (page < 0 || page >= P.n_pages) { report(P.dev_status, MATQ_ERR_PAGE); continue; }
        const int slot = (int)(key - pg * P.page_size);
        const uint8_t* half = P.tiles + ((page * P.kv_heads + h) * (P.page_size / kv4::kTileKeys) + slot / kv4::kTileKeys) * kv4::tile_bytes(D) + (value ? kv4::half_bytes(D) : 0);
        const uint32_t codes = *reinterpret_cast<const uint32_t*>(half + (piece / 4) * 256 + (slot % 16) * 16 + (piece % 4) * 4);
        const uint32_t group = *reinterpret_cast<const uint32_t*>(half + kv4::groups_at(D) + (piece / 8) * 64 + (slot % 16) * 4);
        const float by = value ? f[1] : f[0], scale = scale_of(group), low = low_of(group);
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __half2 x = __floats2half2_rn(fmaf(scale, (float)((codes >> (8 * e)) & 15u), low) * by, fmaf(scale, (float)((codes >> (8 * e + 4)) & 15u), low) * by);
            w[e] = *reinterpret_cast<const uint32_t*>(&x);
        }
        *reinterpret_cast<uint4*>((value ? P.v : P.k) + (row0 + j) * D + piece * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

struct Plan4 {
    int rows;                    // of a CTA of the few-row kernel: 4, 8 or 16
    int64_t tiles_per_seq, splits, split_keys;
    bool few;                    // the few-row kernel is needed
    int64_t most_rows;           // of its sequences; those with more than above_rows are unpacked
    int64_t above_rows;
    // unpacked sequences; round = 0: there are none
    int64_t round, new_width, new_pages;
    size_t few_bytes, dense_bytes, table_bytes, query_bytes, scale_bytes, top_bytes, cache_bytes;
    size_t total() const { return few_bytes + dense_bytes + table_bytes + query_bytes + scale_bytes + top_bytes + 2 * cache_bytes; }
};

inline size_t padded(size_t n) { return (n + 255) / 256 * 256; }

inline Plan4 plan4(int64_t T, int batch, int q_heads, int kv_heads, int D, int64_t max_q, int64_t max_kv, int64_t window, int sms) {
    Plan4 p;
    const int group = q_heads / kv_heads;
    if (max_q > T) max_q = T;
    if (max_kv > kMost) max_kv = kMost;
    const bool mixed = max_q * group > kDirectRows;
    p.few = !mixed || batch > 1;
    p.most_rows = mixed ? kMixedRows : (1ll << 62);
    p.above_rows = batch > 1 ? kMixedRows : 0;
    const int64_t rows = mixed ? kMixedRows : max_q * group;
    p.rows = rows <= 4 ? 4 : D == 256 || rows <= 8 ? 8 : 16;
    p.tiles_per_seq = (rows + p.rows - 1) / p.rows;
    if (p.tiles_per_seq < 1) p.tiles_per_seq = 1;
    // Parts of the key range: the number whose rounds over the SMs cost least (ns; see plan_kind).
    const int warps = decode4_warps(D, p.rows), keys = 16 * warps;       // a step: a tile for each warp of a CTA
    int64_t range = max_kv;
    if (window > 0 && window < range && window + p.rows + 16 < range) range = window + p.rows + 16;
    range = (range + keys - 1) / keys + 1;
    const double ctas = (double)p.tiles_per_seq * batch * kv_heads, row_bytes = ctas * p.rows * D * 8;
    const double bytes = (double)warps * kv4::tile_bytes(D), mean = batch > 1 ? 0.9 : 1.0;
    double best = -1;
    int64_t splits = 1;
    for (int64_t n = 1; n <= kMaxSplits && n <= range && (n == 1 || (p.few && (double)n * T * q_heads * (D + 2) * 4 <= kPartBytes)); ++n) {
        const double slots = (double)sms * decode4_ctas(D, p.rows);
        const double busy = ctas * (n * mean > 1.0 ? n * mean : 1.0), at_work = busy < slots ? busy : slots;
        const double share = bytes * at_work / 6300.0, alone = (D == 256 ? 1100 : D == 128 ? 850 : 500) * (p.rows == 4 ? 1.0 : p.rows == 8 ? 1.2 : 1.45), step = share > alone ? share : alone;
        const double part = (double)((range + n - 1) / n) * step + (D == 256 ? 7000 : D == 128 ? 5000 : 4000);
        const double all = part * busy / slots * (n * mean > 1.0 ? 1.0 : mean);
        const double cost = (busy <= slots ? part : all + part / 2) + (n > 1 ? 3500 + row_bytes * n / 5000.0 : 0);
        if (best < 0 || cost < best) { best = cost; splits = n; }
        if (ctas * n >= 6 * slots) break;
    }
    const int64_t per = (range + splits - 1) / splits;
    p.splits = (range + per - 1) / per;
    p.split_keys = per * keys;
    p.few_bytes = p.splits > 1 ? padded((size_t)p.splits * T * q_heads * (D + 2) * sizeof(float)) : 0;
    p.round = 0;
    p.dense_bytes = p.table_bytes = p.query_bytes = p.scale_bytes = p.top_bytes = p.cache_bytes = 0;
    p.new_width = p.new_pages = 0;
    if (mixed) {
        p.new_width = (max_kv + kUnpackPage - 1) / kUnpackPage;
        if (p.new_width < 1) p.new_width = 1;
        p.new_pages = p.new_width;
        if (window > 0 && window < max_kv && (window + max_q) / kUnpackPage + 2 < p.new_pages) p.new_pages = (window + max_q) / kUnpackPage + 2;
        const int64_t per_seq = p.new_pages * kUnpackPage * kv_heads * D * 4;
        int64_t fit = kUnpackBytes / per_seq;
        const int64_t by_index = kMost / (p.new_pages * kUnpackPage * kv_heads);     // matq_attn_paged's limit on the rows of a cache
        if (fit > by_index) fit = by_index;
        p.round = fit < 1 ? 1 : fit < batch ? fit : batch;
        p.dense_bytes = padded(paged_workspace_bytes(T, (int)p.round, q_heads, kv_heads, D, max_q, max_kv, window, true));
        // the last round may have fewer sequences, which can be split into more parts
        if (batch % p.round != 0) {
            const size_t last = padded(paged_workspace_bytes(T, (int)(batch % p.round), q_heads, kv_heads, D, max_q, max_kv, window, true));
            if (last > p.dense_bytes) p.dense_bytes = last;
        }
        p.table_bytes = padded((size_t)p.round * p.new_width * sizeof(int32_t));
        p.query_bytes = padded((size_t)T * q_heads * D * 2);
        p.scale_bytes = padded((size_t)T * q_heads * sizeof(float));
        p.top_bytes = padded((size_t)4 * batch * kv_heads * sizeof(float));      // maxima and factors of keys and values
        p.cache_bytes = padded((size_t)p.round * p.new_pages * kUnpackPage * kv_heads * D * 2);
    }
    return p;
}

template <int D, int R>
int launch_decode4(const Params4& P, unsigned grid, cudaStream_t s) {
    using C = Dec4Cfg<D, R>;
    static std::atomic<unsigned long long> smem_ok{0};
    if (!opt_in_max_smem(attn4_decode_kernel<D, R>, smem_ok)) return MATQ_ERR_CUDA;
    if (launch_overlapped(attn4_decode_kernel<D, R>, dim3(grid), dim3(C::kThreads), C::kSmem, s, P) != cudaSuccess) {
        cudaGetLastError();
        return MATQ_ERR_CUDA;
    }
    return MATQ_OK;
}

template <int D>
int launch4(const Params4& P, int rows, unsigned grid, int64_t most_rows, cudaStream_t s) {
    int st;
    if (rows == 4) st = launch_decode4<D, 4>(P, grid, s);
    else if constexpr (D == 256) st = launch_decode4<D, 8>(P, grid, s);
    else st = rows == 8 ? launch_decode4<D, 8>(P, grid, s) : launch_decode4<D, 16>(P, grid, s);
    if (st == MATQ_OK && P.splits > 1) {
        Params J = {};
        J.out = P.out; J.cu_q = P.cu_q; J.ldo = P.ldo; J.T = P.T; J.batch = P.batch; J.q_heads = P.q_heads; J.group = P.group; J.splits = P.splits;
        J.part_o = P.part_o; J.part_ml = P.part_ml;
        J.filter = most_rows == kMixedRows; J.above_rows = kMixedRows; J.join_above = 0;
        st = launch_join<D>(J, s);
    }
    return st == MATQ_OK ? launch_status() : st;
}

template <int D>
int launch_queries(const void* q, int64_t ldq, int64_t T, int q_heads, __half* to, float* scale, uint32_t* top, int64_t n_top, cudaStream_t s) {
    const int64_t rows = T * q_heads, per = kUnpackThreads / 32;
    if (launch_overlapped(attn4_queries_kernel<D>, dim3((unsigned)((rows + per - 1) / per)), dim3(kUnpackThreads), 0, s, static_cast<const __nv_bfloat16*>(q), ldq, T, q_heads, to,
                          scale, top, n_top) != cudaSuccess) {
        cudaGetLastError();
        return MATQ_ERR_CUDA;
    }
    return launch_status();
}
template <int D>
int launch_unpack(const Unpack& U, int batch, cudaStream_t s) {
    const int64_t keys = (int64_t)U.new_pages * kUnpackPage, tops = keys / (kTopTiles * kv4::kTileKeys) + 1;
    if (launch_overlapped(attn4_top_kernel<D>, dim3((unsigned)(tops * U.kv_heads), (unsigned)batch), dim3(kUnpackThreads), 0, s, U) != cudaSuccess ||
        launch_overlapped(attn4_unpack_kernel<D>, dim3((unsigned)(keys / kUnpackKeys * U.kv_heads), (unsigned)batch), dim3(kUnpackThreads), 0, s, U) != cudaSuccess) {
        cudaGetLastError();
        return MATQ_ERR_CUDA;
    }
    return launch_status();
}

inline bool sizes_ok(int64_t T, int batch, int q_heads, int kv_heads, int D, int64_t max_q, int64_t max_kv, int64_t window) {
    return T > 0 && batch > 0 && q_heads > 0 && kv_heads > 0 && q_heads % kv_heads == 0 && q_heads / kv_heads <= 64 && (D == 64 || D == 128 || D == 256) && max_q >= 0 &&
           max_kv >= 0 && window >= 0 && T < (1ll << 31) && kv_heads <= (1 << 22);
}

}  // namespace attn
}  // namespace matq

extern "C" size_t matq_attn_paged4_workspace_bytes(int64_t T, int batch, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv, int64_t window) {
    using namespace matq::attn;
    if (!sizes_ok(T, batch, q_heads, kv_heads, head_dim, max_q, max_kv, window)) return 0;
    return plan4(T, batch, q_heads, kv_heads, head_dim, max_q, max_kv, window, matq::sm_count()).total();
}

extern "C" int matq_attn_paged4(const matq_paged_kv4* cache, int64_t T, const void* q, int q_heads, int64_t ldq, float scale, float softcap, int64_t window,
                                int64_t max_q, int64_t max_kv, void* out, int64_t ldo, void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    using namespace matq;
    using namespace matq::attn;
    if (!cache || T < 0 || q_heads < 1 || cache->batch < 0 || cache->n_pages < 0 || cache->kv_heads < 1 || cache->table_width < 0 ||
        (cache->batch > 1 && cache->table_stride < cache->table_width) || window < 0 || max_q < 0 || max_kv < 0 || !(softcap >= 0.f) || !(scale > 0.f))
        return MATQ_ERR_INVALID_ARG;
    const int D = cache->head_dim, ps = cache->page_size;
    if (D != 64 && D != 128 && D != 256) return MATQ_ERR_UNSUPPORTED;
    if (ps != 16 && ps != 32 && ps != 64 && ps != 128 && ps != 256) return MATQ_ERR_UNSUPPORTED;
    if (q_heads % cache->kv_heads != 0 || q_heads / cache->kv_heads > 64) return MATQ_ERR_UNSUPPORTED;
    const int64_t w = (int64_t)q_heads * D;
    if (ldq < w || ldq % 8 != 0 || ldo < w || ldo % 8 != 0 || T >= (1ll << 31) || cache->kv_heads > (1 << 22) || cache->n_pages > (1ll << 31) - 1) return MATQ_ERR_SHAPE;
    if (T == 0 || cache->batch == 0) return MATQ_OK;
    if (!q || !out || !cache->tiles || !cache->page_table || !cache->cu_q || !cache->kv_len || cache->n_pages == 0) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || !aligned16(cache->tiles) || !aligned16(workspace)) return MATQ_ERR_ALIGNMENT;
    const int group = q_heads / cache->kv_heads;
    const Plan4 p = plan4(T, cache->batch, q_heads, cache->kv_heads, D, max_q, max_kv, window, sm_count());
    const double ctas = (double)p.splits * cache->kv_heads * cache->batch * p.tiles_per_seq;
    const int64_t blocks = p.new_pages * (kUnpackPage / kUnpackKeys);
    if (ctas >= 2147483648.0 || (p.splits > 1 && T * q_heads >= (1ll << 31)) || (double)blocks * cache->kv_heads >= 2147483648.0 || p.round > 65535 || (p.round && T * q_heads >= (1ll << 31))) return MATQ_ERR_SHAPE;
    if (p.total() > workspace_bytes || (p.total() > 0 && !workspace)) return MATQ_ERR_WORKSPACE;
    const float cap = softcap < 0x1p100f ? softcap : 0.f;               // as in matq_attn_paged
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    unsigned char* at = static_cast<unsigned char*>(workspace);

    Params4 P;
    P.q = static_cast<const __nv_bfloat16*>(q); P.tiles = static_cast<const uint8_t*>(cache->tiles); P.out = static_cast<__nv_bfloat16*>(out);
    P.table = cache->page_table; P.cu_q = cache->cu_q; P.kv_len = cache->kv_len;
    P.ldq = ldq; P.ldo = ldo; P.table_stride = cache->table_stride; P.table_width = cache->table_width; P.n_pages = cache->n_pages; P.T = T;
    P.window = window; P.most_rows = p.most_rows;
    P.batch = cache->batch; P.q_heads = q_heads; P.kv_heads = cache->kv_heads; P.group = group;
    P.page_size = ps; P.page_shift = ps == 16 ? 4 : ps == 32 ? 5 : ps == 64 ? 6 : ps == 128 ? 7 : 8;
    P.tiles_per_seq = (int)p.tiles_per_seq; P.splits = (int)p.splits; P.split_keys = p.split_keys;
    P.scale = scale; P.softcap = cap;
    P.part_o = reinterpret_cast<float*>(at);
    P.part_ml = reinterpret_cast<float2*>(P.part_o + (size_t)p.splits * T * q_heads * D);
    P.dev_status = dev_status;
    const unsigned grid = (unsigned)ctas;
    int st = MATQ_OK;
    if (p.few)
        st = D == 64 ? launch4<64>(P, p.rows, grid, p.most_rows, s) : D == 128 ? launch4<128>(P, p.rows, grid, p.most_rows, s) : launch4<256>(P, p.rows, grid, p.most_rows, s);
    if (p.round == 0 || st != MATQ_OK) return st;

    void* dense = at + p.few_bytes;
    unsigned char* next = at + p.few_bytes + p.dense_bytes;
    const auto take = [&](size_t bytes) { unsigned char* here = next; next += bytes; return here; };
    Unpack U;
    U.tiles = P.tiles; U.table_stride = P.table_stride; U.table_width = P.table_width; U.n_pages = P.n_pages; U.window = window; U.above_rows = p.above_rows;
    U.kv_heads = P.kv_heads; U.group = group; U.page_size = ps; U.new_width = p.new_width; U.new_pages = (int)p.new_pages;
    U.new_table = reinterpret_cast<int32_t*>(take(p.table_bytes));
    __half* queries = reinterpret_cast<__half*>(take(p.query_bytes));
    float* q_scale = reinterpret_cast<float*>(take(p.scale_bytes));
    const int64_t heads = (int64_t)cache->batch * cache->kv_heads;
    U.top = reinterpret_cast<uint32_t*>(take(p.top_bytes));
    U.scale = reinterpret_cast<float*>(U.top) + 2 * heads;
    U.k = reinterpret_cast<__half*>(take(p.cache_bytes));
    U.v = reinterpret_cast<__half*>(take(p.cache_bytes));
    U.all = cache->batch;
    U.dev_status = dev_status;
    st = D == 64 ? launch_queries<64>(q, ldq, T, q_heads, queries, q_scale, U.top, 2 * heads, s) : D == 128 ? launch_queries<128>(q, ldq, T, q_heads, queries, q_scale, U.top, 2 * heads, s)
         : launch_queries<256>(q, ldq, T, q_heads, queries, q_scale, U.top, 2 * heads, s);
    for (int64_t b0 = 0; b0 < cache->batch && st == MATQ_OK; b0 += p.round) {
        const int n = (int)(cache->batch - b0 < p.round ? cache->batch - b0 : p.round);
        U.batch = n; U.first_seq = b0; U.table = P.table + b0 * P.table_stride; U.cu_q = P.cu_q + b0; U.kv_len = P.kv_len + b0;
        st = D == 64 ? launch_unpack<64>(U, n, s) : D == 128 ? launch_unpack<128>(U, n, s) : launch_unpack<256>(U, n, s);
        if (st != MATQ_OK) break;
        matq_paged_kv c;
        c.k = U.k; c.v = U.v; c.n_pages = (int64_t)n * p.new_pages; c.page_size = kUnpackPage; c.kv_heads = P.kv_heads; c.head_dim = D; c.batch = n;
        c.page_table = U.new_table; c.table_stride = c.table_width = p.new_width; c.cu_q = U.cu_q; c.kv_len = U.kv_len;
        const Half half = {q_scale, U.scale + b0 * cache->kv_heads, U.scale + heads + b0 * cache->kv_heads, p.above_rows};
        st = paged(&c, T, queries, q_heads, w, scale, softcap, window, max_q, max_kv, out, ldo, dense, p.dense_bytes, &half, dev_status, stream);
    }
    return st;
}
