// matq_attn_paged4: attention of new tokens over a paged cache in 4-bit groups (argument checks, choice of kernels and split).
//
// Few rows per sequence and key head (single tokens, drafts) go to attn4_decode_kernel, which reads the cache as it is.  Sequences with more rows (chunks) are bound
// by their products: their keys and values are unpacked once, into the workspace, and the 128-row kernels of matq_attn_paged take them from there.  That is one
// more pass over what a chunk sees (read 9/16 of a byte an element, written and read 2), where unpacking inside the product kernel would be repeated by every query
// tile and compete with the softmax for the SM's issue slots.  4096 tokens over 8192 keys, 32/8 heads of 128: 453 us, of which about 20 are the
// maxima, the unpacking and the queries; on a bf16 cache 416.
//
// Unpacked to bf16 a key would be rounded to 8 bits once more, and scores with it (with a few large channels outputs were off by 4.6e-3 of their norm, 2.7 times
// what rounding them alone is).  fp16 keeps 11 bits.  Its range is made to suffice by powers of two: a query row is scaled by its largest element, the keys and the
// values of a sequence and head by the largest that their groups can stand for; scores and outputs are scaled back in fp32.
#include <cuda_fp16.h>

#include "attn4_decode.cuh"

namespace matq {
namespace attn {

constexpr int64_t kMost = (1ll << 31) - 1;                              // lengths are 32-bit numbers
constexpr int kUnpackPage = 256, kUnpackThreads = 256, kUnpackKeys = 128;
// In a call that unpacks, sequences with no more rows than this are left to the few-row kernel.
constexpr int64_t kMixedRows = 16;
// Bytes of unpacked keys and values that a call's workspace holds at a time: sequences that do not fit together are served one round after another.
constexpr int64_t kUnpackBytes = 512ll << 20;
// Calls whose bounds let a single sequence take more than this read the cache as it is.
constexpr int64_t kUnpackMost = 16ll << 30;
// Most bytes of partial outputs: they are indexed by the call's tokens, of which few may be of sequences that are split.
constexpr double kPartBytes = 256.0 * (1 << 20);

constexpr int kHalfExp = 14;             // the largest magnitudes come to lie in [2^14, 2^15)

struct Unpack {
    const uint8_t* tiles;
    const int32_t *table, *cu_q, *kv_len;
    int64_t table_stride, table_width, n_pages, window, above_rows;
    int batch, kv_heads, group, page_size, page_shift;
    int64_t new_width;           // entries of a row of the new table
    int new_pages;               // pages of kUnpackPage keys per sequence
    int32_t* new_table;
    __half *k, *v;               // [batch * new_pages][kv_heads][kUnpackPage][D]
    uint32_t* top;               // [2][batch][kv_heads][tops]: largest magnitudes of keys and of values, as the bits of floats
    int64_t tops;
    float* scale;                // [2][batch][kv_heads]: what to multiply with afterwards
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
__device__ __forceinline__ int64_t heads_of(const Unpack& P) { return (int64_t)P.batch * P.kv_heads; }
// The tile that holds a key, or null where its page is out of range.
__device__ __forceinline__ const uint8_t* tile_of(const Unpack& P, int b, int h, int64_t key, int D) {
    const int64_t pg = key >> P.page_shift;
    const int64_t page = pg < P.table_width ? P.table[(int64_t)b * P.table_stride + pg] : -1;
    if (page < 0 || page >= P.n_pages) return nullptr;
    return P.tiles + ((page * P.kv_heads + h) * (P.page_size >> 4) + ((key & (P.page_size - 1)) >> 4)) * kv4::tile_bytes(D);
}
__device__ __forceinline__ int half_exponent(uint32_t top) { return max((int)(top >> 23) - 127 - kHalfExp, -126); }        // what was taken off: 2^-126 .. 2^114

// Before the unpacking: the largest magnitudes that the groups of a sequence's keys and values can stand for, per head; a CTA takes kTopTiles tiles and leaves their
// maximum for the unpacking to join.
constexpr int kTopTiles = 32, kQueryPieces = 4;
template <int D>
__global__ void __launch_bounds__(kUnpackThreads) attn4_top_kernel(const Unpack P) {
    after_previous_kernel();
    let_next_kernel_start();
    const int tid = threadIdx.x;
    const unsigned rest = blockIdx.x, bh = rest / (unsigned)P.tops;
    const int b = (int)(bh / (unsigned)P.kv_heads), h = (int)(bh % (unsigned)P.kv_heads), chunk = (int)(rest % (unsigned)P.tops);
    __shared__ uint32_t s_most[2];
    if (tid < 2) s_most[tid] = 0u;
    __syncthreads();
    Seen s;
    if (seen_keys(P, b, s)) {
        const int64_t tile0 = s.first / kv4::kTileKeys + (int64_t)chunk * kTopTiles;
        constexpr int kPieces = D / 16;                                  // of 16 bytes, of a tile's keys' (or values') groups
        uint32_t most[2] = {0u, 0u};
        for (int i = tid; i < kTopTiles * kPieces * 2; i += kUnpackThreads) {
            const int value = i / (kTopTiles * kPieces), r = i % (kTopTiles * kPieces), piece = r % kPieces;
            const int64_t key = (tile0 + r / kPieces) * kv4::kTileKeys;
            const uint8_t* tile = key < s.kv_len ? tile_of(P, b, h, key, D) : nullptr;       // a page out of range is reported by the unpacking
            if (!tile) continue;
            const uint4 v = *reinterpret_cast<const uint4*>(tile + (value ? kv4::half_bytes(D) : 0) + kv4::groups_at(D) + piece * 16);
            const uint32_t g[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t at = key + (piece % 4) * 4 + e;            // the key that the group belongs to
                const float low = fabsf(low_of(g[e])), high = fabsf(fmaf(15.f, scale_of(g[e]), low_of(g[e])));
                const float top = fminf(fmaxf(low, high), 3.402823466e38f);
                if (at >= s.first && at < s.kv_len && scale_of(g[e]) == scale_of(g[e]))      // not of a group that stands for NaN
                    most[value] = max(most[value], __float_as_uint(top));
            }
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const uint32_t m = __reduce_max_sync(0xffffffffu, most[v]);
            if ((tid & 31) == 0 && m) atomicMax(&s_most[v], m);
        }
    }
    __syncthreads();
    if (tid < 2) P.top[((int64_t)tid * heads_of(P) + bh) * P.tops + chunk] = s_most[tid];
}

// Keys and values to fp16: a warp per tile of 16 keys, a lane 32 elements of a key at a time (its codes and those of its neighbours are 512 bytes side by side).
// Queries to fp16, by the CTAs behind those: they are waited for no longer than keys and values are.
// Bound: HBM, or the L2 that holds what it writes.
struct Queries {
    const __nv_bfloat16* q;
    int64_t ldq, T;
    int q_heads;
    int64_t first_cta;
    __half* to;
    float* scale;
};
template <int D>
__global__ void __launch_bounds__(kUnpackThreads) attn4_unpack_kernel(const Unpack P, const Queries Q) {
    constexpr int kTiles = kUnpackThreads / 32, kCtaKeys = kTiles * kv4::kTileKeys;
    static_assert(kCtaKeys == kUnpackKeys, "a warp per tile");
    __shared__ float s_by[2];
    after_previous_kernel();
    let_next_kernel_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (blockIdx.x >= Q.first_cta) {
        // a lane takes eight elements; the D / 8 lanes of a row share its largest
        constexpr int kLanes = D / 8;
        uint4 v[kQueryPieces];
        const int64_t first = ((blockIdx.x - Q.first_cta) * kQueryPieces * kUnpackThreads + tid) / kLanes, rows = Q.T * Q.q_heads;
        const int at = tid % kLanes * 8;
#pragma unroll
        for (int i = 0; i < kQueryPieces; ++i) {
            const int64_t row = first + i * (kUnpackThreads / kLanes), t = rows <= 0x7fffffff ? (int64_t)((uint32_t)row / (uint32_t)Q.q_heads) : row / Q.q_heads;
            v[i] = row < rows ? *reinterpret_cast<const uint4*>(Q.q + t * Q.ldq + (row - t * Q.q_heads) * D + at) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < kQueryPieces; ++i) {
            const int64_t row = first + i * (kUnpackThreads / kLanes);
            uint32_t top = top_of_piece(v[i]);
#pragma unroll
            for (int w = 1; w < kLanes; w <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, w));
            const int e = half_exponent(top);
            const float f = exp2i(-e);
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            uint32_t o[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const __half2 h = __floats2half2_rn(__uint_as_float(w[x] << 16) * f, __uint_as_float(w[x] & 0xffff0000u) * f);
                o[x] = *reinterpret_cast<const uint32_t*>(&h);
            }
            if (row < rows) {
                *reinterpret_cast<uint4*>(Q.to + row * D + at) = make_uint4(o[0], o[1], o[2], o[3]);
                if (at == 0) Q.scale[row] = exp2i(e);
            }
        }
        return;
    }
    const unsigned per_batch = (unsigned)(P.new_pages * (kUnpackPage / kUnpackKeys)) * (unsigned)P.kv_heads, in_batch = blockIdx.x % per_batch;
    const int b = (int)(blockIdx.x / per_batch), h = (int)(in_batch % (unsigned)P.kv_heads);
    const int64_t chunk = in_batch / (unsigned)P.kv_heads;
    if (warp < 2) {                                                      // the factors of keys and of values
        uint32_t top = 0u;
        const uint32_t* from = P.top + ((int64_t)warp * heads_of(P) + (int64_t)b * P.kv_heads + h) * P.tops;
        for (int64_t i = lane; i < P.tops; i += 32) top = max(top, from[i]);
        const int e = half_exponent(__reduce_max_sync(0xffffffffu, top));
        if (lane == 0) {
            s_by[warp] = exp2i(-e);
            if (chunk == 0) P.scale[(int64_t)warp * heads_of(P) + (int64_t)b * P.kv_heads + h] = exp2i(e);
        }
    }
    __syncthreads();
    Seen s;
    const bool any = seen_keys(P, b, s);
    const int64_t first_page = any ? s.first / kUnpackPage : 0;
    if (h == 0 && chunk == 0)
        for (int64_t i = tid; i < P.new_width; i += kUnpackThreads) {
            const int64_t at = i - first_page;
            P.new_table[b * P.new_width + i] = at >= 0 && at < P.new_pages ? (int)(b * P.new_pages + at) : -1;
        }
    if (!any) return;
    const int64_t key0 = first_page * kUnpackPage + chunk * kCtaKeys + warp * kv4::kTileKeys;
    if (key0 >= s.kv_len || key0 + kv4::kTileKeys <= s.first) return;
    const int64_t at = key0 / kUnpackPage - first_page;
    if (at >= P.new_pages) return;                                      // more keys than the call was told of: the new table has no page for them either
    const uint8_t* tile = tile_of(P, b, h, key0, D);
    if (!tile) {
        if (lane == 0) report(P.dev_status, MATQ_ERR_PAGE);
        return;
    }
    const int64_t row0 = ((b * (int64_t)P.new_pages + at) * P.kv_heads + h) * kUnpackPage + key0 % kUnpackPage;
    constexpr int kEach = D / 32, kHalf = D / 2;                        // pieces of a lane, and of a tile's keys
    uint4 codes[kEach];
    uint32_t group[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int p = lane + 32 * i, value = p / kHalf, r = p % kHalf;
        const uint8_t* half = tile + value * kv4::half_bytes(D);
        codes[i] = ld_stream_u4(half + r * 16);
        group[i] = *reinterpret_cast<const uint32_t*>(half + kv4::groups_at(D) + (r / 32) * 64 + (r % 16) * 4);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int p = lane + 32 * i, value = p / kHalf, r = p % kHalf;
        const float by = s_by[value], scale = scale_of(group[i]) * by, mid = fmaf(8.f, scale_of(group[i]), low_of(group[i])) * by;
        const uint32_t c[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
        uint4* dst = reinterpret_cast<uint4*>((value ? P.v : P.k) + (row0 + r % 16) * D + (r / 16) * 32);
        const bool wide = (reinterpret_cast<uintptr_t>(P.k) & 31u) == 0 && (reinterpret_cast<uintptr_t>(P.v) & 31u) == 0;       // the workspace is aligned to 16 bytes, or better
        uint32_t o[2][4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            // (code - 8) / 64 of codes 0 and 4, 1 and 5, 2 and 6, 3 and 7
            const uint32_t x[4] = {centred_low(c[w]), centred_high(c[w]), centred_low(c[w] >> 8), centred_high(c[w] >> 8)};
            const auto of = [&](int e) {
                const float centred = __uint_as_float(e < 4 ? x[e] << 16 : x[e - 4] & 0xffff0000u);
                return fmaf(scale, centred * 64.f, mid);
            };
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __half2 y = __floats2half2_rn(of(2 * e), of(2 * e + 1));
                o[w & 1][e] = *reinterpret_cast<const uint32_t*>(&y);
            }
            if (w & 1) {                                                // 32 bytes, a whole sector, in one store where the address allows it
                if (wide) {
                    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst + w - 1), "r"(o[0][0]), "r"(o[0][1]), "r"(o[0][2]), "r"(o[0][3]),
                                 "r"(o[1][0]), "r"(o[1][1]), "r"(o[1][2]), "r"(o[1][3]) : "memory");
                } else {
                    dst[w - 1] = make_uint4(o[0][0], o[0][1], o[0][2], o[0][3]);
                    dst[w] = make_uint4(o[1][0], o[1][1], o[1][2], o[1][3]);
                }
            }
        }
    }
}

struct Plan4 {
    int rows;                    // of a CTA of the few-row kernel: 4, 8 or 16
    int64_t tiles_per_seq, splits, split_keys;
    bool few;                    // the few-row kernel is needed
    int64_t most_rows;           // of its sequences; those with more than above_rows are unpacked
    int64_t above_rows;
    // unpacked sequences; round = 0: there are none
    int64_t round, new_width, new_pages, tops;
    size_t few_bytes, dense_bytes, table_bytes, query_bytes, scale_bytes, top_bytes, cache_bytes;
    size_t total() const { return few_bytes + dense_bytes + table_bytes + query_bytes + scale_bytes + top_bytes + 2 * cache_bytes; }
};

inline size_t padded(size_t n) { return (n + 255) / 256 * 256; }

// Tiles of `rows` rows and the split of the few-row kernel for sequences of at most most_rows rows, and what they cost (ns): the number of parts of the key range
// whose rounds over the SMs cost least.  Measured: a step, a tile of 16 keys for each warp of a CTA, alone on an SM, beside another CTA, or at the share of HBM that
// the CTAs at work leave each other; a CTA's start and end; the join.
inline double plan_rows(Plan4& p, int rows, int64_t most_rows, int64_t T, int batch, int q_heads, int kv_heads, int D, int64_t max_kv, int64_t window, int sms) {
    p.rows = rows;
    p.tiles_per_seq = (most_rows + rows - 1) / rows;
    if (p.tiles_per_seq < 1) p.tiles_per_seq = 1;
    const int warps = decode4_warps(D, rows), keys = 16 * warps;
    int64_t range = max_kv;
    if (window > 0 && window < range && window + rows + 16 < range) range = window + rows + 16;
    range = (range + keys - 1) / keys + 1;
    // Tiles of the batch; fewer where its tokens do not go round.  The last of a sequence is half full, in steps of the heads that share a key head.
    const int group = q_heads / kv_heads;
    int common = rows;
    while (group % common != 0) common /= 2;
    const double all_tiles = (double)p.tiles_per_seq * batch, some = (double)T * group / rows + 0.5 * (1.0 - (double)common / rows) * batch;
    const double ctas = (T * group < most_rows * batch && some < all_tiles ? some : all_tiles) * kv_heads, row_bytes = all_tiles * kv_heads * rows * D * 8, slots = (double)sms * decode4_ctas(D, rows);
    const double bytes = (double)warps * kv4::tile_bytes(D);
    const int kind = rows == 4 ? 0 : rows == 8 ? 1 : 2;
    constexpr double kAlone[3][3] = {{500, 520, 830}, {850, 850, 1050}, {1100, 1320, 0}}, kBeside[3][3] = {{720, 740, 1040}, {1230, 1170, 1280}, {1600, 1850, 0}};
    const int width = D == 64 ? 0 : D == 128 ? 1 : 2;
    const double ends = D == 256 ? 7000 : D == 128 ? 5000 : 4000;
    double best = -1;
    int64_t splits = 1;
    for (int64_t n = 1; n <= kMaxSplits && n <= range && (n == 1 || (double)n * T * q_heads * (D + 2) * 4 <= kPartBytes); ++n) {
        const double busy = ctas * n, at_work = busy < slots ? busy : slots;
        const double share = bytes * at_work / 6300.0, own = (busy <= sms ? kAlone : kBeside)[width][kind], step = share > own ? share : own;
        const double part = (double)((range + n - 1) / n) * step + ends;
        const double rounds = busy / slots, late = rounds < 1.25 ? 4 * (rounds - 1) : 1.0;       // the last round's end: half a part, if it is not all but empty
        const double cost = (rounds <= 1 ? part : part * (rounds + late / 2)) + (n > 1 ? 4500 + row_bytes * n / 5000.0 : 0);
        if (best < 0 || cost < best) { best = cost; splits = n; }
        if (ctas * n >= 6 * slots) break;
    }
    const int64_t per = (range + splits - 1) / splits;
    p.splits = (range + per - 1) / per;
    p.split_keys = per * keys;
    return best;
}

// Rows of a tile: 4 or 8 where they hold a sequence's, else 8 or 16, whichever costs less.  Tiles of 8 unpack the cache twice as often, but 16 warps of theirs share an
// SM, not 12, and more CTAs fill rounds better: 16 ragged sequences of 8 to 24 rows over 4096 keys, heads of 128, 46 us, in tiles of 16 rows 58; 24 rows of 4 sequences
// over 4000 keys 23.5 and 26.8.  But 16 rows over 32000 keys 27.2 and 24.0; 24 rows of 16 sequences over 4000 keys 66 and 58.
inline double plan_few(Plan4& p, int64_t rows, int64_t T, int batch, int q_heads, int kv_heads, int D, int64_t max_kv, int64_t window, int sms) {
    const double cost = plan_rows(p, rows <= 4 ? 4 : 8, rows, T, batch, q_heads, kv_heads, D, max_kv, window, sms);
    if (rows <= 8 || D == 256) return cost;
    Plan4 wide = p;
    const double of_wide = plan_rows(wide, 16, rows, T, batch, q_heads, kv_heads, D, max_kv, window, sms);
    if (of_wide >= cost) return cost;
    p = wide;
    return of_wide;
}

inline Plan4 plan4(int64_t T, int batch, int q_heads, int kv_heads, int D, int64_t max_q, int64_t max_kv, int64_t window, int sms) {
    Plan4 p;
    const int group = q_heads / kv_heads;
    if (max_q > T) max_q = T;
    if (max_kv > kMost) max_kv = kMost;
    window = window_of(window);
    // Rows of the longest sequence: all of them for the few-row kernel, or unpacking for sequences with more than kMixedRows (a batch of one whatever it has),
    // whichever costs less.
    const int64_t rows = max_q * group;
    const double direct = plan_few(p, rows, T, batch, q_heads, kv_heads, D, max_kv, window, sms);
    bool mixed = false;
    const int64_t width = max_kv > kUnpackPage ? (max_kv + kUnpackPage - 1) / kUnpackPage : 1;
    int64_t pages = width;                                              // of kUnpackPage keys, that a sequence is unpacked to
    if (window > 0 && window < max_kv && (window + max_q) / kUnpackPage + 2 < pages) pages = (window + max_q) / kUnpackPage + 2;
    const double per_seq = (double)(pages * kUnpackPage) * kv_heads * D * 4;        // bytes; the rows of a cache that the 128-row kernels index are far fewer than 2^31 then
    if (rows > kMixedRows && per_seq <= (double)kUnpackMost) {
        const int64_t range = window > 0 && window + max_q < max_kv ? window + max_q : max_kv;
        const double dense = 9000 + 4.0 * T * q_heads * D / 6000 + 8.0 * batch * range * kv_heads * D / 5000 + paged_cost(T, batch, q_heads, kv_heads, D, max_q, max_kv, window);
        mixed = dense < direct;
    }
    p.few = !mixed || batch > 1;
    p.most_rows = mixed ? kMixedRows : (1ll << 62);
    p.above_rows = batch > 1 ? kMixedRows : 0;
    if (mixed) plan_few(p, kMixedRows, T, batch, q_heads, kv_heads, D, max_kv, window, sms);
    if (!p.few) p.splits = 1;
    p.few_bytes = p.splits > 1 ? padded((size_t)p.splits * T * q_heads * (D + 2) * sizeof(float)) : 0;
    p.round = 0;
    p.dense_bytes = p.table_bytes = p.query_bytes = p.scale_bytes = p.top_bytes = p.cache_bytes = 0;
    p.new_width = p.new_pages = p.tops = 0;
    if (mixed) {
        p.new_width = width;
        p.new_pages = pages;
        const int64_t fit = (int64_t)((double)kUnpackBytes / per_seq);
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
        p.tops = p.new_pages * kUnpackPage / (kTopTiles * kv4::kTileKeys) + 1;
        p.top_bytes = padded((size_t)2 * p.round * kv_heads * (p.tops + 1) * sizeof(float));
        p.cache_bytes = padded((size_t)p.round * p.new_pages * kUnpackPage * kv_heads * D * 2);
    }
    return p;
}

inline Plan4 recent_plan4(int64_t T, int batch, int q_heads, int kv_heads, int D, int64_t max_q, int64_t max_kv, int64_t window) {
    static thread_local Recent<Plan4, 9> recent;
    const int sms = sm_count();
    return recent.of({T, batch, q_heads, kv_heads, D, max_q, max_kv, window, sms}, [&] { return plan4(T, batch, q_heads, kv_heads, D, max_q, max_kv, window, sms); });
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
        J.filter = most_rows == kMixedRows; J.above_rows = kMixedRows; J.join_above = 0;         // the other sequences are joined by their own
        st = launch_join<D>(J, s);
    }
    return st == MATQ_OK ? launch_status() : st;
}

template <int D>
int launch_unpack(const Unpack& U, Queries Q, cudaStream_t s) {
    const int64_t rows_of_cta = (int64_t)kQueryPieces * kUnpackThreads / (D / 8), query_ctas = (Q.T * Q.q_heads + rows_of_cta - 1) / rows_of_cta;
    Q.first_cta = (int64_t)U.new_pages * (kUnpackPage / kUnpackKeys) * U.kv_heads * U.batch;
    if (launch_overlapped(attn4_top_kernel<D>, dim3((unsigned)(U.tops * U.kv_heads * U.batch)), dim3(kUnpackThreads), 0, s, U) != cudaSuccess ||
        launch_overlapped(attn4_unpack_kernel<D>, dim3((unsigned)(Q.first_cta + query_ctas)), dim3(kUnpackThreads), 0, s, U, Q) != cudaSuccess) {
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
    return recent_plan4(T, batch, q_heads, kv_heads, head_dim, max_q, max_kv, window).total();
}

extern "C" int matq_attn_paged4_plan(int64_t T, int batch, int q_heads, int kv_heads, int head_dim, int64_t max_q, int64_t max_kv, int64_t window, int* rows, int* row_parts,
                                     int* unpacked, int* tiles, int* parts) {
    using namespace matq::attn;
    if (!sizes_ok(T, batch, q_heads, kv_heads, head_dim, max_q, max_kv, window)) return MATQ_ERR_INVALID_ARG;
    const Plan4 p = recent_plan4(T, batch, q_heads, kv_heads, head_dim, max_q, max_kv, window);
    int t = 0, n = 0;
    if (p.round) paged_cost(T, (int)p.round, q_heads, kv_heads, head_dim, max_q, max_kv, window, &t, &n);
    if (rows) *rows = p.few ? p.rows : 0;
    if (row_parts) *row_parts = p.few ? (int)p.splits : 0;
    if (unpacked) *unpacked = (int)p.round;
    if (tiles) *tiles = t;
    if (parts) *parts = n;
    return MATQ_OK;
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
    window = window_of(window);
    const Plan4 p = recent_plan4(T, cache->batch, q_heads, cache->kv_heads, D, max_q, max_kv, window);
    const double ctas = (double)p.splits * cache->kv_heads * cache->batch * p.tiles_per_seq;
    const int64_t blocks = p.new_pages * (kUnpackPage / kUnpackKeys);
    const double rows = (double)T * q_heads;
    if (ctas >= 2147483648.0 || (p.splits > 1 && rows >= 2147483648.0) ||
        (p.round && ((double)blocks * cache->kv_heads * p.round + rows >= 2147483648.0 || (double)p.tops * cache->kv_heads * p.round >= 2147483648.0)))
        return MATQ_ERR_SHAPE;
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
    Queries Q;
    U.tiles = P.tiles; U.table_stride = P.table_stride; U.table_width = P.table_width; U.n_pages = P.n_pages; U.window = window; U.above_rows = p.above_rows;
    U.kv_heads = P.kv_heads; U.group = group; U.page_size = ps; U.page_shift = P.page_shift; U.new_width = p.new_width; U.new_pages = (int)p.new_pages; U.tops = p.tops;
    U.new_table = reinterpret_cast<int32_t*>(take(p.table_bytes));
    Q.to = reinterpret_cast<__half*>(take(p.query_bytes));
    Q.scale = reinterpret_cast<float*>(take(p.scale_bytes));
    U.top = reinterpret_cast<uint32_t*>(take(p.top_bytes));
    U.k = reinterpret_cast<__half*>(take(p.cache_bytes));
    U.v = reinterpret_cast<__half*>(take(p.cache_bytes));
    U.dev_status = dev_status;
    Q.q = P.q; Q.ldq = ldq; Q.T = T; Q.q_heads = q_heads;
    for (int64_t b0 = 0; b0 < cache->batch && st == MATQ_OK; b0 += p.round) {
        const int n = (int)(cache->batch - b0 < p.round ? cache->batch - b0 : p.round);
        const int64_t heads = (int64_t)n * cache->kv_heads;
        U.batch = n; U.table = P.table + b0 * P.table_stride; U.cu_q = P.cu_q + b0; U.kv_len = P.kv_len + b0;
        U.scale = reinterpret_cast<float*>(U.top) + 2 * heads * p.tops;
        st = D == 64 ? launch_unpack<64>(U, Q, s) : D == 128 ? launch_unpack<128>(U, Q, s) : launch_unpack<256>(U, Q, s);
        if (st != MATQ_OK) break;
        Q.T = 0;                                                        // once for all rounds
        matq_paged_kv c;
        c.k = U.k; c.v = U.v; c.n_pages = (int64_t)n * p.new_pages; c.page_size = kUnpackPage; c.kv_heads = P.kv_heads; c.head_dim = D; c.batch = n;
        c.page_table = U.new_table; c.table_stride = c.table_width = p.new_width; c.cu_q = U.cu_q; c.kv_len = U.kv_len;
        const Half half = {Q.scale, U.scale, U.scale + heads, p.above_rows};
        st = paged(&c, T, Q.to, q_heads, w, scale, softcap, window, max_q, max_kv, out, ldo, dense, p.dense_bytes, &half, dev_status, stream);
    }
    return st;
}
