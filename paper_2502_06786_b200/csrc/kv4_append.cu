// matq_kv4_append: new keys and values into a paged cache held in 4-bit groups, keys and queries rotated by their positions on the way.
//
// As matq_kv_append (a CTA per token, a thread keeps its place within the heads, angles in registers, the first heads requested before the position is known),
// but a thread's place is eight neighbouring elements, which is what it quantises: with halves as pairs it reads its eight partners beside them (from L1, where
// the thread that owns them has brought them), and the eight lanes of a group exchange its ends.
//
// Bound: few tokens, a launch and two dependent look-ups; prompts, each token's chain of look-ups (sequence, length, page, angles), which 40 % of an SM's warps hide in part
// (64 registers a thread; 57 % of the issue slots used; 4.0 TB/s with 64 threads a token).
#include "kv4_cache.cuh"

namespace matq {
namespace kva4 {

// Threads of a token: 256 in a decode step, where a call is a chain of trips to memory; for many tokens 64, which share what is looked up among fewer warps (three
// prompts of 1500 to 4000 tokens, 16/8 heads of 256: 60 us, with 256 threads 75; 64 single tokens, 32/8 heads of 128: 3.6 us with 256).
constexpr int kThreadsFew = 256, kThreadsMany = 64;
constexpr int64_t kMany = 2048;

struct Params {
    uint8_t* cache;
    const int32_t *table, *cu_q, *kv_len;
    int64_t n_pages, table_stride, table_width;
    int page_size, kv_heads, q_heads, batch;
    const __nv_bfloat16 *q, *k, *v;
    int64_t ldq, ldk, ldv, ldqo;
    const float* cos_sin;
    int64_t max_pos;
    int rot, interleaved;
    __nv_bfloat16* q_out;
    int32_t* dev_status;
};

constexpr int kAhead = 2;        // heads per thread whose data are requested before the position is known

template <int D, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) kv4_append_kernel(const Params P) {
    constexpr int kPlaces = D / 8, kStep = kThreads / kPlaces;          // 8, 16 or 32 threads along a head; heads side by side
    after_previous_kernel();
    let_next_kernel_start();
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31;
    const int keys_from = P.q_heads, values_from = P.q_heads + P.kv_heads, heads = values_from + P.kv_heads, half = P.rot / 2;
    const int first = tid / kPlaces, e0 = tid % kPlaces * 8;
    const bool turns = e0 < P.rot, paired = turns && !P.interleaved, upper = paired && e0 >= half;
    const int partner = (paired ? upper ? e0 - half : e0 + half : e0) - e0;
    // this thread's place in a head of each kind, as if the heads of all kinds stood one behind another
    const __nv_bfloat16 *q_at = P.q + t * P.ldq + e0, *k_at = P.k + t * P.ldk + e0 - (int64_t)keys_from * D, *v_at = P.v + t * P.ldv + e0 - (int64_t)values_from * D;
    uint4 data[kAhead][2];
    const auto load = [&](int hd, uint4 (&d)[2]) {
        d[0] = d[1] = make_uint4(0u, 0u, 0u, 0u);
        if (hd >= heads) return;
        const __nv_bfloat16* at = (hd < keys_from ? q_at : hd < values_from ? k_at : v_at) + (int64_t)hd * D;
        d[0] = *reinterpret_cast<const uint4*>(at);
        if (paired && hd < values_from) d[1] = *reinterpret_cast<const uint4*>(at + partner);
    };

    // the token's sequence: the number of sequences that end at or before it (32 bounds per step, every warp for itself)
    int b = 0;
    for (int at = 0; at < P.batch; at += 32) {
        const int i = at + lane;
        const int end = i < P.batch ? P.cu_q[i + 1] : 0x7fffffff;
        b += __popc(__ballot_sync(0xffffffffu, (int64_t)end <= t));
    }
    if (b >= P.batch) return;                                          // a row that belongs to no sequence (and is not read)
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(first + i * kStep, data[i]);
    const int64_t q0 = P.cu_q[b], q1 = P.cu_q[b + 1];
    const int64_t pos = (int64_t)P.kv_len[b] - (q1 - q0) + (t - q0);
    const unsigned pg = pos >= 0 && pos <= 0x7fffffff ? (unsigned)pos / (unsigned)P.page_size : 0xffffffffu;
    bool ok = pg != 0xffffffffu && t >= q0 && pg < P.table_width && (P.rot == 0 || pos < P.max_pos);
    int64_t page = 0;
    if (ok) {
        page = P.table[(int64_t)b * P.table_stride + pg];
        ok = page >= 0 && page < P.n_pages;
    }
    if (!ok) {
        if (tid == 0) report(P.dev_status, MATQ_ERR_PAGE);
        return;
    }
    const unsigned slot = (unsigned)pos - pg * (unsigned)P.page_size, key = slot % kv4::kTileKeys;
    // angles: of eight pairs when pairs are halves apart, of four when they are neighbours.  a c - b s is a c + b (-s): the sign goes with the angle.
    float c[8], s[8];
    if (turns) {
        const float* cs = P.cos_sin + pos * P.rot + (paired ? upper ? e0 - half : e0 : e0 / 2);
        const float sign = upper || !paired ? 1.f : -1.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i == 1 && !paired) break;
            const float4 cv = *reinterpret_cast<const float4*>(cs + 4 * i), sv = *reinterpret_cast<const float4*>(cs + half + 4 * i);
            c[4 * i] = cv.x; c[4 * i + 1] = cv.y; c[4 * i + 2] = cv.z; c[4 * i + 3] = cv.w;
            s[4 * i] = sv.x * sign; s[4 * i + 1] = sv.y * sign; s[4 * i + 2] = sv.z * sign; s[4 * i + 3] = sv.w * sign;
        }
    }
    // Every product and sum is rounded by itself: the values that are quantised are defined bit for bit.
    const auto turned = [&](const uint4 (&d)[2]) {
        const uint32_t o[4] = {d[0].x, d[0].y, d[0].z, d[0].w}, p[4] = {d[1].x, d[1].y, d[1].z, d[1].w};
        const auto both = [](uint32_t w) { return two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); };
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint64_t u, w;
            if (paired) {
                u = two_products(both(o[i]), two(c[2 * i], c[2 * i + 1]));
                w = two_products(both(p[i]), two(s[2 * i], s[2 * i + 1]));
            } else {
                u = two_products(both(o[i]), two(c[i], c[i]));
                w = two_products(both(__byte_perm(o[i], 0u, 0x1032)), two(-s[i], s[i]));
            }
            const __nv_bfloat162 h = __floats2bfloat162_rn(__fadd_rn(__uint_as_float((uint32_t)u), __uint_as_float((uint32_t)w)),
                                                           __fadd_rn(__uint_as_float((uint32_t)(u >> 32)), __uint_as_float((uint32_t)(w >> 32))));
            r[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(r[0], r[1], r[2], r[3]);
    };
    __nv_bfloat16* q_to = P.q_out + t * P.ldqo + e0;
    const int64_t head_bytes = (int64_t)(P.page_size / kv4::kTileKeys) * kv4::tile_bytes(D);
    uint8_t* tile = P.cache + page * P.kv_heads * head_bytes + (int64_t)(slot / kv4::kTileKeys) * kv4::tile_bytes(D);
    const int codes_at = e0 / 32 * 256 + (int)key * 16 + e0 % 32 / 2, group_at = kv4::groups_at(D) + e0 / 64 * 64 + (int)key * 4;
    bool bad = false;
    const auto finish = [&](int hd, const uint4 (&d)[2]) {
        if (hd >= heads) return;                                        // the lanes of a group share their head
        const bool value = hd >= values_from;
        const uint4 x = turns && !value ? turned(d) : d[0];
        if (hd < keys_from) {
            *reinterpret_cast<uint4*>(q_to + (int64_t)hd * D) = x;
            return;
        }
        uint32_t codes;
        const uint32_t group = quantise_piece<8>(x, codes, 0xffu << (lane & 24));
        uint8_t* to = tile + (hd - (value ? values_from : keys_from)) * head_bytes + (value ? kv4::half_bytes(D) : 0);
        *reinterpret_cast<uint32_t*>(to + codes_at) = codes;
        if ((lane & 7) == 0) {
            *reinterpret_cast<uint32_t*>(to + group_at) = group;
            bad |= group == kNoGroup;
        }
    };
    // Rotating in place, a thread's partners are another thread's output: all heads of a turn are read before any is written, and no two turns share a head.
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) finish(first + i * kStep, data[i]);
    for (int h0 = kAhead * kStep; h0 < heads; h0 += kAhead * kStep) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(h0 + first + i * kStep, data[i]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) finish(h0 + first + i * kStep, data[i]);
    }
    if (bad) report(P.dev_status, MATQ_ERR_NONFINITE);
}

}  // namespace kva4
}  // namespace matq

extern "C" int64_t matq_kv4_tile_bytes(int head_dim) { return head_dim == 64 || head_dim == 128 || head_dim == 256 ? matq::kv4::tile_bytes(head_dim) : -1; }

extern "C" int matq_kv4_append(const matq_paged_kv4* cache, int64_t T, const void* q, int q_heads, int64_t ldq, const void* k, int64_t ldk,
                               const void* v, int64_t ldv, const float* cos_sin, int64_t max_pos, int rot_dim, int interleaved,
                               void* q_out, int64_t ldqo, int32_t* dev_status, void* stream) {
    using namespace matq;
    using namespace matq::kva4;
    if (!cache || T < 0 || q_heads < 0 || cache->batch < 0 || cache->n_pages < 0 || cache->page_size < 1 || cache->kv_heads < 1 ||
        cache->head_dim < 1 || cache->table_width < 0 || (cache->batch > 1 && cache->table_stride < cache->table_width) || max_pos < 0 || rot_dim < 0)
        return MATQ_ERR_INVALID_ARG;
    if ((q == nullptr) != (q_out == nullptr)) return MATQ_ERR_INVALID_ARG;
    if (rot_dim > 0 && !cos_sin) return MATQ_ERR_INVALID_ARG;
    const int D = cache->head_dim;
    if ((D != 64 && D != 128 && D != 256) || cache->page_size % kv4::kTileKeys != 0) return MATQ_ERR_UNSUPPORTED;
    if (rot_dim % 16 != 0 || rot_dim > D || T >= (1ll << 31)) return MATQ_ERR_SHAPE;
    if (!q) q_heads = 0;
    const int64_t kvw = (int64_t)cache->kv_heads * D, qw = (int64_t)q_heads * D;
    if (q_heads + 2ll * cache->kv_heads > (1 << 30)) return MATQ_ERR_SHAPE;
    if (ldk < kvw || ldk % 8 != 0 || ldv < kvw || ldv % 8 != 0 || (q && (ldq < qw || ldq % 8 != 0 || ldqo < qw || ldqo % 8 != 0))) return MATQ_ERR_SHAPE;
    if (T == 0 || cache->batch == 0) return MATQ_OK;
    if (!k || !v || !cache->tiles || !cache->page_table || !cache->cu_q || !cache->kv_len) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || !aligned16(cache->tiles) || !aligned16(q) || !aligned16(q_out) || !aligned16(cos_sin)) return MATQ_ERR_ALIGNMENT;
    if (q && q == q_out && ldq != ldqo) return MATQ_ERR_INVALID_ARG;
    Params P;
    P.cache = static_cast<uint8_t*>(cache->tiles);
    P.table = cache->page_table; P.cu_q = cache->cu_q; P.kv_len = cache->kv_len;
    P.n_pages = cache->n_pages; P.table_stride = cache->table_stride; P.table_width = cache->table_width;
    P.page_size = cache->page_size; P.kv_heads = cache->kv_heads; P.q_heads = q_heads; P.batch = cache->batch;
    P.q = static_cast<const __nv_bfloat16*>(q); P.k = static_cast<const __nv_bfloat16*>(k); P.v = static_cast<const __nv_bfloat16*>(v);
    P.ldq = ldq; P.ldk = ldk; P.ldv = ldv; P.ldqo = ldqo;
    P.cos_sin = cos_sin; P.max_pos = max_pos; P.rot = rot_dim; P.interleaved = interleaved ? 1 : 0;
    P.q_out = static_cast<__nv_bfloat16*>(q_out);
    P.dev_status = dev_status;
    const bool many = T >= kMany;
    const auto kernel = D == 64 ? (many ? kv4_append_kernel<64, kThreadsMany> : kv4_append_kernel<64, kThreadsFew>)
                        : D == 128 ? (many ? kv4_append_kernel<128, kThreadsMany> : kv4_append_kernel<128, kThreadsFew>)
                                   : (many ? kv4_append_kernel<256, kThreadsMany> : kv4_append_kernel<256, kThreadsFew>);
    const cudaError_t e = launch_overlapped(kernel, dim3((unsigned)T), dim3(many ? kThreadsMany : kThreadsFew), 0, static_cast<cudaStream_t>(stream), P);
    if (e != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}
