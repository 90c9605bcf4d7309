// matq_kv_append: new keys and values into a paged cache, keys and queries rotated by their positions on the way.
//
// Every element is read once and written once and meets three or four operations: HBM-bound for prompts, a chain of four trips to memory
// (sequence bounds -> length -> page and angles -> store) for a decode step.  A CTA takes one token; a thread takes pieces of
// 16 bytes.  With halves as pairs a piece is eight elements of the first half together with their partners, so that each thread
// holds both members of its pairs; neighbouring elements as pairs lie within one piece.  The data loads do not depend on the position and are
// issued before it is known.
#include "common.cuh"

namespace matq {
namespace kva {

constexpr int kThreads = 256;

struct Params {
    __nv_bfloat16 *kc, *vc;
    const int32_t *table, *cu_q, *kv_len;
    int64_t n_pages, table_stride, table_width;
    int page_size, kv_heads, q_heads, D, batch;
    const __nv_bfloat16 *q, *k, *v;
    int64_t ldq, ldk, ldv, ldqo;
    const float* cos_sin;
    int64_t max_pos;
    int rot, interleaved;
    __nv_bfloat16* q_out;
    int32_t* dev_status;
};

__device__ __forceinline__ void unpack8(uint4 v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

// One piece of work of a token: `a` (and its partner `b` when the piece holds the first members of eight pairs)
struct Piece {
    const uint4* src;
    const uint4* src2;
    int head, elem, kind;       // kind 0 query, 1 key, 2 value
    bool live;
};

__global__ void __launch_bounds__(kThreads) kv_append_kernel(const Params P) {
    after_previous_kernel();
    let_next_kernel_start();
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31;
    const int halves = P.interleaved ? 0 : P.rot / 16;                 // pieces of two 16-byte halves per rotated head
    const int rot_pieces = P.interleaved ? P.rot / 8 : halves;
    const int per_head = rot_pieces + (P.D - P.rot) / 8, per_v = P.D / 8;
    const int n_rot = (P.q_heads + P.kv_heads) * per_head, total = n_rot + P.kv_heads * per_v;

    auto piece = [&](int i) {
        Piece w;
        w.live = i < total;
        w.src2 = nullptr;
        w.src = nullptr;
        w.head = w.elem = w.kind = 0;
        if (!w.live) return w;
        if (i < n_rot) {
            w.head = i / per_head;
            const int j = i - w.head * per_head;
            w.elem = j < rot_pieces ? j * 8 : P.rot + (j - rot_pieces) * 8;
            const bool is_q = w.head < P.q_heads;
            if (!is_q) w.head -= P.q_heads;
            w.kind = is_q ? 0 : 1;
            const __nv_bfloat16* base = is_q ? P.q + t * P.ldq : P.k + t * P.ldk;
            base += (int64_t)w.head * P.D + w.elem;
            w.src = reinterpret_cast<const uint4*>(base);
            if (j < halves) w.src2 = reinterpret_cast<const uint4*>(base + P.rot / 2);
        } else {
            const int j = i - n_rot;
            w.head = j / per_v;
            w.elem = (j - w.head * per_v) * 8;
            w.kind = 2;
            w.src = reinterpret_cast<const uint4*>(P.v + t * P.ldv + (int64_t)w.head * P.D + w.elem);
        }
        return w;
    };

    // the token's sequence: the number of sequences that end at or before it (32 bounds per step, every warp for itself)
    int b = 0;
    for (int at = 0; at < P.batch; at += 32) {
        const int i = at + lane;
        const int end = i < P.batch ? P.cu_q[i + 1] : 0x7fffffff;
        b += __popc(__ballot_sync(0xffffffffu, (int64_t)end <= t));
    }
    if (b >= P.batch) return;                                          // a row that belongs to no sequence
    const int64_t q0 = P.cu_q[b], q1 = P.cu_q[b + 1];
    const int64_t pos = (int64_t)P.kv_len[b] - (q1 - q0) + (t - q0);
    const int64_t pg = pos / P.page_size;
    bool ok = pos >= 0 && t >= q0 && pg < P.table_width && (P.rot == 0 || pos < P.max_pos);
    int64_t page = 0;
    if (ok) {
        page = P.table[(int64_t)b * P.table_stride + pg];
        ok = page >= 0 && page < P.n_pages;
    }
    if (!ok) {
        if (tid == 0) report(P.dev_status, MATQ_ERR_PAGE);
        return;
    }
    const int64_t slot = pos - pg * P.page_size;
    const float* cs = P.cos_sin + pos * P.rot;
    const int half = P.rot / 2;

    for (int i = tid; i < total; i += kThreads) {
        const Piece w = piece(i);
        const uint4 a = *w.src;
        __nv_bfloat16* dst;
        if (w.kind == 0) dst = P.q_out + t * P.ldqo + (int64_t)w.head * P.D;
        else dst = (w.kind == 1 ? P.kc : P.vc) + ((page * P.kv_heads + w.head) * P.page_size + slot) * P.D;
        dst += w.elem;
        if (w.src2) {
            const uint4 b4 = *w.src2;
            float x[8], y[8], ox[8], oy[8], c[8], s[8];
            unpack8(a, x);
            unpack8(b4, y);
            *reinterpret_cast<float4*>(c) = *reinterpret_cast<const float4*>(cs + w.elem);
            *reinterpret_cast<float4*>(c + 4) = *reinterpret_cast<const float4*>(cs + w.elem + 4);
            *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(cs + half + w.elem);
            *reinterpret_cast<float4*>(s + 4) = *reinterpret_cast<const float4*>(cs + half + w.elem + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ox[e] = x[e] * c[e] - y[e] * s[e];
                oy[e] = y[e] * c[e] + x[e] * s[e];
            }
            *reinterpret_cast<uint4*>(dst) = pack8(ox);
            *reinterpret_cast<uint4*>(dst + half) = pack8(oy);
        } else if (w.kind < 2 && w.elem < P.rot) {                     // neighbouring elements are pairs
            float x[8], o[8];
            unpack8(a, x);
            const float4 c = *reinterpret_cast<const float4*>(cs + w.elem / 2);
            const float4 s = *reinterpret_cast<const float4*>(cs + half + w.elem / 2);
            const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[2 * e] = x[2 * e] * cc[e] - x[2 * e + 1] * ss[e];
                o[2 * e + 1] = x[2 * e + 1] * cc[e] + x[2 * e] * ss[e];
            }
            *reinterpret_cast<uint4*>(dst) = pack8(o);
        } else {
            *reinterpret_cast<uint4*>(dst) = a;
        }
    }
}

}  // namespace kva
}  // namespace matq

extern "C" int matq_kv_append(const matq_paged_kv* cache, int64_t T, const void* q, int q_heads, int64_t ldq, const void* k, int64_t ldk,
                              const void* v, int64_t ldv, const float* cos_sin, int64_t max_pos, int rot_dim, int interleaved,
                              void* q_out, int64_t ldqo, int32_t* dev_status, void* stream) {
    using namespace matq;
    using namespace matq::kva;
    if (!cache || T < 0 || q_heads < 0 || cache->batch < 0 || cache->n_pages < 0 || cache->page_size < 1 || cache->kv_heads < 1 ||
        cache->head_dim < 1 || cache->table_width < 0 || (cache->batch > 1 && cache->table_stride < cache->table_width) || max_pos < 0 || rot_dim < 0)
        return MATQ_ERR_INVALID_ARG;
    if ((q == nullptr) != (q_out == nullptr)) return MATQ_ERR_INVALID_ARG;
    if (rot_dim > 0 && !cos_sin) return MATQ_ERR_INVALID_ARG;
    const int D = cache->head_dim;
    if (D % 8 != 0 || rot_dim % 16 != 0 || rot_dim > D || T >= (1ll << 31)) return MATQ_ERR_SHAPE;
    if (!q) q_heads = 0;
    const int64_t kvw = (int64_t)cache->kv_heads * D, qw = (int64_t)q_heads * D;
    if (ldk < kvw || ldk % 8 != 0 || ldv < kvw || ldv % 8 != 0 || (q && (ldq < qw || ldq % 8 != 0 || ldqo < qw || ldqo % 8 != 0))) return MATQ_ERR_SHAPE;
    if (T == 0 || cache->batch == 0) return MATQ_OK;
    if (!k || !v || !cache->k || !cache->v || !cache->page_table || !cache->cu_q || !cache->kv_len) return MATQ_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || !aligned16(cache->k) || !aligned16(cache->v) || !aligned16(q) || !aligned16(q_out) || !aligned16(cos_sin))
        return MATQ_ERR_ALIGNMENT;
    if (q && q == q_out && ldq != ldqo) return MATQ_ERR_INVALID_ARG;
    Params P;
    P.kc = static_cast<__nv_bfloat16*>(cache->k); P.vc = static_cast<__nv_bfloat16*>(cache->v);
    P.table = cache->page_table; P.cu_q = cache->cu_q; P.kv_len = cache->kv_len;
    P.n_pages = cache->n_pages; P.table_stride = cache->table_stride; P.table_width = cache->table_width;
    P.page_size = cache->page_size; P.kv_heads = cache->kv_heads; P.q_heads = q_heads; P.D = D; P.batch = cache->batch;
    P.q = static_cast<const __nv_bfloat16*>(q); P.k = static_cast<const __nv_bfloat16*>(k); P.v = static_cast<const __nv_bfloat16*>(v);
    P.ldq = ldq; P.ldk = ldk; P.ldv = ldv; P.ldqo = ldqo;
    P.cos_sin = cos_sin; P.max_pos = max_pos; P.rot = rot_dim; P.interleaved = interleaved ? 1 : 0;
    P.q_out = static_cast<__nv_bfloat16*>(q_out);
    P.dev_status = dev_status;
    const cudaError_t e = launch_overlapped(kv_append_kernel, dim3((unsigned)T), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), P);
    if (e != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}
