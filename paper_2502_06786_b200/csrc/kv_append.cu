// matq_kv_append: new keys and values into a paged cache, keys and queries rotated by their positions on the way.
//
// Every element is read once and written once and meets three or four operations: HBM-bound for prompts, a chain of trips to memory (sequence bounds
// -> length -> page and angles -> store) for a decode step.  A CTA takes one token; a thread keeps its place within the heads and walks over
// queries, keys and values, so that its angles stay in registers.  A place is two pieces of eight elements: with halves as pairs a piece of the first
// half and its partners, otherwise neighbours.  The data of its first heads are requested before the position is known.
// Three prompts of 1500 to 4000 tokens, 16/8 heads of 256: 60 us = 5.3 TB/s, half of it writes.  64 single tokens, 32/8 heads of 128: 3.2 us.
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

constexpr int kAhead = 2;        // heads per thread whose data are requested before the position is known

__global__ void __launch_bounds__(kThreads, 4) kv_append_kernel(const Params P) {
    after_previous_kernel();
    let_next_kernel_start();
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31;
    const int heads = P.q_heads + 2 * P.kv_heads, half = P.rot / 2;
    const int places = (P.D + 15) / 16, step = kThreads / places;       // threads along a head; heads side by side
    const int y = tid / places, x = tid - y * places;
    const int first = y < step ? y : heads;                             // left-over threads have no head
    // this thread's two pieces of a rotated head, and of a value (or of a head whose pairs are neighbours)
    const bool paired = !P.interleaved && x < P.rot / 16;
    const int e0 = paired ? x * 8 : x * 16, e1 = paired ? half + x * 8 : x * 16 + 8;
    const auto source = [&](int hd, int piece) -> const uint4* {
        if (hd >= heads) return nullptr;
        const bool value = hd >= P.q_heads + P.kv_heads;
        const int e = value ? x * 16 + 8 * piece : piece ? e1 : e0;
        if (e >= P.D) return nullptr;
        const __nv_bfloat16* row = hd < P.q_heads ? P.q + t * P.ldq + (int64_t)hd * P.D
                                   : value ? P.v + t * P.ldv + (int64_t)(hd - P.q_heads - P.kv_heads) * P.D : P.k + t * P.ldk + (int64_t)(hd - P.q_heads) * P.D;
        return reinterpret_cast<const uint4*>(row + e);
    };
    uint4 data[kAhead][2];
    const auto load = [&](int hd, uint4 (&d)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4* p = source(hd, i);
            d[i] = p ? *p : make_uint4(0u, 0u, 0u, 0u);
        }
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
    for (int i = 0; i < kAhead; ++i) load(first + i * step, data[i]);
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
    // angles: of eight pairs when the pieces are partners, of four pairs per piece when neighbours are
    const float* cs = P.cos_sin + pos * P.rot;
    float c[8], s[8];
    const int at = paired ? e0 : e0 / 2;
    const bool turns = P.rot > 0 && (paired || (P.interleaved && e0 < P.rot));       // rot is a multiple of 16: both pieces of a place turn, or neither
    if (turns) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 cv = *reinterpret_cast<const float4*>(cs + at + 4 * i), sv = *reinterpret_cast<const float4*>(cs + half + at + 4 * i);
            c[4 * i] = cv.x; c[4 * i + 1] = cv.y; c[4 * i + 2] = cv.z; c[4 * i + 3] = cv.w;
            s[4 * i] = sv.x; s[4 * i + 1] = sv.y; s[4 * i + 2] = sv.z; s[4 * i + 3] = sv.w;
        }
    }
    const auto finish = [&](int hd, const uint4 (&d)[2]) {
        if (hd >= heads) return;
        const bool value = hd >= P.q_heads + P.kv_heads;
        const int f0 = value ? x * 16 : e0, f1 = value ? x * 16 + 8 : e1;
        __nv_bfloat16* dst;
        if (hd < P.q_heads) {
            dst = P.q_out + t * P.ldqo + (int64_t)hd * P.D;
        } else {
            const int h = hd - P.q_heads - (value ? P.kv_heads : 0);
            dst = (value ? P.vc : P.kc) + ((page * P.kv_heads + h) * P.page_size + slot) * P.D;
        }
        uint4 o0 = d[0], o1 = d[1];
        if (!value && turns) {
            float a[8], b8[8], oa[8], ob[8];
            unpack8(d[0], a);
            unpack8(d[1], b8);
            if (paired) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    oa[e] = a[e] * c[e] - b8[e] * s[e];
                    ob[e] = b8[e] * c[e] + a[e] * s[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    oa[2 * e] = a[2 * e] * c[e] - a[2 * e + 1] * s[e];
                    oa[2 * e + 1] = a[2 * e + 1] * c[e] + a[2 * e] * s[e];
                    ob[2 * e] = b8[2 * e] * c[4 + e] - b8[2 * e + 1] * s[4 + e];
                    ob[2 * e + 1] = b8[2 * e + 1] * c[4 + e] + b8[2 * e] * s[4 + e];
                }
            }
            o0 = pack8(oa);
            o1 = pack8(ob);
        }
        if (f0 < P.D) *reinterpret_cast<uint4*>(dst + f0) = o0;
        if (f1 < P.D) *reinterpret_cast<uint4*>(dst + f1) = o1;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) finish(first + i * step, data[i]);
    for (int hd = first + kAhead * step; hd < heads; hd += kAhead * step) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(hd + i * step, data[i]);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) finish(hd + i * step, data[i]);
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
    if (D % 8 != 0 || rot_dim % 16 != 0 || rot_dim > D || D > 16 * kThreads || T >= (1ll << 31)) return MATQ_ERR_SHAPE;
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
