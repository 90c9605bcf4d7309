// matq_kv4_append: new keys and values into a paged cache held in 4-bit groups, keys and queries rotated by their positions on the way.
//
// As matq_kv_append (a CTA per token, a thread keeps its place within the heads, angles in registers, the first heads requested before the position is known),
// but a thread's place is eight neighbouring elements, which is what it quantises: with halves as pairs it reads its eight partners beside them (from L1, where
// the thread that owns them has brought them), and the eight lanes of a group exchange its ends.
#include "kv4_cache.cuh"

namespace matq {
namespace kva4 {

constexpr int kThreads = 256;

struct Params {
    uint8_t* cache;
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

constexpr int kAhead = 2;        // heads per thread whose data are requested before the position is known

__global__ void __launch_bounds__(kThreads, 4) kv4_append_kernel(const Params P) {
    after_previous_kernel();
    let_next_kernel_start();
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31;
    const int heads = P.q_heads + 2 * P.kv_heads, half = P.rot / 2;
    const int places = P.D / 8, step = kThreads / places;              // 8, 16 or 32 threads along a head; heads side by side
    const int first = tid / places, e0 = (tid - first * places) * 8;
    const bool turns = e0 < P.rot, paired = turns && !P.interleaved, upper = paired && e0 >= half;
    const int partner = paired ? upper ? e0 - half : e0 + half : e0;
    uint4 data[kAhead][2];
    const auto load = [&](int hd, uint4 (&d)[2]) {
        d[0] = d[1] = make_uint4(0u, 0u, 0u, 0u);
        if (hd >= heads) return;
        const bool value = hd >= P.q_heads + P.kv_heads;
        const __nv_bfloat16* row = hd < P.q_heads ? P.q + t * P.ldq + (int64_t)hd * P.D
                                   : value ? P.v + t * P.ldv + (int64_t)(hd - P.q_heads - P.kv_heads) * P.D : P.k + t * P.ldk + (int64_t)(hd - P.q_heads) * P.D;
        d[0] = *reinterpret_cast<const uint4*>(row + e0);
        if (paired && !value) d[1] = *reinterpret_cast<const uint4*>(row + partner);
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
    const int slot = (int)(pos - pg * P.page_size);
    // angles: of eight pairs when pairs are halves apart, of four when they are neighbours
    float c[8], s[8];
    if (turns) {
        const float* cs = P.cos_sin + pos * P.rot + (paired ? upper ? e0 - half : e0 : e0 / 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i == 1 && !paired) break;
            const float4 cv = *reinterpret_cast<const float4*>(cs + 4 * i), sv = *reinterpret_cast<const float4*>(cs + half + 4 * i);
            c[4 * i] = cv.x; c[4 * i + 1] = cv.y; c[4 * i + 2] = cv.z; c[4 * i + 3] = cv.w;
            s[4 * i] = sv.x; s[4 * i + 1] = sv.y; s[4 * i + 2] = sv.z; s[4 * i + 3] = sv.w;
        }
    }
    // Every product and sum is rounded by itself: the values that are quantised are defined bit for bit.
    const auto turned = [&](const uint4 (&d)[2]) {
        const uint32_t o[4] = {d[0].x, d[0].y, d[0].z, d[0].w}, p[4] = {d[1].x, d[1].y, d[1].z, d[1].w};
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x0 = __uint_as_float(o[i] << 16), x1 = __uint_as_float(o[i] & 0xffff0000u);
            float y0, y1;
            if (paired) {
                const float z0 = __uint_as_float(p[i] << 16), z1 = __uint_as_float(p[i] & 0xffff0000u);
                const float u0 = __fmul_rn(x0, c[2 * i]), u1 = __fmul_rn(x1, c[2 * i + 1]), w0 = __fmul_rn(z0, s[2 * i]), w1 = __fmul_rn(z1, s[2 * i + 1]);
                y0 = upper ? __fadd_rn(u0, w0) : __fsub_rn(u0, w0);
                y1 = upper ? __fadd_rn(u1, w1) : __fsub_rn(u1, w1);
            } else {
                y0 = __fsub_rn(__fmul_rn(x0, c[i]), __fmul_rn(x1, s[i]));
                y1 = __fadd_rn(__fmul_rn(x1, c[i]), __fmul_rn(x0, s[i]));
            }
            r[i] = bf16_rne(y0) | (bf16_rne(y1) << 16);
        }
        return make_uint4(r[0], r[1], r[2], r[3]);
    };
    bool bad = false;
    const auto finish = [&](int hd, const uint4 (&d)[2]) {
        if (hd >= heads) return;                                        // the lanes of a group share their head
        const bool value = hd >= P.q_heads + P.kv_heads;
        const uint4 x = turns && !value ? turned(d) : d[0];
        if (hd < P.q_heads) {
            *reinterpret_cast<uint4*>(P.q_out + t * P.ldqo + (int64_t)hd * P.D + e0) = x;
            return;
        }
        uint32_t codes;
        const uint32_t group = quantise_piece<8>(x, codes, 0xffu << (lane & 24));
        const int h = hd - P.q_heads - (value ? P.kv_heads : 0), key = slot % kv4::kTileKeys;
        uint8_t* tile = P.cache + ((page * P.kv_heads + h) * (P.page_size / kv4::kTileKeys) + slot / kv4::kTileKeys) * kv4::tile_bytes(P.D) + (value ? kv4::half_bytes(P.D) : 0);
        *reinterpret_cast<uint32_t*>(tile + (e0 / 32) * 256 + key * 16 + (e0 % 32) / 2) = codes;
        if ((lane & 7) == 0) {
            *reinterpret_cast<uint32_t*>(tile + kv4::groups_at(P.D) + (e0 / 64) * 64 + key * 4) = group;
            bad |= group == kNoGroup;
        }
    };
    // Rotating in place, a thread's partners are another thread's output: all heads of a turn are read before any is written, and no two turns share a head.
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) finish(first + i * step, data[i]);
    for (int h0 = kAhead * step; h0 < heads; h0 += kAhead * step) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(h0 + first + i * step, data[i]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) finish(h0 + first + i * step, data[i]);
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
    P.page_size = cache->page_size; P.kv_heads = cache->kv_heads; P.q_heads = q_heads; P.D = D; P.batch = cache->batch;
    P.q = static_cast<const __nv_bfloat16*>(q); P.k = static_cast<const __nv_bfloat16*>(k); P.v = static_cast<const __nv_bfloat16*>(v);
    P.ldq = ldq; P.ldk = ldk; P.ldv = ldv; P.ldqo = ldqo;
    P.cos_sin = cos_sin; P.max_pos = max_pos; P.rot = rot_dim; P.interleaved = interleaved ? 1 : 0;
    P.q_out = static_cast<__nv_bfloat16*>(q_out);
    P.dev_status = dev_status;
    const cudaError_t e = launch_overlapped(kv4_append_kernel, dim3((unsigned)T), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), P);
    if (e != cudaSuccess) { cudaGetLastError(); return MATQ_ERR_CUDA; }
    return launch_status();
}
