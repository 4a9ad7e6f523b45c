// New tokens into the paged cache, keys and queries rotated by their positions on the way:
//   (x, y) -> (x cos - y sin, x sin + y cos), the angle's cosine and sine read from an fp32 table.
//
// One pass over q, k and v: each thread takes 16 entries of a head at a time, which are the two halves of
// 8 pairs (HALF: 8 entries at j and 8 at j + rot/2; PAIRS: 16 neighbours), 16 entries behind the rotated
// part, or 16 of v.  Both ends of a pair are in one thread, so q may be turned in place.
#include "common.cuh"
#include "layer.h"
#include "vec8.cuh"

namespace griffin {

struct AppendParams {
    const void *q, *k, *v;
    void *q_out, *k_cache, *v_cache;
    const float *table;
    const int *q_start, *seq_len, *page_table;
    void *ws;
    long long ld_q, ld_k, ld_v, ld_q_out, stride_page, stride_head, stride_token;
    int n_seq, n_pages, table_stride, prefix_len, page_shift;
    int hq, hkv, d, rot, n_pos, style, groups_qk, groups_v;  // groups: 16-entry pieces of one head
};

constexpr int APPEND_THREADS = 128;

template <typename T>
__global__ void __launch_bounds__(APPEND_THREADS) kv_append_kernel(const __grid_constant__ AppendParams p) {
    const int t = blockIdx.x;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    // the token's sequence: how many sequences end at or before it (empty ones included)
    int seq = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += APPEND_THREADS) {
        const int s = s0 + threadIdx.x;
        seq += __syncthreads_count(s < p.n_seq && __ldg(p.q_start + s + 1) <= t);
    }
    if (seq >= p.n_seq) return;  // a row behind the last sequence
    const int i = __ldg(p.seq_len + seq) - (__ldg(p.q_start + seq + 1) - t);
    const int pos = p.prefix_len + i;
    long long at = -1;  // the token's place in the cache, in elements; -1: it has none
    if (i >= 0) {
        const int col = i >> p.page_shift;
        const int page = col < p.table_stride ? __ldg(p.page_table + (long long)seq * p.table_stride + col) : -1;
        if (page >= 0 && page < p.n_pages && (p.rot == 0 || pos < p.n_pos))
            at = page * p.stride_page + (i & ((1 << p.page_shift) - 1)) * p.stride_token;
        else if (threadIdx.x == 0 && blockIdx.y == 0)
            raise_status(p.ws, DEV_STATUS_BAD_INDEX, 40);
    }

    const int hq = p.q != nullptr ? p.hq : 0;
    const int n_qk = (hq + p.hkv) * p.groups_qk, n = n_qk + p.hkv * p.groups_v;
    for (int it = blockIdx.y * APPEND_THREADS + threadIdx.x; it < n; it += gridDim.y * APPEND_THREADS) {
        const bool is_v = it >= n_qk;
        const int per = is_v ? p.groups_v : p.groups_qk, j = is_v ? it - n_qk : it;
        int head = j / per;
        const int piece = j - head * per;
        const void *src;
        void *dst;
        long long from, to;
        bool to_q = false;
        if (is_v) {
            src = p.v; from = t * p.ld_v + head * p.d;
            dst = p.v_cache; to = at + head * p.stride_head;
        } else if (head < hq) {
            src = p.q; from = t * p.ld_q + head * p.d;
            dst = p.q_out; to = t * p.ld_q_out + head * p.d;
            to_q = true;
        } else {
            head -= hq;
            src = p.k; from = t * p.ld_k + head * p.d;
            dst = p.k_cache; to = at + head * p.stride_head;
        }
        if (!to_q && at < 0) continue;
        const int turned = is_v ? 0 : p.rot >> 4;  // pieces of the head that turn
        float a[8], b[8];
        if (piece < turned) {
            const int e0 = p.style == GRIFFIN_ROPE_HALF ? piece * 8 : piece * 16;
            const int e1 = p.style == GRIFFIN_ROPE_HALF ? (p.rot >> 1) + piece * 8 : piece * 16 + 8;
            load8<T>(src, from + e0, a);
            load8<T>(src, from + e1, b);
            if (at >= 0) {
                float c[8], s[8];
                const float *row = p.table + (long long)pos * p.rot + piece * 8;
                load8<float>(row, 0, c);
                load8<float>(row, p.rot >> 1, s);
                if (p.style == GRIFFIN_ROPE_HALF) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = a[e], y = b[e];
                        a[e] = x * c[e] - y * s[e];
                        b[e] = x * s[e] + y * c[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float x0 = a[e], y0 = a[e + 1], x1 = b[e], y1 = b[e + 1];
                        a[e] = x0 * c[e >> 1] - y0 * s[e >> 1];
                        a[e + 1] = x0 * s[e >> 1] + y0 * c[e >> 1];
                        b[e] = x1 * c[4 + (e >> 1)] - y1 * s[4 + (e >> 1)];
                        b[e + 1] = x1 * s[4 + (e >> 1)] + y1 * c[4 + (e >> 1)];
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] = b[e] = 0.f;  // padding, or a token that could not be placed
            }
            store8<T>(dst, to + e0, a);
            store8<T>(dst, to + e1, b);
        } else {
            const int e0 = (is_v ? 0 : p.rot) + (piece - turned) * 16, n8 = e0 + 8 < p.d ? 2 : 1;
            for (int h = 0; h < n8; ++h) {
                load8<T>(src, from + e0 + h * 8, a);
                if (at < 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) a[e] = 0.f;
                }
                store8<T>(dst, to + e0 + h * 8, a);
            }
        }
    }
}

griffin_status launch_kv_append(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                const griffin_kv_cache *cache, const griffin_rope *rope, const void *q, int64_t ld_q,
                                const void *k, int64_t ld_k, const void *v, int64_t ld_v, void *q_out, int64_t ld_q_out,
                                void *ws, cudaStream_t stream) {
    AppendParams p{};
    p.q = q; p.k = k; p.v = v; p.q_out = q_out; p.k_cache = cache->k; p.v_cache = cache->v;
    p.q_start = batch->q_start; p.seq_len = batch->seq_len; p.page_table = batch->page_table;
    p.ws = ws;
    p.ld_q = ld_q; p.ld_k = ld_k; p.ld_v = ld_v; p.ld_q_out = ld_q_out;
    p.stride_page = cache->stride_page; p.stride_head = cache->stride_head; p.stride_token = cache->stride_token;
    p.n_seq = batch->n_seq; p.n_pages = cache->n_pages; p.table_stride = batch->table_stride; p.prefix_len = batch->prefix_len;
    while ((1 << p.page_shift) < desc->page_size) ++p.page_shift;
    p.hq = desc->n_q_heads; p.hkv = desc->n_kv_heads; p.d = desc->head_dim;
    if (rope != nullptr) {
        p.table = rope->table; p.rot = rope->rot_dim; p.n_pos = rope->n_pos; p.style = rope->style;
    }
    p.groups_qk = (p.rot >> 4) + (p.d - p.rot + 15) / 16;
    p.groups_v = (p.d + 15) / 16;
    const int n = ((q != nullptr ? p.hq : 0) + p.hkv) * p.groups_qk + p.hkv * p.groups_v;
    // the pieces of one token on several CTAs while the tokens alone do not fill the device, else three
    // pieces per thread
    const int sms = device_sm_count();
    if (sms <= 0) return GRIFFIN_ERR_CUDA;
    const int full = (n + APPEND_THREADS - 1) / APPEND_THREADS;
    const int y = batch->n_tokens >= 4 * sms ? (full + 2) / 3 : full;
    const void *fn = desc->dtype == GRIFFIN_DT_F32 ? reinterpret_cast<const void *>(kv_append_kernel<float>)
                                                   : reinterpret_cast<const void *>(kv_append_kernel<__nv_bfloat16>);
    void *args[] = {&p};
    return launch_maybe_overlapped(fn, dim3(batch->n_tokens, y), dim3(APPEND_THREADS), 0, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
