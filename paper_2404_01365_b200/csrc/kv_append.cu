// New tokens into the paged cache, keys and queries rotated by their positions on the way:
//   (x, y) -> (x cos - y sin, x sin + y cos), the angle's cosine and sine read from an fp32 table.
//
// One pass over q, k and v.  A thread takes one piece of one head, of TPC tokens: the two halves
// of 8 pairs (HALF: 8 entries at j and 8 at j + rot/2; PAIRS: 16 neighbours), or 16 entries that do not turn (behind the
// rotated part, or of v).  Both ends of a pair are in one thread, so q may be turned in place.
//
// A token's place takes three dependent trips to L2 (sequence, length, page) and its angles a fourth: the CTA takes
// them for its TPC tokens together (with more than one, the angles through shared memory: every head wants the
// same ones), while the data of all the tokens is on the way.
//
// Bound by memory where there is much of it: 4096 tokens of 32 query heads and 8 key heads of 128, bf16 (101 MB), take
// 20.7 us, 4.9 TB/s, where a copy of the same bytes takes 16; 8 tokens of 40 heads take 2.1 us, the launch and the trips.
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
    int n_tokens, n_seq, n_pages, table_stride, prefix_len, page_shift;
    int hq, hkv, d, rot, n_pos, style;
};

constexpr int APPEND_THREADS = 128;

template <typename T> struct Piece {  // a thread's two times 8 entries, as they lie in memory
    uint4 v[sizeof(T)];               // (bf16: one 16-byte word for 8 entries; fp32: two)
};
template <typename T> __device__ __forceinline__ void load_half(Piece<T> &p, int half, const T *at) {
    constexpr int N = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < N; ++i) p.v[half * N + i] = reinterpret_cast<const uint4 *>(at)[i];
}
template <typename T> __device__ __forceinline__ void store_half(const Piece<T> &p, int half, T *at) {
    constexpr int N = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<uint4 *>(at)[i] = p.v[half * N + i];
}
template <typename T> __device__ __forceinline__ void get_half(const Piece<T> &p, int half, float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        Elem<__nv_bfloat16>::unpack(p.v[half], f);
    } else {
        const uint4 a = p.v[2 * half], b = p.v[2 * half + 1];
        f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
        f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
    }
}

template <typename T, int TPC>
__global__ void __launch_bounds__(APPEND_THREADS) kv_append_kernel(const __grid_constant__ AppendParams p) {
    __shared__ long long s_at[TPC];   // the tokens' places in the cache, in elements; -1: none; -2: of no sequence
    __shared__ int s_pos[TPC];
    __shared__ __align__(16) float s_table[TPC][TPC > 1 ? 256 : 4];
    const int t0 = blockIdx.x * TPC, pieces = (p.d + 15) >> 4, per_round = APPEND_THREADS / pieces;  // heads side by side
    const int slot = threadIdx.x / pieces, piece = threadIdx.x - slot * pieces, turned = p.rot >> 4;
    const int hq = p.q != nullptr ? p.hq : 0, h = blockIdx.y * per_round + slot;
    const bool on = slot < per_round && h < hq + 2 * p.hkv, is_v = h >= hq + p.hkv, is_q = h < hq;   // heads: q, k, v
    const bool turn = on && !is_v && piece < turned;
    const int e0 = turn && p.style == GRIFFIN_ROPE_HALF ? piece * 8 : piece * 16;
    const int e1 = turn && p.style == GRIFFIN_ROPE_HALF ? (p.rot >> 1) + piece * 8 : piece * 16 + 8;
    const bool two = e1 < p.d;        // (the last piece of a head may be one of 8)
    const T *const src = static_cast<const T *>(is_q ? p.q : is_v ? p.v : p.k) + (is_q ? h : is_v ? h - hq - p.hkv : h - hq) * p.d;
    const long long ld = is_q ? p.ld_q : is_v ? p.ld_v : p.ld_k;
    pdl_launch_dependents();
    pdl_wait_prior_grids();

    Piece<T> x[TPC];
#pragma unroll
    for (int u = 0; u < TPC; ++u)
        if (on && t0 + u < p.n_tokens) {
            load_half<T>(x[u], 0, src + (t0 + u) * ld + e0);
            if (two) load_half<T>(x[u], 1, src + (t0 + u) * ld + e1);
        }
    // the first token's sequence: how many sequences end at or before it (empty ones included)
    int seq = 0;
    if (p.n_seq > 1) {
        for (int s0 = 0; s0 < p.n_seq; s0 += APPEND_THREADS) {
            const int s = s0 + threadIdx.x;
            seq += __syncthreads_count(s < p.n_seq && __ldg(p.q_start + s + 1) <= t0);
        }
    }
    // a token's place and position (with one token every thread looks them up for itself)
    long long at1 = -2;
    int pos1 = 0;
    if (TPC == 1 || threadIdx.x < TPC) {
        const int t = TPC == 1 ? t0 : t0 + threadIdx.x;
        if (TPC > 1 || p.n_seq == 1)  // (otherwise the count above was this token's)
            while (seq < p.n_seq && __ldg(p.q_start + seq + 1) <= t) ++seq;
        int first = t + 1, end = 0, len = 0;   // (three loads in one trip)
        if (seq < p.n_seq && t < p.n_tokens) {
            first = __ldg(p.q_start + seq);
            end = __ldg(p.q_start + seq + 1);
            len = __ldg(p.seq_len + seq);
        }
        if (t >= first) {   // (rows in front of the first sequence's, as those behind the last one's, belong to none)
            const long long own = (long long)len - (end - t);   // index among its own tokens
            const int k = (int)max(min(own, (long long)GRIFFIN_MAX_ATTN_TOKENS), -1ll);
            at1 = -1;
            pos1 = p.prefix_len + k;   // (2^31 - 1 at most for an index below the limit)
            if (k >= 0) {
                const int col = k >> p.page_shift;
                const int page = k < GRIFFIN_MAX_ATTN_TOKENS && col < p.table_stride ? __ldg(p.page_table + (long long)seq * p.table_stride + col) : -1;
                if (page >= 0 && page < p.n_pages && (p.rot == 0 || pos1 < p.n_pos))
                    at1 = page * p.stride_page + (k & ((1 << p.page_shift) - 1)) * p.stride_token;
                else if (blockIdx.y == 0 && threadIdx.x < TPC)
                    raise_status(p.ws, DEV_STATUS_BAD_INDEX, 40);
            }
        }
        if (TPC > 1) {
            s_at[threadIdx.x] = at1;
            s_pos[threadIdx.x] = pos1;
        }
    }
    if (TPC > 1) __syncthreads();
    if (TPC > 1 && p.rot > 0) {
        const int quads = p.rot >> 2;
        for (int i = threadIdx.x; i < TPC * quads; i += APPEND_THREADS) {
            const int u = i / quads, e = (i - u * quads) * 4;
            if (s_at[u] >= 0)
                *reinterpret_cast<float4 *>(&s_table[u][e]) = __ldg(reinterpret_cast<const float4 *>(p.table + (long long)s_pos[u] * p.rot + e));
        }
        __syncthreads();
    }
    if (!on) return;
    T *const cache = static_cast<T *>(is_v ? p.v_cache : p.k_cache) + (is_v ? h - hq - p.hkv : h - hq) * p.stride_head;
#pragma unroll
    for (int u = 0; u < TPC; ++u) {
        const long long at = TPC > 1 ? s_at[u] : at1;
        if (at == -2) continue;
        const int t = t0 + u;
        if (at < 0) {   // padding, or a token that could not be placed
            if (!is_q) continue;
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) x[u].v[i] = make_uint4(0, 0, 0, 0);
        } else if (turn) {
            float a[8], b[8], c[8], s[8];
            const float *const row = TPC > 1 ? s_table[u] : p.table + (long long)pos1 * p.rot;
            load8<float>(row, piece * 8, c);
            load8<float>(row, (p.rot >> 1) + piece * 8, s);
            get_half<T>(x[u], 0, a);
            get_half<T>(x[u], 1, b);
            if (p.style == GRIFFIN_ROPE_HALF) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = a[e], w = b[e];
                    a[e] = v * c[e] - w * s[e];
                    b[e] = v * s[e] + w * c[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float v0 = a[e], w0 = a[e + 1], v1 = b[e], w1 = b[e + 1];
                    a[e] = v0 * c[e >> 1] - w0 * s[e >> 1];
                    a[e + 1] = v0 * s[e >> 1] + w0 * c[e >> 1];
                    b[e] = v1 * c[4 + (e >> 1)] - w1 * s[4 + (e >> 1)];
                    b[e + 1] = v1 * s[4 + (e >> 1)] + w1 * c[4 + (e >> 1)];
                }
            }
            T *const dst = is_q ? static_cast<T *>(p.q_out) + t * p.ld_q_out + h * p.d : cache + at;
            store8<T>(dst, e0, a);
            store8<T>(dst, e1, b);
            continue;
        }
        T *const dst = is_q ? static_cast<T *>(p.q_out) + t * p.ld_q_out + h * p.d : cache + at;
        store_half<T>(x[u], 0, dst + e0);
        if (two) store_half<T>(x[u], 1, dst + e1);
    }
}

// (800 tokens of 16 heads of 80, fp32: 5.4 us one by one, 6.3 in pairs; 4096 tokens of 48 heads of 128, bf16: 21.3 us one by one,
// 20.5 in pairs, 21.0 and 23.7 by four and eight: a copy of the same bytes takes 16)
constexpr int APPEND_TOKENS = 2;
template <typename T> static const void *append_kernel(bool many) {
    return many ? reinterpret_cast<const void *>(kv_append_kernel<T, APPEND_TOKENS>) : reinterpret_cast<const void *>(kv_append_kernel<T, 1>);
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
    p.n_tokens = batch->n_tokens; p.n_seq = batch->n_seq; p.n_pages = cache->n_pages; p.table_stride = batch->table_stride; p.prefix_len = batch->prefix_len;
    while ((1 << p.page_shift) < desc->page_size) ++p.page_shift;
    p.hq = desc->n_q_heads; p.hkv = desc->n_kv_heads; p.d = desc->head_dim;
    if (rope != nullptr) {
        p.table = rope->table; p.rot = rope->rot_dim; p.n_pos = rope->n_pos; p.style = rope->style;
    }
    // several tokens per CTA once there are enough for all SMs
    const int sms = device_sm_count();
    if (sms <= 0) return GRIFFIN_ERR_CUDA;
    const bool many = batch->n_tokens >= 16 * sms;
    const int per_round = APPEND_THREADS / ((p.d + 15) / 16), tpc = many ? APPEND_TOKENS : 1;
    const int x = (batch->n_tokens + tpc - 1) / tpc, y = ((q != nullptr ? p.hq : 0) + 2 * p.hkv + per_round - 1) / per_round;
    const void *fn = desc->dtype == GRIFFIN_DT_F32 ? append_kernel<float>(many) : append_kernel<__nv_bfloat16>(many);
    void *args[] = {&p};
    return launch_maybe_overlapped(fn, dim3(x, y), dim3(APPEND_THREADS), 0, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
