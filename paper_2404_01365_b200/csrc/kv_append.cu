// New tokens into the paged cache, keys and queries rotated by their positions on the way:
//   (x, y) -> (x cos - y sin, x sin + y cos), the angle's cosine and sine read from an fp32 table.
//
// The cache is in the storage type, or in 4 bits (q4.cuh): then the thread that has a group of 16 entries of a key or value
// quantises it on the way; a turned group of a HALF rotation needs the other ends of its pairs, which it loads as well.
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
// 20.7 us, 4.9 TB/s, where a copy of the same bytes takes 16; 8 tokens of 40 heads take 2.1 us, the launch and the trips.  Into 4 bits
// the same take 23.0 us (88 MB, 3.8 TB/s; a copy 13.5) and 2.5: it issues 2.5 instructions of 4 a clock, the integer
// pipe busy for half of it; with divisions for the quotients it was 27.5.  4096 tokens in fp32 take 38 us (into fp32 35).  For eight
// CTAs to an SM the kernels into 4 bits have 64 registers, of which the two that take tokens in pairs spill 28 (bf16) and 132 bytes (fp32).
#include "common.cuh"
#include "kv_place.cuh"
#include "layer.h"
#include "q4.cuh"
#include "vec8.cuh"

namespace griffin {

struct AppendParams {
    PlaceParams place;
    const void *q, *k, *v;
    void *q_out, *k_cache, *v_cache;
    const float *table;
    long long ld_q, ld_k, ld_v, ld_q_out, stride_page, stride_head, stride_token;   // of the cache held in 4 bits: in bytes
    Q4Layout q4;
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

// A group of 16 entries from e0 on, of a key (turned, where it turns) or a value.  Every product and sum is rounded to fp32 by
// itself, so that the codes are those of the formulas in any other fp32 arithmetic, bit for bit.
template <typename T>
__device__ __forceinline__ void append_group(const Piece<T> &x, const Piece<T> &y, bool turn, int style, int e0, int half, const float *row,
                                             float (&f)[16]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int e = e0 + 8 * i;
        float a[8], c[8], s[8];
        get_half<T>(x, i, a);
        if (turn && style == GRIFFIN_ROPE_HALF) {
            const bool low = e < half;    // (8 entries lie on one side: rot / 2 is a multiple of 8)
            const int j = low ? e : e - half;
            float b[8];
            get_half<T>(y, i, b);
            load8<float>(row, j, c);
            load8<float>(row, half + j, s);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float near = __fmul_rn(a[k], c[k]), far = __fmul_rn(b[k], s[k]);
                a[k] = low ? __fsub_rn(near, far) : __fadd_rn(far, near);
            }
        } else if (turn) {
            const float4 cq = *reinterpret_cast<const float4 *>(row + (e >> 1)), sq = *reinterpret_cast<const float4 *>(row + half + (e >> 1));
            c[0] = cq.x; c[1] = cq.y; c[2] = cq.z; c[3] = cq.w;
            s[0] = sq.x; s[1] = sq.y; s[2] = sq.z; s[3] = sq.w;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float v = a[2 * k], w = a[2 * k + 1];
                a[2 * k] = __fsub_rn(__fmul_rn(v, c[k]), __fmul_rn(w, s[k]));
                a[2 * k + 1] = __fadd_rn(__fmul_rn(v, s[k]), __fmul_rn(w, c[k]));
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) f[8 * i + k] = a[k];
    }
}

template <typename T, int TPC, bool Q4>
__global__ void __launch_bounds__(APPEND_THREADS, Q4 ? 8 : 1) kv_append_kernel(const __grid_constant__ AppendParams p) {
    __shared__ Place s_at[TPC];
    __shared__ __align__(16) float s_table[TPC][TPC > 1 ? 256 : 4];
    const int t0 = blockIdx.x * TPC, pieces = (p.d + 15) >> 4, per_round = APPEND_THREADS / pieces;  // heads side by side
    const int slot = threadIdx.x / pieces, piece = threadIdx.x - slot * pieces, turned = p.rot >> 4, half = p.rot >> 1;
    const int hq = p.q != nullptr ? p.hq : 0, h = blockIdx.y * per_round + slot;
    const bool on = slot < per_round && h < hq + 2 * p.hkv, is_v = h >= hq + p.hkv, is_q = h < hq;   // heads: q, k, v
    const bool turn = on && !is_v && piece < turned;
    // (what is quantised is taken by groups of 16 neighbours, and the other ends of its pairs with it)
    const bool apart = turn && p.style == GRIFFIN_ROPE_HALF && !(Q4 && !is_q), mates = Q4 && turn && !is_q && p.style == GRIFFIN_ROPE_HALF;
    const int e0 = apart ? piece * 8 : piece * 16, e1 = apart ? half + piece * 8 : piece * 16 + 8;
    const int m0 = e0 < half ? e0 + half : e0 - half, m1 = e1 < half ? e1 + half : e1 - half;
    const bool two = e1 < p.d;        // (the last piece of a head may be one of 8)
    const T *const src = static_cast<const T *>(is_q ? p.q : is_v ? p.v : p.k) + (is_q ? h : is_v ? h - hq - p.hkv : h - hq) * p.d;
    const long long ld = is_q ? p.ld_q : is_v ? p.ld_v : p.ld_k;
    pdl_launch_dependents();
    pdl_wait_prior_grids();

    Piece<T> x[TPC], y[Q4 ? TPC : 1];
#pragma unroll
    for (int u = 0; u < TPC; ++u)
        if (on && t0 + u < p.place.n_tokens) {
            load_half<T>(x[u], 0, src + (t0 + u) * ld + e0);
            if (two) load_half<T>(x[u], 1, src + (t0 + u) * ld + e1);
            if constexpr (Q4) {
                if (mates) {
                    load_half<T>(y[u], 0, src + (t0 + u) * ld + m0);
                    load_half<T>(y[u], 1, src + (t0 + u) * ld + m1);
                }
            }
        }
    const Place mine = place_token<TPC, APPEND_THREADS>(p.place, t0, p.rot == 0 ? -1 : p.n_pos);
    if (TPC > 1) {
        if (threadIdx.x < TPC) s_at[threadIdx.x] = mine;
        __syncthreads();
    }
    if (TPC > 1 && p.rot > 0) {
        const int quads = p.rot >> 2;
        for (int i = threadIdx.x; i < TPC * quads; i += APPEND_THREADS) {
            const int u = i / quads, e = (i - u * quads) * 4;
            if (s_at[u].page >= 0)
                *reinterpret_cast<float4 *>(&s_table[u][e]) = __ldg(reinterpret_cast<const float4 *>(p.table + (long long)s_at[u].pos * p.rot + e));
        }
        __syncthreads();
    }
    if (!on) return;
    const long long head = (is_v ? h - hq - p.hkv : h - hq) * p.stride_head;
#pragma unroll
    for (int u = 0; u < TPC; ++u) {
        const Place at = TPC > 1 ? s_at[u] : mine;
        if (at.page == -2) continue;
        const int t = t0 + u;
        const float *const row = TPC > 1 ? s_table[u] : p.table + (long long)at.pos * p.rot;
        if constexpr (Q4) {
            if (!is_q) {
                if (at.page < 0) continue;
                uint8_t *const block = static_cast<uint8_t *>(is_v ? p.v_cache : p.k_cache) + at.page * p.stride_page + head;
                float f[16];
                append_group<T>(x[u], y[u], turn, p.style, e0, half, row, f);
                uint2 codes;
                const uint32_t scale = q4_quantise(f, codes);
                *reinterpret_cast<uint2 *>(block + at.slot * p.q4.code_row + piece * 8) = codes;
                block[p.q4.scale_off + at.slot * p.q4.scale_row + piece] = (uint8_t)scale;
                continue;
            }
        }
        T *const to = is_q ? static_cast<T *>(p.q_out) + t * p.ld_q_out + h * p.d
                           : static_cast<T *>(is_v ? p.v_cache : p.k_cache) + head + at.page * p.stride_page + at.slot * p.stride_token;
        if (at.page < 0) {   // padding, or a token that could not be placed
            if (!is_q) continue;
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) x[u].v[i] = make_uint4(0, 0, 0, 0);
        } else if (turn) {
            float a[8], b[8], c[8], s[8];
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
            store8<T>(to, e0, a);
            store8<T>(to, e1, b);
            continue;
        }
        store_half<T>(x[u], 0, to + e0);
        if (two) store_half<T>(x[u], 1, to + e1);
    }
}

// (800 tokens of 16 heads of 80, fp32: 5.4 us one by one, 6.3 in pairs; 4096 tokens of 48 heads of 128, bf16: 21.3 us one by one,
// 20.5 in pairs, 21.0 and 23.7 by four and eight: a copy of the same bytes takes 16)
constexpr int APPEND_TOKENS = 2;
template <typename T, bool Q4> static const void *append_kernel(bool many) {
    return many ? reinterpret_cast<const void *>(kv_append_kernel<T, APPEND_TOKENS, Q4>) : reinterpret_cast<const void *>(kv_append_kernel<T, 1, Q4>);
}

static griffin_status launch(AppendParams &p, const griffin_attn_desc *desc, const griffin_rope *rope, bool q4, cudaStream_t stream) {
    p.hq = desc->n_q_heads; p.hkv = desc->n_kv_heads; p.d = desc->head_dim;
    if (rope != nullptr) {
        p.table = rope->table; p.rot = rope->rot_dim; p.n_pos = rope->n_pos; p.style = rope->style;
    }
    // several tokens per CTA once there are enough for all SMs
    const int sms = device_sm_count(), n = p.place.n_tokens;
    if (sms <= 0) return GRIFFIN_ERR_CUDA;
    const bool many = n >= 16 * sms;
    const int per_round = APPEND_THREADS / ((p.d + 15) / 16), tpc = many ? APPEND_TOKENS : 1;
    const int x = (n + tpc - 1) / tpc, y = ((p.q != nullptr ? p.hq : 0) + 2 * p.hkv + per_round - 1) / per_round;
    const void *fn = desc->dtype == GRIFFIN_DT_F32 ? (q4 ? append_kernel<float, true>(many) : append_kernel<float, false>(many))
                                                   : (q4 ? append_kernel<__nv_bfloat16, true>(many) : append_kernel<__nv_bfloat16, false>(many));
    void *args[] = {&p};
    return launch_maybe_overlapped(fn, dim3(x, y), dim3(APPEND_THREADS), 0, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

griffin_status launch_kv_append(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                const griffin_kv_cache *cache, const griffin_rope *rope, const void *q, int64_t ld_q,
                                const void *k, int64_t ld_k, const void *v, int64_t ld_v, void *q_out, int64_t ld_q_out,
                                void *ws, cudaStream_t stream) {
    AppendParams p{};
    p.place = place_params(desc, batch, cache->n_pages, ws);
    p.q = q; p.k = k; p.v = v; p.q_out = q_out; p.k_cache = cache->k; p.v_cache = cache->v;
    p.ld_q = ld_q; p.ld_k = ld_k; p.ld_v = ld_v; p.ld_q_out = ld_q_out;
    p.stride_page = cache->stride_page; p.stride_head = cache->stride_head; p.stride_token = cache->stride_token;
    return launch(p, desc, rope, false, stream);
}

griffin_status launch_kv_append_q4(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                   const griffin_kv_cache_q4 *cache, const griffin_rope *rope, const void *q, int64_t ld_q,
                                   const void *k, int64_t ld_k, const void *v, int64_t ld_v, void *q_out, int64_t ld_q_out,
                                   void *ws, cudaStream_t stream) {
    AppendParams p{};
    p.place = place_params(desc, batch, cache->n_pages, ws);
    p.q = q; p.k = k; p.v = v; p.q_out = q_out; p.k_cache = cache->k; p.v_cache = cache->v;
    p.ld_q = ld_q; p.ld_k = ld_k; p.ld_v = ld_v; p.ld_q_out = ld_q_out;
    p.stride_page = cache->stride_page; p.stride_head = cache->stride_head;
    p.q4 = q4_layout(desc->head_dim, desc->page_size);
    return launch(p, desc, rope, true, stream);
}

}  // namespace griffin
