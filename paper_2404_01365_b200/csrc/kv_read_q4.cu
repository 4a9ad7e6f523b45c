// Tokens of the cache held in 4 bits (q4.cuh) back to the storage type: out = (code - 8) s, which rounds nothing.
//
// A thread has one group of 16 entries of one key or value, of every SUBS-th of the CTA's tokens: 9 bytes in, 32 (bf16) or 64
// out.  A CTA takes its tokens' places together, which is three dependent trips to L2; a call of many tokens is cut into as many
// CTAs as fit at once, all with the same number (16 tokens to each were 1.2 times that many).
// Bound by memory: 22046 tokens of 8 heads, 128 wide (25 MB in, 90 MB out), take 24.1 us to bf16, 4.8 TB/s, of which a copy of the
// same bytes takes 17.7 at the measured rate; 4096 tokens that the append has just written 6.3.
#include "common.cuh"
#include "kv_place.cuh"
#include "layer.h"
#include "q4.cuh"

namespace griffin {

struct ReadParams {
    PlaceParams place;
    const uint8_t *k, *v;
    void *k_out, *v_out;
    long long ld_k, ld_v, stride_page, stride_head;
    Q4Layout q4;
    int units, groups, hkv;   // units: groups of a token's keys and values; groups: of a head
    int per, wide;            // units of a token that a CTA has; whether rows begin on 32-byte boundaries
    int tokens;               // that a CTA has
};

constexpr int READ_THREADS = 128, READ_CTAS = 10;   // of an SM

// 16 entries to a row.
template <typename T> __device__ __forceinline__ void store16(T *to, uint2 w, uint32_t scale, bool wide, uint32_t magic) {
    const uint32_t h = q4_scale_bits(scale);
    const Q4Scale2 s = q4_scale2(h, h);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {   // 32 bytes each
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (sizeof(T) == 2) {
                v[e] = q4_pair(e < 4 ? w.x : w.y, e & 3, s, magic);
            } else {
                const uint32_t two = q4_pair(i ? w.y : w.x, e >> 1, s, magic);   // (exact in bf16)
                v[e] = e & 1 ? two & 0xffff0000u : two << 16;
            }
        }
        uint32_t *const at = reinterpret_cast<uint32_t *>(to) + 8 * i;
        if (wide) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                         "r"(v[5]), "r"(v[6]), "r"(v[7])
                         : "memory");
        } else {
            reinterpret_cast<uint4 *>(at)[0] = make_uint4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<uint4 *>(at)[1] = make_uint4(v[4], v[5], v[6], v[7]);
        }
    }
}

template <typename T, int TPC>
__global__ void __launch_bounds__(READ_THREADS, READ_CTAS) kv_read_q4_kernel(const __grid_constant__ ReadParams p) {
    __shared__ Place s_at[TPC];
    const int tokens = TPC == 1 ? 1 : p.tokens, t0 = blockIdx.x * tokens;
    const int sub = threadIdx.x / p.per, subs = READ_THREADS / p.per, unit = blockIdx.y * p.per + threadIdx.x - sub * p.per;
    const int h = unit / p.groups, g = unit - h * p.groups;
    const bool is_v = h >= p.hkv;
    const int head = is_v ? h - p.hkv : h;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    const Place mine = place_token<TPC, READ_THREADS>(p.place, t0, -1, tokens);
    if (threadIdx.x < TPC) s_at[threadIdx.x] = mine;
    __syncthreads();
    if (unit >= p.units || sub >= subs) return;
    const uint8_t *const block = (is_v ? p.v : p.k) + head * p.stride_head;
    const long long ld = is_v ? p.ld_v : p.ld_k;
    T *const out = static_cast<T *>(is_v ? p.v_out : p.k_out) + (long long)(head * p.groups + g) * 16;
    constexpr int AT_ONCE = TPC < 4 ? TPC : 4;
#pragma unroll 1
    for (int t = sub; t < tokens; t += AT_ONCE * subs) {
        uint2 w[AT_ONCE];
        uint32_t b[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            w[u] = make_uint2(Q4_ZEROS, Q4_ZEROS);
            b[u] = 0;
            if (t + u * subs >= tokens) continue;
            const Place at = s_at[t + u * subs];
            if (at.page < 0) continue;   // (padding, or a token that has no place, reads as zeros)
            const uint8_t *const from = block + at.page * p.stride_page;
            // (coherent loads: the call in front may have written them while this grid was waiting)
            w[u] = *reinterpret_cast<const uint2 *>(from + at.slot * p.q4.code_row + g * 8);
            b[u] = from[p.q4.scale_off + at.slot * p.q4.scale_row + g];
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (t + u * subs >= tokens || s_at[t + u * subs].page == -2) continue;
            store16<T>(out + (t0 + t + u * subs) * ld, w[u], b[u], p.wide != 0, p.q4.magic);
        }
    }
}

template <typename T> static const void *read_kernel(bool many) {
    return many ? reinterpret_cast<const void *>(kv_read_q4_kernel<T, READ_THREADS>) : reinterpret_cast<const void *>(kv_read_q4_kernel<T, 1>);
}

griffin_status launch_kv_read_q4(const griffin_attn_desc *desc, const griffin_attn_batch *batch, const griffin_kv_cache_q4 *cache,
                                 void *k, int64_t ld_k, void *v, int64_t ld_v, void *ws, cudaStream_t stream) {
    ReadParams p{};
    p.place = place_params(desc, batch, cache->n_pages, ws);
    p.k = static_cast<const uint8_t *>(cache->k); p.v = static_cast<const uint8_t *>(cache->v);
    p.k_out = k; p.v_out = v; p.ld_k = ld_k; p.ld_v = ld_v;
    p.stride_page = cache->stride_page; p.stride_head = cache->stride_head;
    p.q4 = q4_layout(desc->head_dim, desc->page_size);
    p.groups = desc->head_dim / 16; p.hkv = desc->n_kv_heads; p.units = 2 * p.hkv * p.groups;
    const int sms = device_sm_count(), n = batch->n_tokens;
    if (sms <= 0) return GRIFFIN_ERR_CUDA;
    p.per = p.units < READ_THREADS ? p.units : READ_THREADS;
    const int unit = desc->dtype == GRIFFIN_DT_F32 ? 4 : 2;
    p.wide = ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | (uintptr_t)(ld_k * unit) | (uintptr_t)(ld_v * unit)) & 31) == 0;
    const int y = (p.units + p.per - 1) / p.per;
    // a token to a CTA while they are few; else every CTA as many as the other, 4 to 32
    const int most = READ_CTAS * sms / y > 0 ? READ_CTAS * sms / y : 1;
    const bool many = n > 2 * most;
    p.tokens = many ? (n + most - 1) / most : 1;
    p.tokens = !many ? 1 : p.tokens < 4 ? 4 : p.tokens > 32 ? 32 : p.tokens;
    const int x = (n + p.tokens - 1) / p.tokens;
    const void *fn = desc->dtype == GRIFFIN_DT_F32 ? read_kernel<float>(many) : read_kernel<__nv_bfloat16>(many);
    void *args[] = {&p};
    return launch_maybe_overlapped(fn, dim3(x, y), dim3(READ_THREADS), 0, stream, true, args) == cudaSuccess ? GRIFFIN_OK
                                                                                                            : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
