// Tokens of the cache held in 4 bits (q4.cuh) back to the storage type: out = (code - 8) s, which rounds nothing.
//
// A thread has one group of 16 entries of one key or value, of TPC tokens: 9 bytes in, 32 (bf16) or 64 out.  Bound by the
// bytes that are written.
#include "common.cuh"
#include "kv_place.cuh"
#include "layer.h"
#include "q4.cuh"
#include "vec8.cuh"

namespace griffin {

struct ReadParams {
    PlaceParams place;
    const uint8_t *k, *v;
    void *k_out, *v_out;
    long long ld_k, ld_v, stride_page, stride_head;
    Q4Layout q4;
    int units, groups, hkv;   // units: groups of a token's keys and values; groups: of a head
};

constexpr int READ_THREADS = 128;

template <typename T, int TPC> __global__ void __launch_bounds__(READ_THREADS) kv_read_q4_kernel(const __grid_constant__ ReadParams p) {
    __shared__ Place s_at[TPC];
    const int t0 = blockIdx.x * TPC, unit = blockIdx.y * READ_THREADS + threadIdx.x;
    const int h = unit / p.groups, g = unit - h * p.groups;
    const bool is_v = h >= p.hkv;
    const int head = is_v ? h - p.hkv : h;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    const Place mine = place_token<TPC, READ_THREADS>(p.place, t0, -1);
    if (TPC > 1) {
        if (threadIdx.x < TPC) s_at[threadIdx.x] = mine;
        __syncthreads();
    }
    if (unit >= p.units) return;
    uint2 w[TPC];
    uint32_t b[TPC];
#pragma unroll
    for (int u = 0; u < TPC; ++u) {
        const Place at = TPC > 1 ? s_at[u] : mine;
        w[u] = make_uint2(Q4_ZEROS, Q4_ZEROS);
        b[u] = 0;
        if (at.page < 0) continue;   // (padding, or a token that has no place, reads as zeros)
        const uint8_t *const block = (is_v ? p.v : p.k) + at.page * p.stride_page + head * p.stride_head;
        w[u] = __ldg(reinterpret_cast<const uint2 *>(block + at.slot * p.q4.code_row + g * 8));
        b[u] = __ldg(block + p.q4.scale_off + at.slot * p.q4.scale_row + g);
    }
    T *const out = static_cast<T *>(is_v ? p.v_out : p.k_out) + (long long)(head * p.groups + g) * 16;
    const long long ld = is_v ? p.ld_v : p.ld_k;
#pragma unroll
    for (int u = 0; u < TPC; ++u) {
        if ((TPC > 1 ? s_at[u] : mine).page == -2) continue;
        const float s = q4_scale(b[u]);
        float f[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = q4_value(i ? w[u].y : w[u].x, j, s);
            store8<T>(out, (t0 + u) * ld + 8 * i, f);
        }
    }
}

constexpr int READ_TOKENS = 4;
template <typename T> static const void *read_kernel(bool many) {
    return many ? reinterpret_cast<const void *>(kv_read_q4_kernel<T, READ_TOKENS>) : reinterpret_cast<const void *>(kv_read_q4_kernel<T, 1>);
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
    const bool many = n >= 16 * sms;
    const int tpc = many ? READ_TOKENS : 1, x = (n + tpc - 1) / tpc, y = (p.units + READ_THREADS - 1) / READ_THREADS;
    const void *fn = desc->dtype == GRIFFIN_DT_F32 ? read_kernel<float>(many) : read_kernel<__nv_bfloat16>(many);
    void *args[] = {&p};
    return launch_maybe_overlapped(fn, dim3(x, y), dim3(READ_THREADS), 0, stream, true, args) == cudaSuccess ? GRIFFIN_OK
                                                                                                            : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
