// Attention over the shared prefix and each sequence's own keys, fp32 storage, on the plain fp32 pipes:
//   S = scale Q K^T, masked by place;  m' = max(m, max S);  P = 2^(S - m');
//   l = l 2^(m - m') + sum P;  O = O 2^(m - m') + P V        (S in units of log2, all fp32)
// one CTA of 256 threads per SM, each with its share of the call's key tiles (attn_plan.cuh).  Keys and
// values behind what any row of the block sees are read as zeros, whatever the cache holds there.
#include "attn.h"
#include "attn_join.cuh"
#include "vec8.cuh"

namespace griffin {

constexpr int SIMT_ROWS = 64, SIMT_KT = 32, SIMT_THREADS = 256;

template <int DP> constexpr size_t simt_smem(int n_seq) {
    return (size_t)(SIMT_ROWS + 2 * SIMT_KT) * (DP + 4) * 4 + SIMT_ROWS * (SIMT_KT + 1) * 4 + 3 * SIMT_ROWS * 4 +
           ((size_t)n_seq + 3) * 4;
}

// DP: the head's width rounded up to 64, 128 or 256; entries from D on are zeros in shared memory.
template <int DP>
__global__ void __launch_bounds__(SIMT_THREADS) attn_simt_kernel(const __grid_constant__ AttnPlan p,
                                                                 const __grid_constant__ AttnData x) {
    constexpr int LD = DP + 4, NE = DP / 64;  // NE: groups of 4 outputs of a thread, 64 apart
    extern __shared__ __align__(16) uint8_t smem_raw[];
    float *const sq = reinterpret_cast<float *>(smem_raw), *const sk = sq + SIMT_ROWS * LD, *const sv = sk + SIMT_KT * LD;
    float *const ss = sv + SIMT_KT * LD, *const sm = ss + SIMT_ROWS * (SIMT_KT + 1), *const sl = sm + SIMT_ROWS, *const sf = sl + SIMT_ROWS;
    int *const bases = reinterpret_cast<int *>(sf + SIMT_ROWS);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;

    pdl_launch_dependents();
    pdl_wait_prior_grids();
    attn_scan(p, bases);
    const AttnShares shares(bases[p.n_seq], p.grid);
    if ((int)blockIdx.x >= shares.G) return;
    int g = shares.first(blockIdx.x);
    const int g_end = shares.first(blockIdx.x + 1);
    AttnJob j = attn_find(p, bases, g);
    if (tid == 0) attn_note_cut(p, shares, j, g, min(g_end, j.g1));
    for (;;) {
        const int stop = min(g_end, j.g1);
        const bool first = g == j.g0, whole = first && stop == j.g1;
        const int pre_tiles = j.seq < 0 || p.fused ? p.prefix_tiles : 0;
        __syncthreads();  // the segment before is done with shared memory
        for (int i = tid; i < SIMT_ROWS * (DP / 8); i += SIMT_THREADS) {
            const int r = i / (DP / 8), e = i % (DP / 8) * 8;
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (r < j.rows && e < p.d)
                load8<float>(x.q, (j.tok0 + attn_row_token(p, r)) * x.ld_q + (j.head * p.group + r - attn_row_token(p, r) * p.group) * p.d + e, f);
            store8<float>(sq, r * LD + e, f);
        }
        if (tid < SIMT_ROWS) {
            sm[tid] = -INFINITY;
            sl[tid] = 0.f;
        }
        float o[4][NE][4];
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int b = 0; b < NE; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[a][b][c] = 0.f;

        for (; g < stop; ++g) {
            const int t = g - j.g0;
            const bool in_prefix = t < pre_tiles;
            const int k0 = (in_prefix ? t : t - pre_tiles) * SIMT_KT;       // first key of the tile
            const int len = in_prefix ? p.prefix_len : j.own_len;          // keys behind this are not there
            const int *const pages = in_prefix ? p.prefix_pages : p.page_table + (long long)j.seq * p.table_stride;
            __syncthreads();  // the tile before is done with
            for (int i = tid; i < SIMT_KT * (DP / 8); i += SIMT_THREADS) {
                const int r = i / (DP / 8), e = i % (DP / 8) * 8, key = k0 + r;
                float fk[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, fv[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (key < len && e < p.d) {
                    const int page = __ldg(pages + (key >> p.page_shift));
                    if (page >= 0 && page < p.n_pages) {
                        const long long at = page * x.stride_page + j.head * x.stride_head +
                                             (key & ((1 << p.page_shift) - 1)) * x.stride_token + e;
                        load8<float>(x.k, at, fk);
                        load8<float>(x.v, at, fv);
                    } else {
                        raise_status(p.ws, DEV_STATUS_BAD_INDEX, 42);
                    }
                }
                store8<float>(sk, r * LD + e, fk);
                store8<float>(sv, r * LD + e, fv);
            }
            __syncthreads();
            // S: rows 4 ty .., keys tx and tx + 16
            float s[4][2] = {};
#pragma unroll 4
            for (int e = 0; e < DP; e += 4) {
                const float4 b0 = *reinterpret_cast<const float4 *>(sk + tx * LD + e);
                const float4 b1 = *reinterpret_cast<const float4 *>(sk + (tx + 16) * LD + e);
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const float4 q = *reinterpret_cast<const float4 *>(sq + (ty * 4 + a) * LD + e);
                    s[a][0] = fmaf(q.x, b0.x, fmaf(q.y, b0.y, fmaf(q.z, b0.z, fmaf(q.w, b0.w, s[a][0]))));
                    s[a][1] = fmaf(q.x, b1.x, fmaf(q.y, b1.y, fmaf(q.z, b1.z, fmaf(q.w, b1.w, s[a][1]))));
                }
            }
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const int r = ty * 4 + a, seen = in_prefix ? len : min(len, j.seen0 + attn_row_token(p, r));
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    ss[r * (SIMT_KT + 1) + tx + 16 * b] = k0 + tx + 16 * b < seen ? s[a][b] * p.scale_log2 : -INFINITY;
            }
            __syncthreads();
            {   // running maximum and sum: four neighbouring threads per row
                const int r = tid >> 2, c0 = (tid & 3) * (SIMT_KT / 4);
                float *const row = ss + r * (SIMT_KT + 1) + c0;
                float mx = row[0];
#pragma unroll
                for (int c = 1; c < SIMT_KT / 4; ++c) mx = fmaxf(mx, row[c]);
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const float m_old = sm[r], m_new = fmaxf(m_old, mx), base = m_new == -INFINITY ? 0.f : m_new;
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < SIMT_KT / 4; ++c) {
                    const float e = exp2f(row[c] - base);
                    row[c] = e;
                    sum += e;
                }
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                const float f = exp2f(m_old - base);  // 0 while nothing was seen
                if ((tid & 3) == 0) {
                    sm[r] = m_new;
                    sl[r] = sl[r] * f + sum;
                    sf[r] = f;
                }
            }
            __syncthreads();
            // O: rows 4 ty .., entries 4 tx .. and 64 further
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const float f = sf[ty * 4 + a];
#pragma unroll
                for (int b = 0; b < NE; ++b)
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[a][b][c] *= f;
            }
#pragma unroll 4
            for (int k = 0; k < SIMT_KT; ++k) {
                float w[4];
#pragma unroll
                for (int a = 0; a < 4; ++a) w[a] = ss[(ty * 4 + a) * (SIMT_KT + 1) + k];
#pragma unroll
                for (int b = 0; b < NE; ++b) {
                    const float4 v = *reinterpret_cast<const float4 *>(sv + k * LD + b * 64 + tx * 4);
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        o[a][b][0] = fmaf(w[a], v.x, o[a][b][0]);
                        o[a][b][1] = fmaf(w[a], v.y, o[a][b][1]);
                        o[a][b][2] = fmaf(w[a], v.z, o[a][b][2]);
                        o[a][b][3] = fmaf(w[a], v.w, o[a][b][3]);
                    }
                }
            }
        }
        // the segment's result
        const bool direct = attn_direct(p, j, whole);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int r = ty * 4 + a;
            if (r >= j.rows) continue;
            const float m = sm[r], l = sl[r];
            if (direct) {
                const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
                float *const to = static_cast<float *>(x.out) + (j.tok0 + attn_row_token(p, r)) * x.ld_out + (j.head * p.group + r - attn_row_token(p, r) * p.group) * p.d;
#pragma unroll
                for (int b = 0; b < NE; ++b)
                    if (b * 64 + tx * 4 < p.d)
                        *reinterpret_cast<float4 *>(to + b * 64 + tx * 4) =
                            make_float4(o[a][b][0] * inv, o[a][b][1] * inv, o[a][b][2] * inv, o[a][b][3] * inv);
            } else {
                const PartPlace at = attn_place(p, j, first, 0, r);
                if (tx == 0) *reinterpret_cast<float2 *>(at.ml) = make_float2(m, l);
#pragma unroll
                for (int b = 0; b < NE; ++b)
                    if (b * 64 + tx * 4 < p.d)
                        *reinterpret_cast<float4 *>(at.o + b * 64 + tx * 4) = make_float4(o[a][b][0], o[a][b][1], o[a][b][2], o[a][b][3]);
            }
        }
        if (g >= g_end) return;
        j = attn_next(p, bases, j);
    }
}

AttnShape attn_simt_shape() { return {SIMT_ROWS, 1, SIMT_KT, 0}; }

template <int DP> static griffin_status launch_dp(AttnPlan p, AttnData x, cudaStream_t stream) {
    const void *fn = reinterpret_cast<const void *>(attn_simt_kernel<DP>);
    const size_t smem = simt_smem<DP>(p.n_seq);
    if (ensure_dynamic_smem(fn, smem) != cudaSuccess) return GRIFFIN_ERR_CUDA;
    void *args[] = {&p, &x};
    return launch_maybe_overlapped(fn, dim3(p.grid), dim3(SIMT_THREADS), smem, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

griffin_status launch_attn_simt(const AttnPlan &plan, const AttnData &data, cudaStream_t stream) {
    if (plan.d <= 64) return launch_dp<64>(plan, data, stream);
    if (plan.d <= 128) return launch_dp<128>(plan, data, stream);
    return launch_dp<256>(plan, data, stream);
}

}  // namespace griffin
