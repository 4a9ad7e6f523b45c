// Joins the partials of rows whose keys were worked on in more than one place: with M = max m_i,
//   out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i,
// the partials in the order of their keys (prefix, then own).  One CTA per row block and key head, one warp
// per row; rows that the attention kernel finished itself are left alone.  Rows that see nothing get zeros.
#include "attn_join.cuh"
#include "layer.h"

namespace griffin {

constexpr int JOIN_THREADS = 128;

// The partials of one job: n segments on CTAs c0, c0 + 1, ..., `streams` of each.
struct JobParts {
    AttnJob job;
    int c0, streams, n;
};
__device__ __forceinline__ JobParts job_parts(const AttnPlan &p, const AttnJob &j, long long W) {
    JobParts r;
    r.job = j;
    r.streams = j.alt ? 2 : 1;
    r.c0 = 0;
    r.n = 0;
    if (j.g1 > j.g0) {
        const int G = attn_ctas(W, p.grid);
        r.c0 = attn_cta_of(W, G, j.g0);
        r.n = (attn_cta_of(W, G, j.g1 - 1) - r.c0 + 1) * r.streams;
    }
    return r;
}
__device__ __forceinline__ PartPlace part_place(const AttnPlan &p, const JobParts &a, int i, int r) {
    const int stream = a.streams == 2 ? i & 1 : 0, c = a.c0 + (a.streams == 2 ? i >> 1 : i);
    if (c == a.c0) return attn_first_by_row(p, a.job) ? attn_place_row(p, a.job, stream, r) : attn_place_cta(p, c, 1, r);
    return attn_place_cta(p, c, 0, a.job.alt ? stream * (p.cta_rows >> 1) + r : r);
}

template <typename T>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(const __grid_constant__ AttnPlan p, T *__restrict__ out,
                                                                 long long ld_out) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, head = blockIdx.y;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    // Sequence s owns the block numbers from q_start[s] / block_tokens + s on: at least as many as it has blocks.
    int seq = -1;
    for (int s0 = 0; s0 < p.n_seq; s0 += JOIN_THREADS) {
        const int s = s0 + threadIdx.x;
        seq += __syncthreads_count(s < p.n_seq && __ldg(p.q_start + s) / p.block_tokens + s <= (int)blockIdx.x);
    }
    if (seq < 0) return;
    const AttnSeq q = attn_seq(p, seq);
    const int b = blockIdx.x - (__ldg(p.q_start + seq) / p.block_tokens + seq);
    if (b * p.block_tokens >= q.nq) return;
    const long long W = p.bases[p.n_seq];
    const long long base = p.bases[seq], per_head = (p.bases[seq + 1] - base) / p.hkv;
    long long g0 = base + head * per_head;
    for (int k = 0; k < b; ++k) g0 += attn_block_tiles(p, q, k);
    const AttnJob own = attn_own_job(p, q, seq, head, b, g0);
    const JobParts a = job_parts(p, own, W);
    if (a.n == 1 && attn_direct(p, own, true)) return;

    for (int r = warp; r < own.rows; r += JOIN_THREADS / 32) {
        const int tok = own.tok0 + r / p.group, hq = head * p.group + r % p.group;
        JobParts pre = a;
        int rp = 0;
        pre.n = 0;
        if (p.prefix_blocks > 0) {
            const int bp = tok / p.block_tokens;
            pre = job_parts(p, attn_prefix_job(p, head, bp), W);
            rp = (tok - bp * p.block_tokens) * p.group + r % p.group;
        }
        const int n = pre.n + a.n;
        float M = -INFINITY;
        for (int i = lane; i < n; i += 32) {
            const PartPlace at = i < pre.n ? part_place(p, pre, i, rp) : part_place(p, a, i - pre.n, r);
            M = fmaxf(M, at.ml[0]);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        float sum = 0.f, acc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        for (int i = 0; i < n; ++i) {
            const PartPlace at = i < pre.n ? part_place(p, pre, i, rp) : part_place(p, a, i - pre.n, r);
            const float2 ml = *reinterpret_cast<const float2 *>(at.ml);
            if (ml.x == -INFINITY) continue;  // a part in which the row sees nothing leaves no output
            const float w = exp2f(ml.x - M);
            sum = fmaf(w, ml.y, sum);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int e = (k * 32 + lane) * 4;
                if (e >= p.d) continue;
                const float4 o = *reinterpret_cast<const float4 *>(at.o + e);
                acc[k][0] = fmaf(w, o.x, acc[k][0]);
                acc[k][1] = fmaf(w, o.y, acc[k][1]);
                acc[k][2] = fmaf(w, o.z, acc[k][2]);
                acc[k][3] = fmaf(w, o.w, acc[k][3]);
            }
        }
        const float inv = M == -INFINITY ? 0.f : 1.0f / sum;
        T *const to = out + tok * ld_out + hq * p.d;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int e = (k * 32 + lane) * 4;
            if (e >= p.d) continue;
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<float4 *>(to + e) = make_float4(acc[k][0] * inv, acc[k][1] * inv, acc[k][2] * inv, acc[k][3] * inv);
            } else {
                const __nv_bfloat162 x = __floats2bfloat162_rn(acc[k][0] * inv, acc[k][1] * inv);
                const __nv_bfloat162 y = __floats2bfloat162_rn(acc[k][2] * inv, acc[k][3] * inv);
                *reinterpret_cast<uint2 *>(to + e) =
                    make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
            }
        }
    }
}

griffin_status launch_attn_join(const AttnPlan &plan, int dtype, void *out, long long ld_out, cudaStream_t stream) {
    AttnPlan p = plan;
    const void *fn = dtype == GRIFFIN_DT_F32 ? reinterpret_cast<const void *>(attn_join_kernel<float>)
                                             : reinterpret_cast<const void *>(attn_join_kernel<__nv_bfloat16>);
    void *args[] = {&p, &out, &ld_out};
    const dim3 grid(p.n_seq + p.n_tokens / p.block_tokens, p.hkv);
    return launch_maybe_overlapped(fn, grid, dim3(JOIN_THREADS), 0, stream, true, args) == cudaSuccess ? GRIFFIN_OK
                                                                                                       : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
