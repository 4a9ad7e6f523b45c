// Joins the partials of rows whose keys were worked on in more than one place: with M = max m_i,
//   out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i,
// the partials in the order of their keys (prefix, then own).  Rows that the attention kernel finished itself are
// left alone; rows that see nothing get zeros.
#include "attn_join.cuh"
#include "layer.h"

namespace griffin {

constexpr int JOIN_THREADS = 128;

// The partials of one job: n segments on CTAs c0, c0 + 1, ..., `streams` of each.
struct JobParts {
    AttnJob job;
    int c0, streams, n;
};
static __device__ __noinline__ JobParts job_parts(const AttnPlan &p, const AttnJob &j, long long W) {
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

template <typename T> __device__ __forceinline__ void store_row4(T *to, const float (&f)[4]) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(to) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        const __nv_bfloat162 x = __floats2bfloat162_rn(f[0], f[1]), y = __floats2bfloat162_rn(f[2], f[3]);
        *reinterpret_cast<uint2 *>(to) = make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
    }
}

struct JoinShared {
    float ml[4][2];
    float o[4][256];
};

// Rows r0 .. r1 of one job.  `wpr` warps share a row (4, 2 or 1: more when there are fewer rows), each taking a
// stretch of its partials; their sums are added in order through shared memory.
template <typename T>
__device__ __noinline__ void join_rows(const AttnPlan &p, const JobParts &a, long long W, int r0, int r1, T *out, long long ld_out,
                                          JoinShared &sh) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int wpr = r1 - r0 >= 3 ? 1 : r1 - r0 == 2 ? 2 : 4, sub = warp % wpr;
    for (int rb = r0; rb < r1; rb += 4 / wpr) {
        const int r = rb + warp / wpr;
        const bool on = r < r1;
        float M = -INFINITY, sum = 0.f, acc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        const int rt = attn_row_token(p, r), tok = a.job.tok0 + rt, head = a.job.head * p.group + r - rt * p.group;
        if (on) {
            JobParts pre = a;
            int rp = 0;
            pre.n = 0;
            if (p.prefix_blocks > 0) {
                const int bp = tok / p.block_tokens;
                pre = job_parts(p, attn_prefix_job(p, a.job.head, bp), W);
                rp = (tok - bp * p.block_tokens) * p.group + r - rt * p.group;
            }
            const int n = pre.n + a.n, per = (n + wpr - 1) / wpr, i0 = sub * per, i1 = min(n, i0 + per);
            for (int ib = i0; ib < i1; ib += 32) {   // a lane per partial for m, l and the place of the outputs
                const int i = ib + lane;
                PartPlace at{nullptr, nullptr};
                float2 ml = make_float2(-INFINITY, 0.f);
                if (i < i1) {
                    at = i < pre.n ? part_place(p, pre, i, rp) : part_place(p, a, i - pre.n, r);
                    ml = *reinterpret_cast<const float2 *>(at.ml);
                }
                float mb = ml.x;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, o));
                const float m_new = fmaxf(M, mb), f = m_new == -INFINITY ? 0.f : exp2f(M - m_new);
                const float wgt = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m_new);
                M = m_new;
                sum *= f;
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k >> 2][k & 3] *= f;
                const int cnt = min(32, i1 - ib);
#pragma unroll 4
                for (int q = 0; q < cnt; ++q) {
                    const float w = __shfl_sync(0xffffffffu, wgt, q), l = __shfl_sync(0xffffffffu, ml.y, q);
                    const float *src = reinterpret_cast<const float *>(
                        __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(at.o), q));
                    if (w == 0.f) continue;   // a part in which the row sees nothing leaves no output
                    sum = fmaf(w, l, sum);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int e = (k * 32 + lane) * 4;
                        if (e >= p.d) continue;
                        const float4 o = __ldcg(reinterpret_cast<const float4 *>(src + e));
                        acc[k][0] = fmaf(w, o.x, acc[k][0]);
                        acc[k][1] = fmaf(w, o.y, acc[k][1]);
                        acc[k][2] = fmaf(w, o.z, acc[k][2]);
                        acc[k][3] = fmaf(w, o.w, acc[k][3]);
                    }
                }
            }
        }
        if (wpr > 1) {
            if (lane == 0) {
                sh.ml[warp][0] = M;
                sh.ml[warp][1] = sum;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int c = 0; c < 4; ++c) sh.o[warp][(k * 32 + lane) * 4 + c] = acc[k][c];
            __syncthreads();
            if (sub == 0 && on) {
                float m_all = M;
                for (int s = 1; s < wpr; ++s) m_all = fmaxf(m_all, sh.ml[warp + s][0]);
                float f = m_all == -INFINITY ? 0.f : exp2f(M - m_all);
                sum *= f;
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k >> 2][k & 3] *= f;
                for (int s = 1; s < wpr; ++s) {
                    f = m_all == -INFINITY ? 0.f : exp2f(sh.ml[warp + s][0] - m_all);
                    sum = fmaf(f, sh.ml[warp + s][1], sum);
#pragma unroll
                    for (int k = 0; k < 8; ++k) acc[k >> 2][k & 3] = fmaf(f, sh.o[warp + s][((k >> 2) * 32 + lane) * 4 + (k & 3)], acc[k >> 2][k & 3]);
                }
                M = m_all;
            }
            __syncthreads();
        }
        if (on && sub == 0) {
            const float inv = M == -INFINITY ? 0.f : 1.0f / sum;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int e = (k * 32 + lane) * 4;
                if (e >= p.d) continue;
                const float f[4] = {acc[k][0] * inv, acc[k][1] * inv, acc[k][2] * inv, acc[k][3] * inv};
                store_row4<T>(out + tok * ld_out + head * p.d + e, f);
            }
        }
    }
}

constexpr int JOIN_ROWS = 16;  // rows of a cut block that one CTA joins

// CTAs 0 .. by_row: jobs whose partials are kept by row: in a fused call the last row block of each sequence and key
// head (no other has just one row tile), else every row block.  The others (fused calls): the jobs that are
// cut at a CTA's first tile, JOIN_ROWS rows each.
template <typename T>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(const __grid_constant__ AttnPlan p, T *__restrict__ out,
                                                                 long long ld_out, int by_row) {
    __shared__ JoinShared sh;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    const long long W = p.bases[p.n_seq];
    const int G = attn_ctas(W, p.grid);
    if ((int)blockIdx.x >= by_row) {
        const int chunks = p.cta_rows / JOIN_ROWS, c = (blockIdx.x - by_row) / chunks, r0 = (blockIdx.x - by_row) % chunks * JOIN_ROWS;
        if (c >= G) return;
        const long long g = attn_share(W, G, c);
        const AttnJob j = attn_find(p, p.bases, g);
        // (the CTA with the job's last tile: every cut job is met once)
        if (g == j.g0 || attn_first_by_row(p, j) || attn_share(W, G, c + 1) < j.g1 || r0 >= j.rows) return;
        join_rows<T>(p, job_parts(p, j, W), W, r0, min(j.rows, r0 + JOIN_ROWS), out, ld_out, sh);
        return;
    }
    const int head = blockIdx.x % p.hkv, bx = blockIdx.x / p.hkv;
    if (p.fused) {
        const AttnSeq q = attn_seq(p, bx);
        const int n_blocks = ceil_div(q.nq, p.block_tokens);
        const long long per_head = attn_div(p.bases[bx + 1] - p.bases[bx], p.hkv), g1 = p.bases[bx] + (head + 1) * per_head;
        for (int b = 0; b < n_blocks && attn_block_tiles(p, q, b) == 0; ++b) {  // rows that see nothing
            const AttnJob j = attn_own_job(p, q, bx, head, b, g1);
            join_rows<T>(p, job_parts(p, j, W), W, 0, j.rows, out, ld_out, sh);
        }
        if (n_blocks == 0) return;
        const int n = attn_block_tiles(p, q, n_blocks - 1);
        const AttnJob j = attn_own_job(p, q, bx, head, n_blocks - 1, g1 - n);
        if (n > 0 && j.alt) join_rows<T>(p, job_parts(p, j, W), W, 0, j.rows, out, ld_out, sh);
        return;
    }
    // Sequence s owns the block numbers from q_start[s] / block_tokens + s on: at least as many as it has blocks.
    int seq = -1;
    for (int s0 = 0; s0 < p.n_seq; s0 += JOIN_THREADS) {
        const int s = s0 + threadIdx.x;
        seq += __syncthreads_count(s < p.n_seq && __ldg(p.q_start + s) / p.block_tokens + s <= bx);
    }
    if (seq < 0) return;
    const AttnSeq q = attn_seq(p, seq);
    const int b = bx - (__ldg(p.q_start + seq) / p.block_tokens + seq);
    if (b * p.block_tokens >= q.nq) return;
    long long g0 = p.bases[seq] + head * attn_div(p.bases[seq + 1] - p.bases[seq], p.hkv);
    for (int k = 0; k < b; ++k) g0 += attn_block_tiles(p, q, k);
    const AttnJob j = attn_own_job(p, q, seq, head, b, g0);
    join_rows<T>(p, job_parts(p, j, W), W, 0, j.rows, out, ld_out, sh);
}

griffin_status launch_attn_join(const AttnPlan &plan, int dtype, void *out, long long ld_out, cudaStream_t stream) {
    AttnPlan p = plan;
    int by_row = p.hkv * (p.fused ? p.n_seq : p.n_seq + p.n_tokens / p.block_tokens);
    const int cut = p.fused ? p.grid * (p.cta_rows / JOIN_ROWS) : 0;
    const void *fn = dtype == GRIFFIN_DT_F32 ? reinterpret_cast<const void *>(attn_join_kernel<float>)
                                             : reinterpret_cast<const void *>(attn_join_kernel<__nv_bfloat16>);
    void *args[] = {&p, &out, &ld_out, &by_row};
    return launch_maybe_overlapped(fn, dim3(by_row + cut), dim3(JOIN_THREADS), 0, stream, true, args) == cudaSuccess ? GRIFFIN_OK
                                                                                                                     : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
