// Joins the partials of rows whose keys were worked on in more than one place: with M = max m_i,
//   out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i,
// the partials in the order of their keys (prefix, then own).  Rows that the attention kernel finished itself are
// left alone; rows that see nothing get zeros.  Bound by latency: the list of a row's partials, their m and l,
// their outputs are three dependent trips to L2; 32 partials travel in one of each.
// Measured: 5 to 9 us of a call (one sequence of 32 heads 5, 8 sequences of 40 heads 6, 32 sequences of 8 key heads 9), of
// which 3.6 are the launch behind the other kernel.
#include "attn_join.cuh"
#include "layer.h"

namespace griffin {

constexpr int JOIN_THREADS = 256, JOIN_WARPS = JOIN_THREADS / 32;
constexpr int JOIN_ROWS = 16;  // rows of a cut block that one CTA joins

// The partials of one job: n of them on CTAs c0, c0 + 1, ..., `streams` of each.
struct JobParts {
    PartJob job;
    int c0, streams, n;
};
__device__ __forceinline__ JobParts job_parts(const AttnPlan &p, const AttnShares &sh, const AttnJob &j) {
    JobParts r{j, 0, j.alt ? 2 : 1, 0};
    if (j.g1 > j.g0) {
        r.c0 = sh.cta_of(j.g0);
        r.n = (sh.cta_of(j.g1 - 1) - r.c0 + 1) * r.streams;
    }
    return r;
}
__device__ __forceinline__ PartPlace part_place(const AttnPlan &p, const JobParts &a, int i, int r) {
    const int stream = a.streams == 2 ? i & 1 : 0, c = a.c0 + (a.streams == 2 ? i >> 1 : i);
    if (c == a.c0 && attn_first_by_row(p, a.job)) return attn_place_row(p, a.job, stream, r);
    return attn_place_cta(p, c, c == a.c0 ? 1 : 0, a.streams == 2 ? stream * (p.cta_rows >> 1) + r : r);
}

template <typename T> __device__ __forceinline__ void store_row4(T *to, const float (&f)[4]) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(to) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        const __nv_bfloat162 x = __floats2bfloat162_rn(f[0], f[1]), y = __floats2bfloat162_rn(f[2], f[3]);
        *reinterpret_cast<uint2 *>(to) = make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
    }
}

// CTAs 0 .. by_row * split - 1, `split` of them to a job: jobs whose partials are kept by row: in a fused call the last row block of each sequence and
// key head (no other has just one row tile) and the blocks that see nothing, else every row block.  The others
// (fused calls): the blocks that were cut, JOIN_ROWS rows each.
// NV: 128-entry pieces of a row (a lane has 4 entries of each).
template <typename T, int NV>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(const __grid_constant__ AttnPlan p, T *__restrict__ out,
                                                                 long long ld_out, int by_row, int split) {
    __shared__ float sh_ml[JOIN_WARPS][2], sh_o[JOIN_WARPS][NV * 128];
    __shared__ int sh_seq[5];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    const AttnTotals tot = attn_totals(p, p.bases);
    if (tot.W < 0) return;   // the call was not run, and the first tiles of its sequences mean nothing
    if (tot.queued && blockIdx.x == 0 && threadIdx.x == 0) *p.queue = 0;
    const AttnShares sh(tot.W, p.grid);
    JobParts a;
    AttnSeq q{};
    int r0 = 0, r1 = 0, head = 0, seq = 0, n_blocks = 0, b = 0, base0 = 0, base1 = 0;
    bool cut = false;
    const int id = (int)((uint32_t)blockIdx.x / (uint32_t)split), part = blockIdx.x - id * split;
    if (id >= by_row) {
        const int at = blockIdx.x - by_row * split, chunks = p.cta_rows / JOIN_ROWS, c = at / chunks;
        if (c >= sh.G || tot.queued) return;
        const CutJob j = p.cuts[c];
        r0 = at % chunks * JOIN_ROWS;
        r1 = min(j.rows, r0 + JOIN_ROWS);
        if (r0 >= r1) return;
        a = JobParts{PartJob{0, j.head, j.tok0, false}, j.c0, 1, c - j.c0 + 1};
        cut = true;
    } else {
        const int bx = (int)((uint32_t)id / (uint32_t)p.hkv);
        head = id - bx * p.hkv;
        int q_start, q_end, len;
        if (p.fused) {
            seq = bx;
            q_start = __ldg(p.q_start + seq), q_end = __ldg(p.q_start + seq + 1), len = __ldg(p.seq_len + seq);
            base0 = p.bases[seq], base1 = p.bases[seq + 1];
        } else {
            // Sequence s owns the block numbers from q_start[s] / block_tokens + s on: at least as many as it has blocks.
            // (a thread per sequence asks for all that may be wanted of it: one trip to L2, not three)
            seq = -1;
#pragma unroll 1
            for (int s0 = 0; s0 < p.n_seq; s0 += blockDim.x) {
                const int s = s0 + threadIdx.x;
                int v[5] = {};
                if (s < p.n_seq) {
                    v[0] = __ldg(p.q_start + s), v[1] = __ldg(p.q_start + s + 1), v[2] = __ldg(p.seq_len + s);
                    v[3] = p.bases[s], v[4] = p.bases[s + 1];
                }
                const int n = __syncthreads_count(s < p.n_seq && v[0] / p.block_tokens + s <= bx);
                seq += n;
                if ((int)threadIdx.x == n - 1) {
#pragma unroll
                    for (int i = 0; i < 5; ++i) sh_seq[i] = v[i];
                }
            }
            if (seq < 0) return;
            __syncthreads();
            q_start = sh_seq[0], q_end = sh_seq[1], len = sh_seq[2], base0 = sh_seq[3], base1 = sh_seq[4];
            b = bx - (q_start / p.block_tokens + seq);
        }
        q = attn_seq_of(p, q_start, q_end, len);
        n_blocks = ceil_div(q.nq, p.block_tokens);
        if (b < 0 || b >= n_blocks) return;   // (b < 0: q_start does not ascend, which attn_seq_of has reported)
    }
#pragma unroll 1
    for (;;) {
        if (!cut) {
            // this job's place among the tiles: behind those of the heads and blocks before it
            const int per_head = (int)((uint32_t)(base1 - base0) / (uint32_t)p.hkv);
            if (p.fused && attn_block_tiles(p, q, b) > 0) b = n_blocks - 1;
            int g0 = base0 + (head + 1) * per_head;
            g0 -= (int)attn_sum_tiles(p, q, b, n_blocks);
            const AttnJob j = attn_own_job(p, q, seq, head, b, g0);
            a = job_parts(p, sh, j);
            const int per = (j.rows + split - 1) / split;   // this CTA's rows of the job
            r0 = part * per;
            r1 = min(j.rows, r0 + per);
            if (p.fused && j.g1 > j.g0 && (!j.alt || tot.queued)) return;  // finished by the attention kernel, or cut
        }
        // Each row is joined by `wpr` warps (more when there are fewer rows), each taking a stretch of its partials; their
        // sums are added in order through shared memory.
        const int wpr = r1 - r0 == 1 ? warps : r1 - r0 == 2 ? warps / 2 : 2 * (r1 - r0) <= warps ? warps / 4 : 1, sub = warp % wpr;
        constexpr int AT_ONCE = NV == 1 ? 8 : 4;
#pragma unroll 1
        for (int rb = r0; rb < r1; rb += warps / wpr) {
            const int r = rb + warp / wpr;
            const bool on = r < r1;
            const int rt = attn_row_token(p, r), tok = a.job.tok0 + rt, hq = a.job.head * p.group + r - rt * p.group;
            float M = -INFINITY, sum = 0.f, acc[NV][4] = {};
            if (on) {
                JobParts pre = a;
                int rp = 0;
                pre.n = 0;
                if (p.prefix_blocks > 0) {
                    const int bp = tok / p.block_tokens;
                    pre = job_parts(p, sh, attn_prefix_job(p, a.job.head, bp));
                    rp = (tok - bp * p.block_tokens) * p.group + r - rt * p.group;
                }
                const int n = pre.n + a.n, per = (n + wpr - 1) / wpr, i0 = sub * per, i1 = min(n, i0 + per);
#pragma unroll 1
                for (int ib = i0; ib < i1; ib += 32) {  // a lane per partial for m, l and the place of the outputs
                    const int i = ib + lane;
                    PartPlace at{nullptr, nullptr};
                    float2 ml = make_float2(-INFINITY, 0.f);
                    if (i < i1) {
                        const bool of_prefix = i < pre.n;
                        at = part_place(p, of_prefix ? pre : a, of_prefix ? i : i - pre.n, of_prefix ? rp : r);
                        ml = *reinterpret_cast<const float2 *>(at.ml);
                    }
                    float mb = ml.x;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, o));
                    const float m_new = fmaxf(M, mb), f = m_new == -INFINITY ? 0.f : exp2f(M - m_new);
                    // (a part in which the row sees nothing leaves no output)
                    const float wgt = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m_new);
                    if (wgt == 0.f) at.o = nullptr;
                    M = m_new;
                    sum = sum * f + warp_sum(wgt * ml.y);
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[k][c] *= f;
                    const int cnt = min(32, i1 - ib);
#pragma unroll 1
                    for (int s = 0; s < cnt; s += AT_ONCE) {
                        float4 o[AT_ONCE][NV];
                        float w[AT_ONCE];
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) {   // (lanes beyond cnt hold no part)
                            w[u] = __shfl_sync(0xffffffffu, wgt, (s + u) & 31);
                            const float *src = reinterpret_cast<const float *>(
                                __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(at.o), (s + u) & 31));
#pragma unroll
                            for (int k = 0; k < NV; ++k) {
                                const int e = (k * 32 + lane) * 4;
                                o[u][k] = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (src != nullptr && s + u < cnt && e < p.d) o[u][k] = *reinterpret_cast<const float4 *>(src + e);
                            }
                        }
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
                            for (int k = 0; k < NV; ++k) {
                                acc[k][0] = fmaf(w[u], o[u][k].x, acc[k][0]);
                                acc[k][1] = fmaf(w[u], o[u][k].y, acc[k][1]);
                                acc[k][2] = fmaf(w[u], o[u][k].z, acc[k][2]);
                                acc[k][3] = fmaf(w[u], o[u][k].w, acc[k][3]);
                            }
                    }
                }
            }
            if (wpr > 1) {
                if (lane == 0) {
                    sh_ml[warp][0] = M;
                    sh_ml[warp][1] = sum;
                }
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    *reinterpret_cast<float4 *>(&sh_o[warp][(k * 32 + lane) * 4]) = make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
                __syncthreads();
                if (sub == 0 && on) {
                    float m_all = M;
                    for (int s = 1; s < wpr; ++s) m_all = fmaxf(m_all, sh_ml[warp + s][0]);
                    float own_sum = sum, own[NV][4];
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int c = 0; c < 4; ++c) own[k][c] = acc[k][c], acc[k][c] = 0.f;
                    sum = 0.f;
#pragma unroll 1
                    for (int s = 0; s < wpr; ++s) {
                        const float ms = s == 0 ? M : sh_ml[warp + s][0], f = ms == -INFINITY ? 0.f : exp2f(ms - m_all);
                        sum = fmaf(f, s == 0 ? own_sum : sh_ml[warp + s][1], sum);
#pragma unroll
                        for (int k = 0; k < NV; ++k)
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                acc[k][c] = fmaf(f, s == 0 ? own[k][c] : sh_o[warp + s][(k * 32 + lane) * 4 + c], acc[k][c]);
                    }
                    M = m_all;
                }
                __syncthreads();
            }
            if (on && sub == 0) {
                const float inv = M == -INFINITY ? 0.f : 1.0f / sum;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int e = (k * 32 + lane) * 4;
                    const float f[4] = {acc[k][0] * inv, acc[k][1] * inv, acc[k][2] * inv, acc[k][3] * inv};
                    if (e < p.d) store_row4<T>(out + tok * ld_out + hq * p.d + e, f);
                }
            }
        }
        // (blocks that see nothing come first, and in front of the last one)
        if (cut || !p.fused || ++b >= n_blocks) return;
    }
}

griffin_status launch_attn_join(const AttnPlan &plan, int dtype, void *out, long long ld_out, cudaStream_t stream) {
    AttnPlan p = plan;
    int by_row = p.hkv * (p.fused ? p.n_seq : p.n_seq + p.n_tokens / p.block_tokens);
    // (with no more tokens than a row tile takes, no block has several; a kernel without streams cuts those too)
    const int cut = p.fused && (!p.alt || p.n_tokens > p.tile_tokens) ? p.grid * (p.cta_rows / JOIN_ROWS) : 0;
    const void *fn = dtype == GRIFFIN_DT_F32 ? (p.d <= 128 ? reinterpret_cast<const void *>(attn_join_kernel<float, 1>)
                                                           : reinterpret_cast<const void *>(attn_join_kernel<float, 2>))
                                             : (p.d <= 128 ? reinterpret_cast<const void *>(attn_join_kernel<__nv_bfloat16, 1>)
                                                           : reinterpret_cast<const void *>(attn_join_kernel<__nv_bfloat16, 2>));
    // More warps to a row shorten its chain, more CTAs than fit at once lengthen the whole: with 320 one-row blocks 128
    // threads take 30.7 us with the attention in front (256: 34.8), with 96 five-row blocks 256 take 22.8 (128: 25.6).
    // Jobs of several rows go to several CTAs while there are fewer CTAs than fit at once (8 tokens of one sequence, 32 heads
    // over 8, behind 9000: 52.7 -> 22.1 us), unless the jobs by row are the rare ones (a prompt's last block).
    const bool rows_here = !p.fused || (p.alt && p.n_tokens <= p.n_seq * p.tile_tokens);
    const int most = (p.n_tokens < p.block_tokens ? p.n_tokens : p.block_tokens) * p.group, room = 2 * p.grid / by_row;
    int split = room < 1 || !rows_here ? 1 : room < most ? room : most;
    const int threads = by_row * split + cut > 2 * p.grid ? JOIN_THREADS / 2 : JOIN_THREADS;
    void *args[] = {&p, &out, &ld_out, &by_row, &split};
    return launch_maybe_overlapped(fn, dim3(by_row * split + cut), dim3(threads), 0, stream, true, args) == cudaSuccess ? GRIFFIN_OK
                                                                                                                     : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
