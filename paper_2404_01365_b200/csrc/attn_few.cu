// Attention over the shared prefix and each sequence's own keys, bf16 storage, blocks of up to 8 query rows: single
// tokens and a few drafted ones.  The mathematics is attn_tc.cu's:
//   S = scale Q K^T, masked by place;  m' = max(m, max S);  P = 2^(S - m');
//   l = l 2^(m - m') + sum P;  O = O 2^(m - m') + P V        (S in units of log2; fp32, P rounded to bf16 for P V, whose
//   two operands are of one type)
//
// With 8 rows the products fit the time of the keys' bytes even on the warp-level matrix instruction, so nothing is
// gained by the 128-row tcgen05 tiles, and their long way to the first result (barriers, tensor memory, descriptors, a
// schedule handed from warp to warp) is lost: what counts is to have the keys on their way early.  Here every warp works
// alone: it takes 16 keys of each tile, brings them by cp.async into its own ring of STAGES buffers, multiplies, keeps
// its own m, l and O in registers.  No barrier is met in the loop; the warps' results are put together through shared
// memory once per segment (the next segment's first keys are asked for before), those of other CTAs by the joining
// kernel.
// Fragments (m16n8k16): both products are formed transposed, S^T = K Q^T and O^T = V^T P^T, so that the 16 rows of the
// instruction are keys or entries and its 8 columns the queries: none is empty.  K rows are the left operand as they lie
// (ldmatrix), V rows transposed (ldmatrix.trans), P^T is turned by movmatrix, the queries stay in registers.  16-byte
// pieces of a row are placed at piece ^ (row mod 8), which keeps the loads free of bank conflicts.
//
// Measured, the joining kernel included: one sequence of 32 heads behind 20000 tokens (332 MB) 61.2 us, 5.4 TB/s, 0.83 of
// the measured copy; behind 512 tokens (10 MB) 12.8 us, of which the bytes are 1.6: the launches, the schedule's loads, the
// pages', the keys', and the partials' follow one another.
#include "attn.h"
#include "attn_join.cuh"
#include "decode_mma.cuh"

namespace griffin {

constexpr int FEW_ROWS = 8;

// DP: the head's width rounded up to 64, 128 or 256.
template <int DP> struct FewCfg {
    static constexpr int WARPS = DP == 256 ? 4 : 8, THREADS = 32 * WARPS;
    static constexpr int KT = 16 * WARPS;                     // keys per tile
    static constexpr int STAGES = DP == 64 ? 4 : 3;
    static constexpr int BUF = 16 * DP * 2;                   // 16 keys, or 16 values
    static constexpr int WARP_BYTES = STAGES * 2 * BUF;
    static constexpr int PIECES = DP / 8;                     // 16-byte pieces of a key
    static constexpr int LDO = DP + 4;                        // a warp's results, row by row
    static size_t smem(int n_seq) { return WARPS * WARP_BYTES + 2 * WARPS * FEW_ROWS * 4 + ((size_t)n_seq + 3) * 4; }
};

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t few_pack(float a, float b) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}

// The tiles of one segment.
struct FewKeys {
    const int *own_pages;
    int pre_tiles, own_len, head;
};
// This warp's 16 keys of tile t: the first of them, how many keys there are, their pages.
struct FewTile {
    const int *pages;
    int key0, len;
    bool pre;
};
template <int DP> __device__ __forceinline__ FewTile few_tile(const AttnPlan &p, const FewKeys &s, int t) {
    const bool pre = t < s.pre_tiles;
    const int key0 = (pre ? t : t - s.pre_tiles) * FewCfg<DP>::KT + (threadIdx.x >> 5) * 16;
    return {pre ? p.prefix_pages : s.own_pages, key0, pre ? p.prefix_len : s.own_len, pre};
}
// Pages of keys 0-7 and 8-15 (a page has 8 keys at least).
__device__ __forceinline__ int2 few_pages(const AttnPlan &p, const FewTile &t) {
    return make_int2(t.key0 < t.len ? __ldg(t.pages + (t.key0 >> p.page_shift)) : -1,
                     t.key0 + 8 < t.len ? __ldg(t.pages + ((t.key0 + 8) >> p.page_shift)) : -1);
}
// Asks for them; keys that are not there, and entries from the head's width on, become zeros.
template <int DP>
__device__ __forceinline__ void few_copy(const AttnPlan &p, const AttnData &x, int head, const FewTile &t, int2 page, uint32_t buf) {
    using Cfg = FewCfg<DP>;
    constexpr int STEP = 32 / Cfg::PIECES;   // keys that the warp brings at once
    const int lane = threadIdx.x & 31, mask = (1 << p.page_shift) - 1, r0 = lane / Cfg::PIECES, e = lane % Cfg::PIECES;
    const bool ok[2] = {(unsigned)page.x < (unsigned)p.n_pages, (unsigned)page.y < (unsigned)p.n_pages};
    if ((t.key0 < t.len && !ok[0]) || (t.key0 + 8 < t.len && !ok[1])) raise_status(p.ws, DEV_STATUS_BAD_INDEX, 42);
#pragma unroll
    for (int h = 0; h < 2; ++h) {   // keys 0-7, 8-15
        const int left = ok[h] && e * 8 < p.d ? t.len - t.key0 - h * 8 : 0;
        const long long at = left > 0 ? 2 * ((h ? page.y : page.x) * x.stride_page + head * x.stride_head +
                                             ((t.key0 + h * 8 & mask) + r0) * x.stride_token + e * 8)
                                      : 0;
        const char *k = static_cast<const char *>(x.k) + at, *v = static_cast<const char *>(x.v) + at;
#pragma unroll
        for (int i = 0; i < 8; i += STEP) {
            const bool there = r0 + i < left;
            const uint32_t to = buf + (h * 8 + r0 + i) * (DP * 2) + ((e ^ (r0 + i)) * 16);
            copy16(to, there ? k : static_cast<const char *>(x.k), there);
            copy16(to + Cfg::BUF, there ? v : static_cast<const char *>(x.v), there);
            k += 2 * STEP * x.stride_token;
            v += 2 * STEP * x.stride_token;
        }
    }
}
__device__ __forceinline__ FewKeys few_keys(const AttnPlan &p, const AttnJob &j) {
    return {p.page_table + (long long)j.seq * p.table_stride, j.seq < 0 || p.fused ? p.prefix_tiles : 0, j.own_len, j.head};
}
// Asks for the first tiles of a segment (n from t0 on), into the buffers from `slot` on; the pages of the next one.
template <int DP>
__device__ __forceinline__ int2 few_start(const AttnPlan &p, const AttnData &x, const FewKeys &keys, int t0, int n, uint32_t ring, int slot) {
    using Cfg = FewCfg<DP>;
    int2 page[Cfg::STAGES];
#pragma unroll
    for (int i = 0; i < Cfg::STAGES; ++i) {
        page[i] = make_int2(-1, -1);
        if (i < n) page[i] = few_pages(p, few_tile<DP>(p, keys, t0 + i));
    }
#pragma unroll
    for (int i = 0; i < Cfg::STAGES - 1; ++i) {
        const int to = slot + i < Cfg::STAGES ? slot + i : slot + i - Cfg::STAGES;
        if (i < n) few_copy<DP>(p, x, keys.head, few_tile<DP>(p, keys, t0 + i), page[i], ring + to * 2 * Cfg::BUF);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    return page[Cfg::STAGES - 1];
}

// Values that are not finite, of keys that not all rows of the block see: P = 0 would not keep them from the rows that do not
// (0 times them is NaN).  They are replaced by zero before the product,
template <int DP> static __device__ __noinline__ void few_clear_not_finite(uint8_t *values) {
    __syncwarp();
    for (int i = threadIdx.x & 31; i < 16 * FewCfg<DP>::PIECES; i += 32) {
        uint4 *const at = reinterpret_cast<uint4 *>(values) + i;
        *at = finite_or_zero8(*at);
    }
    __syncwarp();
}
// and added to the warp's results (rows LDO apart) of the rows that do see them: whatever P, the sum is what P times them
// gives.  t0, n: the segment's tiles.  (The 16 keys are cleared together, so those are looked at from their first on.)
template <int DP>
static __device__ __noinline__ void few_add_not_finite(const AttnPlan &p, const AttnData &x, const AttnJob &j, int pre_tiles, int t0, int n,
                                                       float *results) {
    using Cfg = FewCfg<DP>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k0 = max(max(j.seen0, 0) & ~15, (t0 - pre_tiles) * Cfg::KT), k1 = min(j.own_len, (t0 + n - pre_tiles) * Cfg::KT);
    __syncwarp();
    for (int k = k0; k < k1; ++k) {
        if (k / 16 % Cfg::WARPS != warp || lane >= Cfg::PIECES || lane * 8 >= p.d) continue;
        const int page = __ldg(p.page_table + (long long)j.seq * p.table_stride + (k >> p.page_shift));
        if ((unsigned)page >= (unsigned)p.n_pages) continue;
        const __nv_bfloat16 *const v = static_cast<const __nv_bfloat16 *>(x.v) + page * x.stride_page + j.head * x.stride_head +
                                       (k & ((1 << p.page_shift) - 1)) * x.stride_token + lane * 8;
        for (int e = 0; e < 8; ++e) {
            const float f = __bfloat162float(v[e]);
            if (fabsf(f) < INFINITY) continue;
            for (int r = 0; r < j.rows; ++r)
                if (k < j.seen0 + attn_row_token(p, r)) results[r * Cfg::LDO + lane * 8 + e] += f;
        }
    }
    __syncwarp();
}

// The queries of a job as the first product takes them: row lane / 4.
template <int DP>
__device__ __forceinline__ void few_queries(const AttnPlan &p, const AttnData &x, const AttnJob &j, uint32_t (&q)[DP / 16][2]) {
    const int lane = threadIdx.x & 31, r = lane >> 2, tok = attn_row_token(p, r);
    const __nv_bfloat16 *const at = static_cast<const __nv_bfloat16 *>(x.q) + (j.tok0 + tok) * x.ld_q +
                                    (j.head * p.group + r - tok * p.group) * p.d;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = c * 16 + h * 8 + (lane & 3) * 2;
            q[c][h] = r < j.rows && e < p.d ? *reinterpret_cast<const uint32_t *>(at + e) : 0u;
        }
}

template <int DP>
__global__ void __launch_bounds__(FewCfg<DP>::THREADS, 1) attn_few_kernel(const __grid_constant__ AttnPlan p,
                                                                       const __grid_constant__ AttnData x) {
    using Cfg = FewCfg<DP>;
    constexpr int NC = DP / 16, STAGES = Cfg::STAGES;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    float *const sh_m = reinterpret_cast<float *>(smem_raw + Cfg::WARPS * Cfg::WARP_BYTES), *const sh_l = sh_m + Cfg::WARPS * FEW_ROWS;
    int *const bases = reinterpret_cast<int *>(sh_l + Cfg::WARPS * FEW_ROWS);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t *const mine = smem_raw + warp * Cfg::WARP_BYTES;
    const uint32_t ring = smem_u32(mine);

    pdl_launch_dependents();
    pdl_wait_prior_grids();
    attn_scan(p, bases);
    const AttnShares shares(bases[p.n_seq], p.grid);
    if ((int)blockIdx.x >= shares.G) return;
    int g = shares.first(blockIdx.x);
    const int g_end = shares.first(blockIdx.x + 1);
    AttnJob j = attn_find(p, bases, g);
    if (tid == 0) attn_note_cut(p, shares, j, g, min(g_end, j.g1));
    FewKeys keys = few_keys(p, j);
    int slot = 0;
    int2 ahead = few_start<DP>(p, x, keys, g - j.g0, min(g_end, j.g1) - g, ring, slot);
    uint32_t q[NC][2];
    few_queries<DP>(p, x, j, q);
    for (;;) {
        const int stop = min(g_end, j.g1), n = stop - g, t0 = g - j.g0;
        const bool first = g == j.g0, whole = first && stop == j.g1;
        // queries lie by row lane / 4, results by rows ra and ra + 1
        const int rq = lane >> 2, ra = (lane & 3) * 2, tok_a = attn_row_token(p, ra), tok_b = attn_row_token(p, ra + 1);
        float m_a = -INFINITY, m_b = -INFINITY, l_a = 0.f, l_b = 0.f, o[NC][4];
#pragma unroll
        for (int i = 0; i < NC; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

        int used = 0;
        bool marked = false;   // whether values were cleared, and have to be added to the rows that see them
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();   // the tile of this turn has come, for every lane; the buffers of the turn before are done with
            if (i + STAGES - 1 < n) {
                const int to = slot == 0 ? STAGES - 1 : slot - 1;
                few_copy<DP>(p, x, j.head, few_tile<DP>(p, keys, t0 + i + STAGES - 1), ahead, ring + to * 2 * Cfg::BUF);
                if (i + STAGES < n) ahead = few_pages(p, few_tile<DP>(p, keys, t0 + i + STAGES));
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            used = slot * 2 * Cfg::BUF;   // buffer of the tile of this turn
            const uint32_t kb = ring + used, vb = kb + Cfg::BUF;
            slot = slot + 1 == STAGES ? 0 : slot + 1;
            const FewTile t = few_tile<DP>(p, keys, t0 + i);
            if (t.key0 >= t.len) continue;
            float s0[4] = {}, s1[4] = {};   // (two sums, for a shorter chain)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int row = lane & 15, piece = 2 * c + (lane >> 4);
                uint32_t a[4];
                ldmatrix4(a, kb + row * (DP * 2) + ((piece ^ (row & 7)) * 16));
                mma_bf16(c & 1 ? s1 : s0, a[0], a[1], a[2], a[3], q[c][0], q[c][1]);
            }
            // keys of the 16 that the two rows see
            const int see_a = (t.pre ? t.len : min(t.len, j.seen0 + tok_a)) - t.key0, see_b = (t.pre ? t.len : min(t.len, j.seen0 + tok_b)) - t.key0;
            float s[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[2 * h] = rq + 8 * h < see_a ? (s0[2 * h] + s1[2 * h]) * p.scale_log2 : -INFINITY;
                s[2 * h + 1] = rq + 8 * h < see_b ? (s0[2 * h + 1] + s1[2 * h + 1]) * p.scale_log2 : -INFINITY;
            }
            float x_a = max_nan(s[0], s[2]), x_b = max_nan(s[1], s[3]);
#pragma unroll
            for (int w = 4; w < 32; w *= 2) {
                x_a = max_nan(x_a, __shfl_xor_sync(0xffffffffu, x_a, w));
                x_b = max_nan(x_b, __shfl_xor_sync(0xffffffffu, x_b, w));
            }
            const bool up_a = !(x_a <= m_a), up_b = !(x_b <= m_b);
            if (__any_sync(0xffffffffu, up_a || up_b)) {   // (a logit that is NaN or infinite makes the row NaN: x - x)
                float f_a = 1.f, f_b = 1.f;
                if (up_a) {
                    f_a = fast_exp2(m_a - x_a);
                    l_a = l_a * f_a + (x_a - x_a);
                    m_a = x_a == x_a ? x_a : INFINITY;
                }
                if (up_b) {
                    f_b = fast_exp2(m_b - x_b);
                    l_b = l_b * f_b + (x_b - x_b);
                    m_b = x_b == x_b ? x_b : INFINITY;
                }
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    o[c][0] *= f_a;
                    o[c][1] *= f_b;
                    o[c][2] *= f_a;
                    o[c][3] *= f_b;
                }
            }
            const float b_a = m_a == -INFINITY ? 0.f : m_a, b_b = m_b == -INFINITY ? 0.f : m_b;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[2 * h] = fast_exp2(s[2 * h] - b_a);
                s[2 * h + 1] = fast_exp2(s[2 * h + 1] - b_b);
                l_a += s[2 * h];
                l_b += s[2 * h + 1];
            }
            if (!t.pre && j.seen0 < t.len && t.key0 + 16 > j.seen0) {   // keys that some rows see and some do not
                NotFinite8 bad;
                for (int e = lane; e < 16 * Cfg::PIECES; e += 32) bad.add(*reinterpret_cast<const uint4 *>(mine + used + Cfg::BUF + e * 16));
                if (__any_sync(0xffffffffu, bad.any())) {
                    few_clear_not_finite<DP>(mine + used + Cfg::BUF);
                    marked = true;
                }
            }
            const uint32_t w0 = movmatrix_t(few_pack(s[0], s[1])), w1 = movmatrix_t(few_pack(s[2], s[3]));
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int row = (lane >> 4) * 8 + (lane & 7), piece = 2 * c + ((lane >> 3) & 1);
                uint32_t a[4];
                ldmatrix4_t(a, vb + row * (DP * 2) + ((piece ^ (row & 7)) * 16));
                mma_bf16(o[c], a[0], a[1], a[2], a[3], w0, w1);
            }
        }
        // the next segment's first keys, then the warps' results, through the buffers of this one's last tile
        g = stop;
        AttnJob next = j;
        if (g < g_end) {
            next = attn_next(p, bases, j);
            keys = few_keys(p, next);
            ahead = few_start<DP>(p, x, keys, 0, min(g_end, next.g1) - g, ring, slot);
        }
        __syncwarp();
#pragma unroll
        for (int w = 4; w < 32; w *= 2) {
            l_a += __shfl_xor_sync(0xffffffffu, l_a, w);
            l_b += __shfl_xor_sync(0xffffffffu, l_b, w);
        }
        if (lane < 4) {
            *reinterpret_cast<float2 *>(sh_m + warp * FEW_ROWS + ra) = make_float2(m_a, m_b);
            *reinterpret_cast<float2 *>(sh_l + warp * FEW_ROWS + ra) = make_float2(l_a, l_b);
        }
        float *const so = reinterpret_cast<float *>(mine + used) + ra * Cfg::LDO + rq;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (ra < j.rows) {
                so[c * 16] = o[c][0];
                so[c * 16 + 8] = o[c][2];
            }
            if (ra + 1 < j.rows) {
                so[Cfg::LDO + c * 16] = o[c][1];
                so[Cfg::LDO + c * 16 + 8] = o[c][3];
            }
        }
        if (marked) few_add_not_finite<DP>(p, x, j, j.seq < 0 || p.fused ? p.prefix_tiles : 0, t0, n, reinterpret_cast<float *>(mine + used));
        if (g < g_end) few_queries<DP>(p, x, next, q);
        __syncthreads();
        const bool direct = attn_direct(p, j, whole);
        for (int i = tid; i < j.rows * (DP / 4); i += Cfg::THREADS) {
            const int r = i / (DP / 4), e = i % (DP / 4) * 4;
            if (e >= p.d) continue;
            float M = -INFINITY, sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < Cfg::WARPS; ++w) M = fmaxf(M, sh_m[w * FEW_ROWS + r]);
#pragma unroll
            for (int w = 0; w < Cfg::WARPS; ++w) {
                const float m = sh_m[w * FEW_ROWS + r], f = m == -INFINITY ? 0.f : fast_exp2(m - M);
                const float4 v = *reinterpret_cast<const float4 *>(smem_raw + w * Cfg::WARP_BYTES + used + (r * Cfg::LDO + e) * 4);
                sum = fmaf(f, sh_l[w * FEW_ROWS + r], sum);
                if (m != -INFINITY) {   // (a weight of 0 counts: it keeps NaN)
                    acc.x = fmaf(f, v.x, acc.x);
                    acc.y = fmaf(f, v.y, acc.y);
                    acc.z = fmaf(f, v.z, acc.z);
                    acc.w = fmaf(f, v.w, acc.w);
                }
            }
            if (direct) {
                const int tok = attn_row_token(p, r);
                const float inv = M == -INFINITY ? 0.f : 1.0f / sum;
                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(x.out) + (j.tok0 + tok) * x.ld_out +
                                           (j.head * p.group + r - tok * p.group) * p.d + e) =
                    make_uint2(few_pack(acc.x * inv, acc.y * inv), few_pack(acc.z * inv, acc.w * inv));
            } else {
                const PartPlace at = attn_place(p, j, first, 0, r);
                if (e == 0) *reinterpret_cast<float2 *>(at.ml) = make_float2(M, sum);
                *reinterpret_cast<float4 *>(at.o + e) = acc;
            }
        }
        if (g >= g_end) return;
        j = next;
        __syncthreads();  // the results' buffers may be filled again
    }
}

AttnShape attn_few_shape(int head_dim) {
    return {FEW_ROWS, 1, head_dim <= 128 ? FewCfg<128>::KT : FewCfg<256>::KT, 0};
}

template <int DP> static griffin_status launch_dp(AttnPlan p, AttnData x, cudaStream_t stream) {
    const void *fn = reinterpret_cast<const void *>(attn_few_kernel<DP>);
    const size_t smem = FewCfg<DP>::smem(p.n_seq);
    if (ensure_dynamic_smem(fn, smem) != cudaSuccess) return GRIFFIN_ERR_CUDA;
    void *args[] = {&p, &x};
    return launch_maybe_overlapped(fn, dim3(p.grid), dim3(FewCfg<DP>::THREADS), smem, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

griffin_status launch_attn_few(const AttnPlan &plan, const AttnData &data, cudaStream_t stream) {
    if (plan.d <= 64) return launch_dp<64>(plan, data, stream);
    if (plan.d <= 128) return launch_dp<128>(plan, data, stream);
    return launch_dp<256>(plan, data, stream);
}

}  // namespace griffin
