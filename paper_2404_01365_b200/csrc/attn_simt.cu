// Attention over the shared prefix and each sequence's own keys, fp32 storage, on the plain fp32 pipes:
//   S = scale Q K^T, masked by place;  m' = max(m, max S);  P = 2^(S - m');
//   l = l 2^(m - m') + sum P;  O = O 2^(m - m') + P V        (S in units of log2, all fp32)
// one CTA per SM, each with its share of the call's key tiles (attn_plan.cuh).
//
// A half warp has up to A rows, HALVES apart, and walks the whole tile: keys tx, tx + 16, ... of S, entries 4 tx .. of O.  So
// the softmax stays in registers (four shuffles a row), and P goes through shared memory within its own warp; the CTA
// meets once a tile, for the keys and values.  Those come by cp.async, the next tile's behind the present one's
// products, and their pages are looked up a tile ahead.  Keys and values behind what any row of the block sees are
// read as zeros, whatever the cache holds there.
//
// Bound by latency: 5 steps behind 1003 shared tokens (16 heads over 4, 64 wide) take 13.0 us, half of them here and the
// rest in the joining kernel; 1000 causal tokens of 8 heads over 2 take 73 us, 14 TFLOP/s of the 75 of the pipes.
#include <type_traits>

#include "attn.h"
#include "attn_join.cuh"
#include "vec8.cuh"

namespace griffin {

constexpr int SIMT_ROWS = 64;

// DP: the head's width rounded up to 64, 128 or 256.
template <int DP> struct SimtCfg {
    // 16 warps keep the pipes busier than 8 (1000 causal tokens of 8 64-wide heads over 2: 72 us, 8 warps 87); 256-wide heads
    // would read shared memory too often with so few rows to a warp (33 steps behind 3189 tokens of 16 heads: 199 us, 145)
    static constexpr int THREADS = DP == 256 ? 256 : 512, HALVES = THREADS / 16;
    static constexpr int KT = DP == 256 ? 32 : 64;                 // keys per tile: two tiles fit beside the queries
    static constexpr int LD = DP + 4;                              // (rows 16 bytes apart in the banks)
    static constexpr int TILE = KT * LD;                           // keys or values of a tile
    static constexpr int LDP = KT + 4;
    static constexpr int PASSES = KT * (DP / 4) / THREADS;    // 16-byte pieces per thread, keys as values
    static size_t smem(int n_seq) { return (SIMT_ROWS * LD + 4 * TILE + SIMT_ROWS * LDP + (size_t)n_seq + 3) * 4; }
};

// The tiles of one segment, by which the kernel and its loads find keys.
struct SimtKeys {
    const int *own_pages;
    int pre_tiles, own_len, t0, n, head;
};
template <int DP> __device__ __forceinline__ void tile_pages(const AttnPlan &p, const SimtKeys &s, int t, int (&page)[SimtCfg<DP>::PASSES]) {
    const bool pre = t < s.pre_tiles;
    const int k0 = (pre ? t : t - s.pre_tiles) * SimtCfg<DP>::KT, len = pre ? p.prefix_len : s.own_len;
    const int *const pages = pre ? p.prefix_pages : s.own_pages;
#pragma unroll
    for (int i = 0; i < SimtCfg<DP>::PASSES; ++i) {
        const int key = k0 + (threadIdx.x + i * SimtCfg<DP>::THREADS) / (DP / 4);
        page[i] = key < len ? __ldg(pages + (key >> p.page_shift)) : -1;
    }
}
template <int DP>
__device__ __forceinline__ void tile_copy(const AttnPlan &p, const AttnData &x, const SimtKeys &s, int t,
                                          const int (&page)[SimtCfg<DP>::PASSES], float *sk, float *sv) {
    const bool pre = t < s.pre_tiles;
    const int k0 = (pre ? t : t - s.pre_tiles) * SimtCfg<DP>::KT, len = pre ? p.prefix_len : s.own_len;
    const float *const k = static_cast<const float *>(x.k), *const v = static_cast<const float *>(x.v);
#pragma unroll
    for (int i = 0; i < SimtCfg<DP>::PASSES; ++i) {
        const int c = threadIdx.x + i * SimtCfg<DP>::THREADS, r = c / (DP / 4), e = c % (DP / 4) * 4, key = k0 + r;
        if (e >= p.d) continue;
        const bool there = key < len && page[i] >= 0 && page[i] < p.n_pages;
        if (key < len && !there) raise_status(p.ws, DEV_STATUS_BAD_INDEX, 42);
        const long long at = there ? page[i] * x.stride_page + s.head * x.stride_head + (key & ((1 << p.page_shift) - 1)) * x.stride_token + e : 0;
        copy16(smem_u32(sk + r * SimtCfg<DP>::LD + e), k + at, there);
        copy16(smem_u32(sv + r * SimtCfg<DP>::LD + e), v + at, there);
    }
}

// The rows of one segment, A to a half warp.  page: of the segment's first tile.
template <int DP, int A>
__device__ __forceinline__ void simt_segment(const AttnPlan &p, const AttnData &x, const AttnJob &j, const SimtKeys &keys, bool first,
                                             bool whole, float *sq, float *skv, float *sp, int (&page)[SimtCfg<DP>::PASSES]) {
    using Cfg = SimtCfg<DP>;
    constexpr int KT = Cfg::KT, LD = Cfg::LD, LDP = Cfg::LDP, NK = KT / 16, NE = DP / 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const bool on = (ty & ~1) < j.rows;       // any row of the warp
    float2 o[A][NE][2] = {};
    float m[A], l[A];
#pragma unroll
    for (int a = 0; a < A; ++a) m[a] = -INFINITY, l[a] = 0.f;
    tile_copy<DP>(p, x, keys, keys.t0, page, skv, skv + Cfg::TILE);
    if (keys.n > 1) tile_pages<DP>(p, keys, keys.t0 + 1, page);
#pragma unroll 1
    for (int i = 0; i < keys.n; ++i) {
        const int t = keys.t0 + i;
        const float *const sk = skv + (i & 1) * 2 * Cfg::TILE, *const sv = sk + Cfg::TILE;
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();   // this tile has come; the one before is done with
        if (i + 1 < keys.n) {
            float *const next = skv + (i + 1 & 1) * 2 * Cfg::TILE;
            tile_copy<DP>(p, x, keys, t + 1, page, next, next + Cfg::TILE);
            if (i + 2 < keys.n) tile_pages<DP>(p, keys, t + 2, page);
        }
        if (!on) continue;
        float2 s2[A][NK] = {};   // sums over the even and the odd entries
#pragma unroll 4
        for (int e = 0; e < p.d; e += 4) {
            float4 q[A];
#pragma unroll
            for (int a = 0; a < A; ++a) q[a] = *reinterpret_cast<const float4 *>(sq + (ty + Cfg::HALVES * a) * LD + e);
#pragma unroll
            for (int b = 0; b < NK; ++b) {
                const float4 k = *reinterpret_cast<const float4 *>(sk + (tx + 16 * b) * LD + e);
#pragma unroll
                for (int a = 0; a < A; ++a) {
                    s2[a][b] = fma2(make_float2(q[a].x, q[a].y), make_float2(k.x, k.y), s2[a][b]);
                    s2[a][b] = fma2(make_float2(q[a].z, q[a].w), make_float2(k.z, k.w), s2[a][b]);
                }
            }
        }
        float s[A][NK];
        const bool pre = t < keys.pre_tiles;
        const int k0 = (pre ? t : t - keys.pre_tiles) * KT;
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const int seen = pre ? p.prefix_len : min(keys.own_len, j.seen0 + attn_row_token(p, ty + Cfg::HALVES * a));
            float mx = -INFINITY;
#pragma unroll
            for (int b = 0; b < NK; ++b) {
                s[a][b] = k0 + tx + 16 * b < seen ? (s2[a][b].x + s2[a][b].y) * p.scale_log2 : -INFINITY;
                mx = max_nan(mx, s[a][b]);
            }
#pragma unroll
            for (int w = 1; w < 16; w *= 2) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            float f = 1.f;
            if (!(mx <= m[a])) {   // (a logit that is NaN or infinite makes the row NaN: mx - mx)
                f = exp2f(m[a] - mx);
                l[a] = l[a] * f + (mx - mx);
                m[a] = mx == mx ? mx : INFINITY;
            }
            const float base = m[a] == -INFINITY ? 0.f : m[a];
            float sum = 0.f;
#pragma unroll
            for (int b = 0; b < NK; ++b) {
                const float e = exp2f(s[a][b] - base);
                sp[(ty + Cfg::HALVES * a) * LDP + tx + 16 * b] = e;
                sum += e;
            }
#pragma unroll
            for (int w = 1; w < 16; w *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            l[a] += sum;
#pragma unroll
            for (int b = 0; b < NE; ++b)
#pragma unroll
                for (int c = 0; c < 2; ++c) o[a][b][c].x *= f, o[a][b][c].y *= f;
        }
        __syncwarp();
        // A tile with keys that some of the block's rows see and some do not: there P = 0 is no protection, since 0 times a
        // value that is not finite is NaN, so each row leaves the others' keys out.
        const int apart = pre || j.seen0 >= keys.own_len ? KT : j.seen0 - k0;   // from this key of the tile on
        const auto products = [&](const int from, const int to, const auto all_see) {
#pragma unroll(decltype(all_see)::value ? 2 : 1)
            for (int k = from; k < to; k += 4) {
                float4 w[A];
#pragma unroll
                for (int a = 0; a < A; ++a) w[a] = *reinterpret_cast<const float4 *>(sp + (ty + Cfg::HALVES * a) * LDP + k);
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int b = 0; b < NE; ++b) {
                        const float4 v = *reinterpret_cast<const float4 *>(sv + (k + u) * LD + b * 64 + tx * 4);
#pragma unroll
                        for (int a = 0; a < A; ++a) {
                            const float f = u == 0 ? w[a].x : u == 1 ? w[a].y : u == 2 ? w[a].z : w[a].w;
                            if constexpr (!decltype(all_see)::value)
                                if (k0 + k + u >= j.seen0 + attn_row_token(p, ty + Cfg::HALVES * a)) continue;
                            o[a][b][0] = fma2(make_float2(f, f), make_float2(v.x, v.y), o[a][b][0]);
                            o[a][b][1] = fma2(make_float2(f, f), make_float2(v.z, v.w), o[a][b][1]);
                        }
                    }
            }
        };
        const int cut = apart >= KT ? KT : max(apart, 0) & ~3;
        products(0, cut, std::true_type{});
        if (cut < KT) products(cut, KT, std::false_type{});
        __syncwarp();
    }
    // the segment's result
    const bool direct = attn_direct(p, j, whole);
#pragma unroll
    for (int a = 0; a < A; ++a) {
        const int r = ty + Cfg::HALVES * a;
        if (r >= j.rows) continue;
        float *to;
        float inv = 1.f;
        if (direct) {
            const int tok = attn_row_token(p, r);
            inv = m[a] == -INFINITY ? 0.f : 1.0f / l[a];
            to = static_cast<float *>(x.out) + (j.tok0 + tok) * x.ld_out + (j.head * p.group + r - tok * p.group) * p.d;
        } else {
            const PartPlace at = attn_place(p, j, first, 0, r);
            if (tx == 0) *reinterpret_cast<float2 *>(at.ml) = make_float2(m[a], l[a]);
            to = at.o;
        }
#pragma unroll
        for (int b = 0; b < NE; ++b)
            if (b * 64 + tx * 4 < p.d)
                *reinterpret_cast<float4 *>(to + b * 64 + tx * 4) =
                    make_float4(o[a][b][0].x * inv, o[a][b][0].y * inv, o[a][b][1].x * inv, o[a][b][1].y * inv);
    }
}

template <int DP>
__global__ void __launch_bounds__(SimtCfg<DP>::THREADS, 1) attn_simt_kernel(const __grid_constant__ AttnPlan p,
                                                                 const __grid_constant__ AttnData x) {
    using Cfg = SimtCfg<DP>;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    float *const sq = reinterpret_cast<float *>(smem_raw), *const skv = sq + SIMT_ROWS * Cfg::LD, *const sp = skv + 4 * Cfg::TILE;
    int *const bases = reinterpret_cast<int *>(sp + SIMT_ROWS * Cfg::LDP);
    const int tid = threadIdx.x;

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
        const SimtKeys keys{p.page_table + (long long)j.seq * p.table_stride, j.seq < 0 || p.fused ? p.prefix_tiles : 0, j.own_len,
                            g - j.g0, stop - g, j.head};
        int page[Cfg::PASSES];
        tile_pages<DP>(p, keys, keys.t0, page);
        for (int i = tid; i < j.rows * (DP / 4); i += Cfg::THREADS) {
            const int r = i / (DP / 4), e = i % (DP / 4) * 4, tok = attn_row_token(p, r);
            if (e < p.d)
                copy16(smem_u32(sq + r * Cfg::LD + e),
                       static_cast<const float *>(x.q) + (j.tok0 + tok) * x.ld_q + (j.head * p.group + r - tok * p.group) * p.d + e, true);
        }
        constexpr int H = Cfg::HALVES;
        if (j.rows <= H) simt_segment<DP, 1>(p, x, j, keys, first, whole, sq, skv, sp, page);
        else if (2 * H == SIMT_ROWS || j.rows <= 2 * H) simt_segment<DP, 2>(p, x, j, keys, first, whole, sq, skv, sp, page);
        else if constexpr (2 * H < SIMT_ROWS) {
            if (j.rows <= 3 * H) simt_segment<DP, 3>(p, x, j, keys, first, whole, sq, skv, sp, page);
            else simt_segment<DP, 4>(p, x, j, keys, first, whole, sq, skv, sp, page);
        }
        g = stop;
        if (g >= g_end) return;
        j = attn_next(p, bases, j);
        __syncthreads();  // the segment before is done with shared memory
    }
}

AttnShape attn_simt_shape(int head_dim) { return {SIMT_ROWS, 1, head_dim <= 128 ? SimtCfg<64>::KT : SimtCfg<256>::KT, 0}; }

template <int DP> static griffin_status launch_dp(AttnPlan p, AttnData x, cudaStream_t stream) {
    const void *fn = reinterpret_cast<const void *>(attn_simt_kernel<DP>);
    const size_t smem = SimtCfg<DP>::smem(p.n_seq);
    if (ensure_dynamic_smem(fn, smem) != cudaSuccess) return GRIFFIN_ERR_CUDA;
    void *args[] = {&p, &x};
    return launch_maybe_overlapped(fn, dim3(p.grid), dim3(SimtCfg<DP>::THREADS), smem, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

griffin_status launch_attn_simt(const AttnPlan &plan, const AttnData &data, cudaStream_t stream) {
    if (plan.d <= 64) return launch_dp<64>(plan, data, stream);
    if (plan.d <= 128) return launch_dp<128>(plan, data, stream);
    return launch_dp<256>(plan, data, stream);
}

}  // namespace griffin
