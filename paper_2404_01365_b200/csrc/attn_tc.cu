// Attention over the shared prefix and each sequence's own keys on the 5th-generation tensor cores, bf16
// storage, fp32 accumulation:
//   S = Q K^T;  P = 2^(c S - m) with c = scale log2(e) and m the row's running maximum of c S;
//   l += sum P;  O += P V;  when m grows by more than 2^8 can hold, O and l are scaled by 2^(m_old - m_new)
//
// One persistent CTA per SM, each with its share of the call's key tiles (attn_plan.cuh), 384 threads:
//   warp 0      TMA producer: query tiles and, page by page, key and value tiles (128-byte swizzle) into a ring
//   warp 1      MMA issuer: one thread issues tcgen05.mma; it also owns the TMEM allocation
//   warp 2      clears the rows of a value tile that no key stands for (0 * NaN would reach the sum)
//   warps 4-7, 8-11   two softmax groups, a row per thread: S from TMEM, P (bf16) back to TMEM over S,
//               and at the end of a segment O to the output or the partials
// The work is a sequence of UNITS (one row tile times one key tile).  Unit U belongs to softmax group U & 1,
// which has its own S/P columns and (heads of up to 128 entries) its own O columns.  A block of two row
// tiles meets each key tile with two units; a block of one row tile gives its key tiles to the two groups in
// turn, and the two O are joined with the other partials.  The issuer runs S = Q K^T two units ahead of P V, so
// one group's softmax runs under the other's products.  Heads wider than 128 fill the O columns with one
// accumulator; then one group does all units, with the same two S buffers.
//
// MMAs of one thread complete in the order of issue, and tcgen05.commit covers all before it: S of unit U + 2
// is issued behind P V of unit U, so its barrier also says that P V of unit U has read P and updated O.
//
// Every wait is bounded; after a give-up the CTA still frees its TMEM before it returns.
#include "attn.h"
#include "attn_join.cuh"
#include "tc_common.cuh"

namespace griffin {

constexpr int ATC_THREADS = 384, ATC_ROWS = 128;
constexpr float ATC_SLACK = 8.f;  // how far (log2) the true maximum may run ahead of the one P is scaled by

template <int DP> struct AtcCfg {
    static constexpr int KT = DP == 256 ? 64 : 128;       // keys per tile
    static constexpr int NS = DP == 256 ? 1 : 2;          // O accumulators
    static constexpr int CB = DP / 64;                    // 64-entry column blocks (128 swizzled bytes per row)
    static constexpr int Q_BYTES = ATC_ROWS * DP * 2, KV_BYTES = KT * DP * 2;
    static constexpr int O_COL = 2 * KT;                  // TMEM columns: S/P 0, S/P 1, O (0, 1)
    static constexpr int MAX_SLOTS = DP == 64 ? 10 : 5;
};
constexpr int ATC_BARS = 2 * 10 + 10 + 4 + 6;  // kv full/empty, v_ok, q full/empty, s_full, p_ready, o_full

struct AtcMaps {
    CUtensorMap q, k, v;
};
struct AtcParams {
    AttnPlan plan;
    void *out;
    long long ld_out;
    int n_slots, box_rows, q_box_bytes;
};

// Value tiles are read with their entries (not their keys) consecutive: swizzled blocks of 64 entries x 8 keys,
// 1024 bytes from 8 keys to the next, `block` bytes from 64 entries to the next.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(const void *tile, int k16, uint32_t block) {
    const uint32_t addr = smem_u32(tile) + (uint32_t)k16 * 2048u;
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(block >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                             uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, int x, int y, int z, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *map, int x, int y, int z, int w, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&v)[32]) {
    uint32_t r[16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[h * 16 + i]);
        tmem_st16(taddr + h * 16, r);
    }
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 2^x to about 2^-22, 0 for -inf
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A wait of a whole warp: all its lanes go on, or none.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort, void *ws, int where) {
    return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort, ws, where));
}

// Walks a CTA's share, segment by segment (a segment: what the share has of one job).
struct SegWalk {
    AttnJob j;
    long long g, stop, end;
    __device__ __forceinline__ void start(const AttnPlan &p, const long long *bases, long long g0, long long g_end) {
        g = g0;
        end = g_end;
        j = attn_find(p, bases, g0);
        stop = min(end, j.g1);
    }
    __device__ __forceinline__ bool next(const AttnPlan &p, const long long *bases) {
        if (stop >= end) return false;
        g = stop;
        j = attn_next(p, bases, j);
        stop = min(end, j.g1);
        return true;
    }
    __device__ __forceinline__ int tiles() const { return (int)(stop - g); }
    __device__ __forceinline__ int first_tile() const { return (int)(g - j.g0); }
    __device__ __forceinline__ bool from_start() const { return g == j.g0; }
    __device__ __forceinline__ bool whole() const { return g == j.g0 && stop == j.g1; }
};
// One key tile of a job: where its keys are and how many there are.
struct KeyTile {
    const int *pages;
    int k0, len;  // first key; keys behind `len` are not there
    bool prefix;
};
__device__ __forceinline__ KeyTile key_tile(const AttnPlan &p, const AttnJob &j, int t) {
    const int pre = j.seq < 0 || p.fused ? p.prefix_tiles : 0;
    KeyTile k;
    k.prefix = t < pre;
    k.k0 = (k.prefix ? t : t - pre) * p.kt;
    k.len = k.prefix ? p.prefix_len : j.own_len;
    k.pages = k.prefix ? p.prefix_pages : p.page_table + (long long)j.seq * p.table_stride;
    return k;
}

template <int DP>
__global__ void __launch_bounds__(ATC_THREADS) attn_tc_kernel(const __grid_constant__ AtcMaps maps,
                                                              const __grid_constant__ AtcParams prm) {
    using Cfg = AtcCfg<DP>;
    constexpr int KT = Cfg::KT, NS = Cfg::NS, CB = Cfg::CB;
    const AttnPlan &p = prm.plan;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *const s_q = base;                                  // NS query tiles
    uint8_t *const s_kv = base + NS * Cfg::Q_BYTES;             // ring of key and value tiles
    const int n_slots = prm.n_slots;
    uint64_t *const bars = reinterpret_cast<uint64_t *>(s_kv + n_slots * Cfg::KV_BYTES);
    uint64_t *const kv_full = bars, *const kv_empty = bars + 10, *const v_ok = bars + 20, *const q_full = bars + 30,
                   *const q_empty = bars + 32, *const s_full = bars + 34, *const p_ready = bars + 36, *const o_full = bars + 38;
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(bars + ATC_BARS);
    volatile int *const abort = reinterpret_cast<volatile int *>(tmem_slot + 1);
    long long *const bases = reinterpret_cast<long long *>(bars + ATC_BARS + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < n_slots; ++i) {
            mbar_init(&kv_full[i], 1);
            mbar_init(&kv_empty[i], 1);
            mbar_init(&v_ok[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_ready[i], 4);  // one arrival per warp of the group
            mbar_init(&o_full[i], 1);
        }
        *abort = 0;
        mbar_fence_init();
    }
    pdl_wait_prior_grids();
    attn_scan(p, bases);
    const long long W = bases[p.n_seq];
    const int G = attn_ctas(W, p.grid);
    if ((int)blockIdx.x >= G) return;
    if (warp == 1) tmem_alloc(tmem_slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    const long long g0 = attn_share(W, G, blockIdx.x), g_end = attn_share(W, G, blockIdx.x + 1);

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        SegWalk w;
        w.start(p, bases, g0, g_end);
        uint32_t kv = 0, nq = 0;  // ring slots and query buffers handed out so far
        bool ok = true;
        const int per_tile = KT / prm.box_rows;  // boxes per 64-entry block
        do {
            const int q_tiles = NS == 2 && !w.j.alt ? 2 : 1;
            for (int r = 0; r < q_tiles && ok; ++r, ++nq) {
                const int b = nq % NS;
                if (nq >= NS) ok = warp_wait(&q_empty[b], (nq / NS - 1) & 1, abort, p.ws, 50);
                if (ok && lane == 0) {
                    mbar_arrive_expect_tx(&q_full[b], CB * prm.q_box_bytes);
                    for (int c = 0; c < CB; ++c)
                        tma_load_3d(s_q + b * Cfg::Q_BYTES + c * (ATC_ROWS * 128), &maps.q, c * 64, w.j.head * p.group,
                                    w.j.tok0 + r * p.tile_tokens, &q_full[b]);
                }
            }
            const int t0 = w.first_tile(), n = w.tiles();
            for (int t = 0; t < n && ok; ++t) {
                const KeyTile k = key_tile(p, w.j, t0 + t);
                for (int which = 0; which < 2 && ok; ++which, ++kv) {
                    const int slot = kv % n_slots;
                    if (kv >= (uint32_t)n_slots) ok = warp_wait(&kv_empty[slot], (kv / n_slots - 1) & 1, abort, p.ws, 51);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(&kv_full[slot], Cfg::KV_BYTES);
                    __syncwarp();
                    for (int i = lane; i < per_tile * CB; i += 32) {
                        const int r = i / CB, c = i % CB, key = k.k0 + r * prm.box_rows;
                        // a box behind the last key: a page that is not there reads as zeros
                        int page = p.n_pages;
                        if (key < k.len) {
                            page = __ldg(k.pages + (key >> p.page_shift));
                            if (page < 0 || page >= p.n_pages) {
                                raise_status(p.ws, DEV_STATUS_BAD_INDEX, 42);
                                page = p.n_pages;
                            }
                        }
                        tma_load_4d(s_kv + slot * Cfg::KV_BYTES + c * (KT * 128) + r * prm.box_rows * 128, which ? &maps.v : &maps.k,
                                    c * 64, key & ((1 << p.page_shift) - 1), w.j.head, page, &kv_full[slot]);
                    }
                    __syncwarp();
                }
            }
        } while (ok && w.next(p, bases));
        // stay until every copy that was started has landed
        if (lane == 0) {
            const long long t_0 = clock64();
            for (uint32_t i = kv > (uint32_t)n_slots ? kv - n_slots : 0; i < kv; ++i)
                while (!mbar_try_wait(&kv_full[i % n_slots], (i / n_slots) & 1))
                    if (clock64() - t_0 > WAIT_LIMIT_CYCLES) break;
            for (uint32_t i = nq > (uint32_t)NS ? nq - NS : 0; i < nq; ++i)
                while (!mbar_try_wait(&q_full[i % NS], (i / NS) & 1))
                    if (clock64() - t_0 > WAIT_LIMIT_CYCLES) break;
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0) {
            constexpr uint32_t ID_QK = umma_idesc(ATC_ROWS, KT), ID_PV = umma_idesc(ATC_ROWS, DP) | (1u << 16);
            SegWalk a, b;  // where S = Q K^T stands, and where P V
            a.start(p, bases, g0, g_end);
            b = a;
            bool a_more = true, ok = true;
            uint32_t ua = 0, Ua = 0, kva = 0, qa = 0;  // a's unit in its segment, unit of the CTA, first ring slot and query buffer of the segment
            uint32_t ub = 0, kvb = 0;
            const auto units = [](const SegWalk &w) { return (uint32_t)w.tiles() * (NS == 2 && !w.j.alt ? 2u : 1u); };

            const auto issue_qk = [&]() -> bool {
                const bool dual = NS == 2 && !a.j.alt;
                const uint32_t n = units(a), t = dual ? ua >> 1 : ua, qi = qa + (dual ? ua & 1 : 0), qb = qi % NS;
                const uint32_t slot = (kva + 2 * t) % n_slots;
                if (ua < (dual ? 2u : 1u) && !wait_or_abort(&q_full[qb], (qi / NS) & 1, abort, p.ws, 52)) return false;
                if (!wait_or_abort(&kv_full[slot], ((kva + 2 * t) / n_slots) & 1, abort, p.ws, 53)) return false;
                tc_fence_after_sync();
                const uint8_t *const q = s_q + qb * Cfg::Q_BYTES, *const k = s_kv + slot * Cfg::KV_BYTES;
                const uint32_t d = tmem + (Ua & 1) * KT;
#pragma unroll
                for (int kk = 0; kk < DP / 16; ++kk)
                    umma_bf16(d, smem_desc_sw128(q + (kk >> 2) * (ATC_ROWS * 128), kk & 3),
                              smem_desc_sw128(k + (kk >> 2) * (KT * 128), kk & 3), ID_QK, kk > 0);
                umma_commit(&s_full[Ua & 1]);
                if (!dual || (ua & 1)) umma_commit(&kv_empty[slot]);
                if (ua + (dual ? 2 : 1) >= n) umma_commit(&q_empty[qb]);
                ++Ua;
                if (++ua == n) {
                    qa += dual ? 2 : 1;
                    kva += 2 * a.tiles();
                    ua = 0;
                    a_more = a.next(p, bases);
                }
                return true;
            };
            ok = issue_qk() && (!a_more || issue_qk());
            bool b_more = true;
            for (uint32_t U = 0; ok && b_more; ++U) {
                const bool dual = NS == 2 && !b.j.alt;
                const uint32_t n = units(b), t = dual ? ub >> 1 : ub, vi = kvb + 2 * t + 1, slot = vi % n_slots, vt = vi >> 1;
                if (!wait_or_abort(&kv_full[slot], (vi / n_slots) & 1, abort, p.ws, 54)) break;
                if (!wait_or_abort(&v_ok[vt % n_slots], (vt / n_slots) & 1, abort, p.ws, 54)) break;
                if (!wait_or_abort(&p_ready[U & 1], (U >> 1) & 1, abort, p.ws, 55)) break;
                tc_fence_after_sync();
                const uint32_t o = NS == 2 ? U & 1 : 0;
                const uint8_t *const v = s_kv + slot * Cfg::KV_BYTES;
#pragma unroll
                for (int kk = 0; kk < KT / 16; ++kk)
                    umma_bf16_ts(tmem + Cfg::O_COL + o * DP, tmem + (U & 1) * KT + kk * 8, smem_desc_mn_sw128(v, kk, KT * 128),
                                 ID_PV, ub >= NS || kk > 0);
                if (!dual || (ub & 1)) umma_commit(&kv_empty[slot]);
                if (NS == 1 || ub + 2 >= n) umma_commit(&o_full[o]);
                if (a_more) ok = issue_qk();
                if (++ub == n) {
                    kvb += 2 * b.tiles();
                    ub = 0;
                    b_more = b.next(p, bases);
                }
            }
        }
    } else if (warp == 2) {
        // ---------------- value tiles: rows that no key stands for become zeros ----------------
        SegWalk w;
        w.start(p, bases, g0, g_end);
        uint32_t vt = 0;
        bool ok = true;
        do {
            const int t0 = w.first_tile(), n = w.tiles();
            for (int t = 0; t < n && ok; ++t, ++vt) {
                const KeyTile k = key_tile(p, w.j, t0 + t);
                const uint32_t vi = 2 * vt + 1, slot = vi % n_slots;
                ok = warp_wait(&kv_full[slot], (vi / n_slots) & 1, abort, p.ws, 56);
                const int valid = k.len - k.k0;
                if (ok && valid < KT) {
                    for (int i = lane; i < (KT - valid) * 8 * CB; i += 32) {
                        const int c = i % CB, r = valid + i / CB / 8, e = i / CB % 8;
                        *reinterpret_cast<uint4 *>(s_kv + slot * Cfg::KV_BYTES + c * (KT * 128) + r * 128 + e * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(&v_ok[vt % n_slots]);
            }
        } while (ok && w.next(p, bases));
    } else if (warp >= 4 && (NS == 2 || warp < 8)) {
        // ---------------- softmax ----------------
        const uint32_t grp = (warp - 4) >> 2;
        const int wr = (warp & 3) * 32;                            // the group's rows of this warp: wr .. wr + 31
        const uint32_t lanes = tmem + ((uint32_t)wr << 16);
        const int tile_rows = p.tile_tokens * p.group;
        SegWalk w;
        w.start(p, bases, g0, g_end);
        uint32_t U0 = 0, n_o = 0;  // units before this segment; segments finished by this group
        bool ok = true;
        do {
            const AttnJob &j = w.j;
            const bool dual = NS == 2 && !j.alt;
            const uint32_t n = (uint32_t)w.tiles() * (dual ? 2u : 1u);
            uint32_t u = NS == 2 ? (U0 ^ grp) & 1 : 0;             // the group's first unit
            const int t0 = w.first_tile(), row0 = dual ? (int)u * tile_rows : 0, r = wr + lane, row = row0 + r;
            const bool valid = r < tile_rows && row < j.rows;
            const bool warp_on = wr < tile_rows && row0 + wr < j.rows;
            const int tok = row / p.group, own_seen = j.seen0 + tok;
            const int stream = j.alt ? (int)u : 0;
            const bool has = u < n;
            float m = -INFINITY, l = 0.f;
            bool started = false;
            for (; u < n && ok; u += NS) {
                const uint32_t U = U0 + u, buf = U & 1;
                const KeyTile k = key_tile(p, j, t0 + (int)(dual ? u >> 1 : u));
                ok = warp_wait(&s_full[buf], (U >> 1) & 1, abort, p.ws, 57);
                if (!ok) break;
                tc_fence_after_sync();
                if (warp_on) {
                    const uint32_t ts = lanes + buf * KT;
                    const int lim = (k.prefix ? k.len : min(k.len, own_seen)) - k.k0;   // keys of the tile that the row sees
                    const bool masked = __any_sync(0xffffffffu, lim < KT);
                    float mx = -INFINITY;
#pragma unroll
                    for (int c = 0; c < KT; c += 32) {
                        float s[32];
                        tmem_ld32(ts + c, s);
                        if (masked) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) mx = fmaxf(mx, c + i < lim ? s[i] : -INFINITY);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) mx = fmaxf(mx, s[i]);
                        }
                    }
                    mx *= p.scale_log2;
                    // the maximum moves only when 2^(c S - m) could grow too large (or there is none yet)
                    const bool move = mx > m + ATC_SLACK || (m == -INFINITY && mx > m);
                    if (__any_sync(0xffffffffu, move)) {
                        const float f = move ? fast_exp2(m - mx) : 1.f;   // (0 for the first)
                        if (move) m = mx;
                        l *= f;
                        if (started) {
                            // (one accumulator: S of this unit was issued before P V of the last one, so its barrier
                            // does not cover it)
                            if (NS == 1 && !(ok = warp_wait(&o_full[0], (U - 1) & 1, abort, p.ws, 59))) break;
                            tc_fence_after_sync();
                            const uint32_t to = lanes + Cfg::O_COL + (NS == 2 ? buf : 0) * DP;
#pragma unroll 1
                            for (int c = 0; c < DP; c += 32) {
                                float o[32];
                                tmem_ld32(to + c, o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] *= f;
                                tmem_st32(to + c, o);
                            }
                        }
                    }
                    const float off = m == -INFINITY ? 0.f : m;
                    float sum = 0.f;
#pragma unroll
                    for (int c = 0; c < KT; c += 32) {
                        float s[32];
                        tmem_ld32(ts + c, s);
                        uint32_t pk[16];
                        float e[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            e[i] = fast_exp2(fmaf(s[i], p.scale_log2, -off));
                            if (masked && c + i >= lim) e[i] = 0.f;
                            sum += e[i];
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(e[2 * i], e[2 * i + 1]);
                            pk[i] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                        tmem_st16(ts + c / 2, pk);
                    }
                    l += sum;
                    started = true;
                    tmem_wait_st();
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_ready[buf]);
            }
            // the segment's result
            if (ok && has) {
                ok = warp_wait(&o_full[NS == 2 ? grp : 0], (NS == 2 ? n_o : U0 + n - 1) & 1, abort, p.ws, 58);
                ++n_o;
                if (ok && warp_on) {
                    tc_fence_after_sync();
                    const uint32_t to = lanes + Cfg::O_COL + (NS == 2 ? grp : 0) * DP;
                    if (attn_direct(p, j, w.whole())) {
                        const float inv = l == 0.f ? 0.f : 1.0f / l;
                        __nv_bfloat16 *const dst = static_cast<__nv_bfloat16 *>(prm.out) + (j.tok0 + tok) * prm.ld_out +
                                                   (j.head * p.group + row % p.group) * p.d;
#pragma unroll 1
                        for (int c = 0; c < DP; c += 32) {
                            float o[32];
                            tmem_ld32(to + c, o);
                            if (valid) {
#pragma unroll
                                for (int i = 0; i < 32; i += 8) {
                                    if (c + i >= p.d) break;
                                    uint32_t h[4];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const __nv_bfloat162 x = __floats2bfloat162_rn(o[i + 2 * e] * inv, o[i + 2 * e + 1] * inv);
                                        h[e] = *reinterpret_cast<const uint32_t *>(&x);
                                    }
                                    *reinterpret_cast<uint4 *>(dst + c + i) = make_uint4(h[0], h[1], h[2], h[3]);
                                }
                            }
                        }
                    } else {
                        PartPlace at{nullptr, nullptr};
                        if (valid) {
                            at = attn_place(p, j, w.from_start(), stream, row);
                            *reinterpret_cast<float2 *>(at.ml) = make_float2(m, l);
                        }
#pragma unroll 1
                        for (int c = 0; c < DP; c += 32) {
                            float o[32];
                            tmem_ld32(to + c, o);
                            if (valid) {
#pragma unroll
                                for (int i = 0; i < 32; i += 8) {
                                    if (c + i >= p.d) break;
                                    float2 *const dst = reinterpret_cast<float2 *>(at.o + c + i);
#pragma unroll
                                    for (int e = 0; e < 4; ++e) dst[e] = make_float2(o[i + 2 * e], o[i + 2 * e + 1]);
                                }
                            }
                        }
                    }
                    tc_fence_before_sync();
                }
            } else if (ok && valid && j.alt) {  // a segment of one tile leaves the other stream empty
                *reinterpret_cast<float2 *>(attn_place(p, j, w.from_start(), stream, row).ml) = make_float2(-INFINITY, 0.f);
            }
            U0 += n;
        } while (ok && w.next(p, bases));
    }

    // ---------------- teardown: everybody meets, the allocating warp frees TMEM ----------------
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

template <int DP> static griffin_status launch_dp(const AttnPlan &plan, const AttnData &x, cudaStream_t stream) {
    using Cfg = AtcCfg<DP>;
    AtcMaps maps;
    AtcParams prm{};
    prm.plan = plan;
    prm.out = x.out;
    prm.ld_out = x.ld_out;
    const int page = 1 << plan.page_shift;
    prm.box_rows = page < Cfg::KT ? page : Cfg::KT;
    prm.q_box_bytes = plan.tile_tokens * plan.group * 128;
    EncodeTiledFn enc = encode_tiled_fn();
    if (enc == nullptr) return GRIFFIN_ERR_CUDA;
    {
        const cuuint64_t dims[3] = {(cuuint64_t)plan.d, (cuuint64_t)plan.hq, (cuuint64_t)plan.n_tokens};
        const cuuint64_t strides[2] = {(cuuint64_t)plan.d * 2, (cuuint64_t)x.ld_q * 2};
        const cuuint32_t box[3] = {64, (cuuint32_t)plan.group, (cuuint32_t)plan.tile_tokens}, ones[3] = {1, 1, 1};
        if (enc(&maps.q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(x.q), dims, strides, box, ones,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return GRIFFIN_ERR_CUDA;
    }
    for (int which = 0; which < 2; ++which) {
        const cuuint64_t dims[4] = {(cuuint64_t)plan.d, (cuuint64_t)page, (cuuint64_t)plan.hkv, (cuuint64_t)plan.n_pages};
        const cuuint64_t strides[3] = {(cuuint64_t)x.stride_token * 2, (cuuint64_t)x.stride_head * 2, (cuuint64_t)x.stride_page * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)prm.box_rows, 1, 1}, ones[4] = {1, 1, 1, 1};
        if (enc(which ? &maps.v : &maps.k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(which ? x.v : x.k), dims, strides,
                box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return GRIFFIN_ERR_UNSUPPORTED;  // (strides that the copy engine does not take)
    }
    // as many ring slots as fit beside the list of the sequences' first tiles
    const size_t tail = ATC_BARS * 8 + 8 + ((size_t)plan.n_seq + 1) * 8, fixed = 1024 + Cfg::NS * Cfg::Q_BYTES + tail;
    prm.n_slots = (int)((232448 - fixed) / Cfg::KV_BYTES);
    if (prm.n_slots > Cfg::MAX_SLOTS) prm.n_slots = Cfg::MAX_SLOTS;
    const size_t smem = fixed + (size_t)prm.n_slots * Cfg::KV_BYTES;
    const void *fn = reinterpret_cast<const void *>(attn_tc_kernel<DP>);
    if (ensure_dynamic_smem(fn, smem) != cudaSuccess) return GRIFFIN_ERR_CUDA;
    void *args[] = {&maps, &prm};
    return launch_maybe_overlapped(fn, dim3(plan.grid), dim3(ATC_THREADS), smem, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

AttnShape attn_tc_shape(int head_dim) {
    return head_dim > 128 ? AttnShape{ATC_ROWS, 1, AtcCfg<256>::KT, 0} : AttnShape{ATC_ROWS, 2, AtcCfg<128>::KT, 1};
}

griffin_status launch_attn_tc(const AttnPlan &plan, const AttnData &data, cudaStream_t stream) {
    if (plan.d <= 64) return launch_dp<64>(plan, data, stream);
    if (plan.d <= 128) return launch_dp<128>(plan, data, stream);
    return launch_dp<256>(plan, data, stream);
}

}  // namespace griffin
