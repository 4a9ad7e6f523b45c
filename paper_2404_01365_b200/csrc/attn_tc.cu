// Attention over the shared prefix and each sequence's own keys on the 5th-generation tensor cores, bf16
// storage, fp32 accumulation:
//   S = Q K^T;  P = 2^(c S - m) with c = scale log2(e) and m the row's running maximum of c S;
//   l += sum P;  O += P V;  when m grows by more than 2^8 can hold, O and l are scaled by 2^(m_old - m_new)
//
// One persistent CTA per SM, each with its share of the call's key tiles (attn_plan.cuh), 384 threads:
//   warp 0      TMA: query tiles and, page by page, key and value tiles (128-byte swizzle) into a ring
//   warp 1      MMA issuer; it also owns the TMEM allocation
//   warp 2      sees the tiles arrive and clears the rows of a value tile that no key stands for (0 * NaN would reach
//               the sum)
//   warp 3      walks the share, segment by segment (a segment: what the share has of one job), and hands descriptions
//               of the segments to the others through a ring in shared memory
//   warps 4-7, 8-11   two softmax groups, a row per thread: S from TMEM, P (bf16) back to TMEM over S,
//               and at the end of a segment O to the output or the partials
// The work is a sequence of UNITS (one row tile times one key tile).  Unit U belongs to group U & 1, which has
// its own S/P columns and (heads of up to 128 entries) its own O columns.  A block of two row tiles meets each key
// tile with two units; a block of one row tile gives its key tiles to the two groups in turn, and the two O are
// joined with the other partials.  The issuer runs S = Q K^T two units ahead of P V: one group's softmax runs
// under the other's products.  (An issuer for each group was slower: the groups then fall into step, softmax with
// softmax and product with product.)  Heads wider than 128 fill the O columns with one accumulator; then one
// group does all units, with the same two S buffers.
//
// MMAs of one thread complete in the order of issue, and tcgen05.commit covers all before it: with two
// accumulators, S of a group's next unit is issued behind P V of its last, so its barrier also says that P V has
// read P and updated O.
//
// Every wait is bounded; after a give-up the CTA still frees its TMEM before it returns.
#include "attn.h"
#include "attn_join.cuh"
#include "tmem_wide.cuh"

namespace griffin {

constexpr int ATC_THREADS = 384, ATC_ROWS = 128;
constexpr float ATC_SLACK = 8.f;  // how far (log2) the true maximum may run ahead of the one P is scaled by

template <int DP> struct AtcCfg {
    static constexpr int KT = DP == 256 ? 64 : 128;       // keys per tile
    static constexpr int NS = DP == 256 ? 1 : 2;          // O accumulators
    static constexpr int CB = DP / 64;                    // 64-entry column blocks (128 swizzled bytes per row)
    static constexpr int Q_BYTES = ATC_ROWS * DP * 2, KV_BYTES = KT * DP * 2;
    static constexpr int O_COL = 2 * KT;                  // TMEM columns: S/P 0, S/P 1, O (0, 1); P of 64 keys over the first half of their S
    static constexpr int MAX_SLOTS = DP == 64 ? 10 : 5;
};
constexpr int ATC_SEGS = 4;   // ring of segment descriptions
// barriers, by number
constexpr int B_KV_FULL = 0, B_KV_EMPTY = 10, B_Q_FULL = 20, B_Q_EMPTY = 22, B_S_FULL = 24, B_P_READY = 26, B_O_FULL = 28,
              B_SEG_FULL = 30, B_SEG_EMPTY = B_SEG_FULL + ATC_SEGS, B_V_OK = B_SEG_EMPTY + ATC_SEGS, ATC_BARS = B_V_OK + 10;

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
// (stepping 16 keys adds 2048 bytes to the start address)
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(const void *tile, uint32_t block) {
    return (uint64_t)((smem_u32(tile) >> 4) & 0x3FFFu) | ((uint64_t)(block >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
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
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"::
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
// 32 bytes, a whole sector, in one store (the partials' rows start on 32-byte boundaries)
__device__ __forceinline__ void store_8f(float *to, const float *v) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                 "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 2^x to about 2^-22, 0 for -inf
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void prefetch_tensormap(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// the largest of three, NaN if there is one
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// two fp32 lanes in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(d)
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)), "l"(*reinterpret_cast<uint64_t *>(&c)));
    return *reinterpret_cast<float2 *>(&d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return *reinterpret_cast<float2 *>(&d);
}
// 2^x of both lanes on the FMA and integer pipes, x >= -120 after clamping: n = the integer next to x (by adding
// 1.5 * 2^23), f = x - n, a cubic for 2^f on [-1/2, 1/2] (its own minimax fit, relative error 7.5e-5: a fiftieth of
// the rounding of P to bf16 that follows), n into the exponent.
__device__ __forceinline__ float2 poly_exp2(float2 x) {
    const float2 magic = make_float2(12582912.f, 12582912.f), neg = make_float2(-12582912.f, -12582912.f);
    x.x = fmaxf(x.x, -120.f);
    x.y = fmaxf(x.y, -120.f);
    const float2 n = add2(x, magic), back = add2(n, neg);
    const float2 f = fma2(back, make_float2(-1.f, -1.f), x);
    float2 y = fma2(f, make_float2(0.0551716685295105f, 0.0551716685295105f), make_float2(0.2426111251115799f, 0.2426111251115799f));
    y = fma2(y, f, make_float2(0.6932609677314758f, 0.6932609677314758f));
    y = fma2(y, f, make_float2(0.9999280571937561f, 0.9999280571937561f));
    y.x = __int_as_float(__float_as_int(y.x) + (__float_as_int(n.x) << 23));
    y.y = __int_as_float(__float_as_int(y.y) + (__float_as_int(n.y) << 23));
    return y;
}
// P of 64 keys: 2^(c S - m), summed in fp32 and packed to bf16.  ATC_POLY of every 8 pairs go through poly_exp2: the
// special-function unit gives 16 results a clock and SM, and 32768 of them per tile would take as long as the
// four products of the tile do.  (A key that is not seen comes out as 2^-120 there, not 0: a row that sees nothing
// at all is known by its m.)
constexpr int ATC_POLY = 4;
__device__ __forceinline__ void exp_pairs(const float (&s)[64], float2 scale2, float2 off2, float2 (&sum)[2], uint32_t (&pk)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        float2 e = fma2(make_float2(s[2 * i], s[2 * i + 1]), scale2, off2);
        if ((i * 3 & 7) < ATC_POLY) {
            e = poly_exp2(e);
        } else {
            e.x = fast_exp2(e.x);
            e.y = fast_exp2(e.y);
        }
        sum[i & 1] = add2(sum[i & 1], e);
        const __nv_bfloat162 x = __floats2bfloat162_rn(e.x, e.y);
        pk[i] = *reinterpret_cast<const uint32_t *>(&x);
    }
}
// What is not part of every tile's loop is kept out of line: the loops of all warps together have to fit in the SM's
// instruction cache (measured: with the whole row of 128 in one stretch of code, a prompt took a fifth longer).
//
// Keys from `lim` on are not seen: -inf in their places of S, whatever is there.
template <int KT> static __device__ __noinline__ void mask_tile(uint32_t ts, int lim) {
#pragma unroll 1
    for (int c = 0; c < KT; c += 32) {
        float s[32];
        uint32_t r[32];
        tmem_ld32(ts + c, s);
#pragma unroll
        for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(c + i < lim ? s[i] : -INFINITY);
        tmem_st32(ts + c, r);
    }
    tmem_wait_st();
}
template <int DP> static __device__ __noinline__ void scale_out(uint32_t to, float f) {
#pragma unroll 1
    for (int c = 0; c < DP; c += 32) {
        float o[32];
        uint32_t r[32];
        tmem_ld32(to + c, o);
#pragma unroll
        for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(o[i] * f);
        tmem_st32(to + c, r);
    }
}
// A row of O: times `scale` and rounded to dst, or as it is to the partials (dst NULL); nothing where on is false.
template <int DP>
static __device__ __noinline__ void write_out(uint32_t to, int d, bool on, float scale, __nv_bfloat16 *dst, float *part) {
#pragma unroll 1
    for (int c = 0; c < DP; c += 32) {
        float o[32];
        tmem_ld32(to + c, o);
        if (!on) continue;
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
            if (c + i >= d) continue;
            if (dst != nullptr) {
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 x = __floats2bfloat162_rn(o[i + 2 * e] * scale, o[i + 2 * e + 1] * scale);
                    h[e] = *reinterpret_cast<const uint32_t *>(&x);
                }
                *reinterpret_cast<uint4 *>(dst + c + i) = make_uint4(h[0], h[1], h[2], h[3]);
            } else {
                store_8f(part + c + i, o + i);
            }
        }
    }
}

// Barriers by their shared-memory address: the issuers' instructions between two products are what their chains wait for.
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// What every wait needs when it does not succeed at once.
struct WaitCtx {
    volatile int *abort;
    void *ws;
};
// The bounded wait's slow path, in one place: the loops below stay small enough for the instruction cache
// (with everything inlined the kernel was 128 KB of code and spent half its time fetching it).
static __device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int *abort, void *ws, int where) {
    const long long t0 = clock64();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 4096; ++i)
            if (bar_try(bar, parity)) return true;
        if (*abort) return false;
        if (clock64() - t0 > WAIT_LIMIT_CYCLES) {
            *abort = 1;
            raise_status(ws, DEV_STATUS_TIMEOUT, where);
            return false;
        }
    }
}
// A wait of a whole warp: all its lanes go on, or none.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const WaitCtx &c, int where) {
    return __all_sync(0xffffffffu, bar_try(bar, parity) || wait_slow(bar, parity, c.abort, c.ws, where));
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }

// Place in a ring of barriers, and the parity that a wait for this round's completion takes.  (A wait for a barrier's
// n-th completion may only begin when the one before has been seen, or the parity of an older one passes for it: every
// reader of a ring waits at each of its places in turn.)
struct Ring {
    uint32_t slot, parity;
    __device__ __forceinline__ void step(uint32_t by, uint32_t n) {  // by <= n
        slot += by;
        if (slot >= n) {
            slot -= n;
            parity ^= 1u;
        }
    }
};

// A segment, as warp 3 hands it on.
struct __align__(16) Segment {
    int t0, n;            // first key tile (of the job's) and how many; n = 0: the share is done
    int pre_tiles;        // the job's tiles of the prefix; the others are the sequence's own
    int head, seq, tok0, rows, seen0, own_len;
    int alt, direct, first;
};

// One key tile of a job: where its keys are and how many there are.
struct KeyTile {
    int k0, len;  // first key; keys behind `len` are not there
    bool prefix;
};
__device__ __forceinline__ KeyTile key_tile(const AttnPlan &p, const Segment &s, int t) {
    KeyTile k;
    k.prefix = t < s.pre_tiles;
    k.k0 = (k.prefix ? t : t - s.pre_tiles) << p.kt_shift;
    k.len = k.prefix ? p.prefix_len : s.own_len;
    return k;
}

// A reader's place in the ring of segments.
struct SegReader {
    uint32_t slot, parity, bars;
    const Segment *ring;
    // the next segment, copied by a whole warp, which then gives its place back; false: a wait gave up.  n = 0: there is none
    __device__ __forceinline__ bool take(Segment &s, const WaitCtx &c, int where) {
        if (!warp_wait(bars + (B_SEG_FULL + slot) * 8, parity, c, where)) return false;
        s = ring[slot];
        __syncwarp();
        if ((threadIdx.x & 31) == 0) bar_arrive(bars + (B_SEG_EMPTY + slot) * 8);
        if (++slot == ATC_SEGS) {
            slot = 0;
            parity ^= 1u;
        }
        return true;
    }
};

template <int DP>
__global__ void __launch_bounds__(ATC_THREADS, 1) attn_tc_kernel(const __grid_constant__ AtcMaps maps,
                                                              const __grid_constant__ AtcParams prm) {
    using Cfg = AtcCfg<DP>;
    constexpr int KT = Cfg::KT, NS = Cfg::NS, CB = Cfg::CB;
    const AttnPlan &p = prm.plan;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *const s_q = base;                                  // NS query tiles
    uint8_t *const s_kv = base + NS * Cfg::Q_BYTES;             // ring of key and value tiles
    const int n_slots = prm.n_slots;
    uint64_t *const bar_mem = reinterpret_cast<uint64_t *>(s_kv + n_slots * Cfg::KV_BYTES);
    Segment *const segs = reinterpret_cast<Segment *>(bar_mem + ATC_BARS);
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(segs + ATC_SEGS);
    const WaitCtx ctx{reinterpret_cast<volatile int *>(tmem_slot + 1), p.ws};
    int *const bases = reinterpret_cast<int *>(tmem_slot + 2);
    const uint32_t bars = smem_u32(bar_mem);
    const auto bar = [bars](int b, uint32_t i) { return bars + (b + i) * 8; };

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    if (tid < 3) prefetch_tensormap(tid == 0 ? &maps.q : tid == 1 ? &maps.k : &maps.v);
    if (tid == 0) {
#pragma unroll 1
        for (int i = 0; i < ATC_BARS; ++i) {
            int n = 1;
            if (i >= B_P_READY && i < B_O_FULL) n = 4;                   // the group's warps
            else if (i >= B_SEG_EMPTY && i < B_V_OK) n = 3 + 4 * NS;      // warps 0 to 2, softmax warps
            mbar_init(bar_mem + i, n);
        }
        *ctx.abort = 0;
        mbar_fence_init();
    }
    pdl_wait_prior_grids();
    attn_scan(p, bases);
    const AttnShares shares(bases[p.n_seq], p.grid);
    if ((int)blockIdx.x >= shares.G) return;
    if (warp == 1) tmem_alloc(tmem_slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    SegReader seg{0, 0, bars, segs};

    if (warp == 0) {
        // ---------------- loads ----------------
        uint32_t kv_n = 0, nq = 0;  // ring slots and query buffers handed out so far
        Ring kv{0, 0};
        Segment w;
        bool ok = true;
        const int per_tile = KT / prm.box_rows;  // boxes per 64-entry block
        const uint32_t q_at = smem_u32(s_q), kv_at = smem_u32(s_kv);
        while (ok && (ok = seg.take(w, ctx, 49)) && w.n > 0) {
            const int q_tiles = NS == 2 && !w.alt ? 2 : 1;
            for (int r = 0; r < q_tiles && ok; ++r, ++nq) {
                const uint32_t b = nq % NS;
                if (nq >= NS && !(ok = warp_wait(bar(B_Q_EMPTY, b), (nq / NS - 1) & 1, ctx, 50))) break;
                if (lane == 0) {
                    bar_expect(bar(B_Q_FULL, b), CB * prm.q_box_bytes);
#pragma unroll 1
                    for (int c = 0; c < CB; ++c)
                        tma_load_3d(q_at + b * Cfg::Q_BYTES + c * (ATC_ROWS * 128), &maps.q, c * 64, w.head * p.group,
                                    w.tok0 + r * p.tile_tokens, bar(B_Q_FULL, b));
                }
            }
            for (int t = 0; t < w.n && ok; ++t) {
                const KeyTile k = key_tile(p, w, w.t0 + t);
                const int *const pages = k.prefix ? p.prefix_pages : p.page_table + (long long)w.seq * p.table_stride;
#pragma unroll 1
                for (int which = 0; which < 2; ++which) {
                    const uint32_t full = bar(B_KV_FULL, kv.slot), dst = kv_at + kv.slot * Cfg::KV_BYTES;
                    if (kv_n >= (uint32_t)n_slots && !(ok = warp_wait(bar(B_KV_EMPTY, kv.slot), kv.parity ^ 1u, ctx, 51))) break;
                    if (lane == 0) bar_expect(full, Cfg::KV_BYTES);
                    __syncwarp();
#pragma unroll 1
                    for (int i = lane; i < per_tile * CB; i += 32) {
                        const int r = i / CB, c = i % CB, key = k.k0 + r * prm.box_rows;
                        // a box behind the last key: a page that is not there reads as zeros
                        int page = p.n_pages;
                        if (key < k.len) {
                            page = __ldg(pages + (key >> p.page_shift));
                            if (page < 0 || page >= p.n_pages) {
                                attn_bad(p.ws, 42);
                                page = p.n_pages;
                            }
                        }
                        tma_load_4d(dst + c * (KT * 128) + r * prm.box_rows * 128, which ? &maps.v : &maps.k, c * 64,
                                    key & ((1 << p.page_shift) - 1), w.head, page, full);
                    }
                    __syncwarp();
                    kv.step(1, n_slots);
                    ++kv_n;
                }
            }
        }
        // stay until every copy that was started has landed
        if (lane == 0) {
            const long long t_0 = clock64();
            for (uint32_t i = kv_n > (uint32_t)n_slots ? kv_n - n_slots : 0; i < kv_n; ++i)
                while (!bar_try(bar(B_KV_FULL, i % n_slots), (i / n_slots) & 1))
                    if (clock64() - t_0 > WAIT_LIMIT_CYCLES) break;
            for (uint32_t i = nq > (uint32_t)NS ? nq - NS : 0; i < nq; ++i)
                while (!bar_try(bar(B_Q_FULL, i % NS), (i / NS) & 1))
                    if (clock64() - t_0 > WAIT_LIMIT_CYCLES) break;
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        // (the whole warp walks, one lane issues: the operands stay in uniform registers)
        constexpr uint32_t ID_QK = umma_idesc(ATC_ROWS, KT), ID_PV = umma_idesc(ATC_ROWS, DP) | (1u << 16);
        // Where S = Q K^T stands (a) and where P V (b): unit in its segment, units in it, whether blocks of two row tiles.
        uint32_t a_seg = 0, a_par = 0, b_seg = 0, b_par = 0, a_n = 0, b_n = 0, a_u = 0, b_u = 0;
        uint32_t a_U = 0, b_U = 0, qi = 0;   // units of the CTA; first query tile of a's segment
        bool a_dual = false, b_dual = false;
        Ring ka{0, 0}, vb{1, 0}, okb{0, 0};  // ring places of the next key tile, of the next value tile, and the latter's B_V_OK
        const uint64_t q_desc = smem_desc_sw128(s_q, 0), k_desc = smem_desc_sw128(s_kv, 0), v_desc = smem_desc_mn_sw128(s_kv, KT * 128);
        const auto next_segment = [&](uint32_t &place, uint32_t &par, uint32_t &n, bool &dual, bool last_reader) -> bool {
            if (!warp_wait(bar(B_SEG_FULL, place), par, ctx, 48)) return false;
            const Segment &s = segs[place];
            dual = NS == 2 && uniform(s.alt) == 0;
            n = uniform(s.n) << (dual ? 1 : 0);
            __syncwarp();
            if (last_reader && lane == 0) bar_arrive(bar(B_SEG_EMPTY, place));
            if (++place == ATC_SEGS) {
                place = 0;
                par ^= 1u;
            }
            return true;
        };
        bool ok = next_segment(a_seg, a_par, a_n, a_dual, false) && next_segment(b_seg, b_par, b_n, b_dual, true);
        uint32_t ahead = 0;  // units whose S has been issued and P V not: two in front of every P V
        while (ok && b_n > 0) {
            if (ahead < 2 && a_n > 0) {
                const uint32_t q_at = qi + (a_dual ? a_u & 1 : 0), qb = NS == 2 ? q_at & 1 : 0;
                if (a_u < (a_dual ? 2u : 1u) && !(ok = warp_wait(bar(B_Q_FULL, qb), (NS == 2 ? q_at >> 1 : q_at) & 1, ctx, 52))) break;
                if (!(ok = warp_wait(bar(B_KV_FULL, ka.slot), ka.parity, ctx, 53))) break;
                tc_fence_after_sync();
                const uint64_t q = q_desc + (uint64_t)(qb * (Cfg::Q_BYTES >> 4)), k = k_desc + (uint64_t)(ka.slot * (Cfg::KV_BYTES >> 4));
                const uint32_t buf = a_U & 1, d = tmem + buf * KT;
                const bool k_done = !a_dual || (a_u & 1), q_done = a_u + (a_dual ? 2 : 1) >= a_n;
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk)
                        umma_bf16(d, q + (uint64_t)(((kk >> 2) * (ATC_ROWS * 128) + (kk & 3) * 32) >> 4),
                                  k + (uint64_t)(((kk >> 2) * (KT * 128) + (kk & 3) * 32) >> 4), ID_QK, kk > 0);
                    commit_to(bar(B_S_FULL, buf));
                    if (k_done) commit_to(bar(B_KV_EMPTY, ka.slot));
                    if (q_done) commit_to(bar(B_Q_EMPTY, qb));
                }
                __syncwarp();
                if (k_done) ka.step(2, n_slots);
                ++a_U;
                ++ahead;
                if (++a_u == a_n) {
                    qi += a_dual ? 2 : 1;
                    a_u = 0;
                    ok = next_segment(a_seg, a_par, a_n, a_dual, false);
                }
                continue;
            }
            const uint32_t buf = b_U & 1, o = NS == 2 ? buf : 0;
            // (warp 2 has seen the tile arrive)
            if (!warp_wait(bar(B_V_OK, okb.slot), okb.parity, ctx, 54)) break;
            if (!warp_wait(bar(B_P_READY, buf), (b_U >> 1) & 1, ctx, 55)) break;
            tc_fence_after_sync();
            const uint32_t d = tmem + Cfg::O_COL + o * DP, pt = tmem + buf * KT, add = b_u >= NS;
            const uint64_t v = v_desc + (uint64_t)(vb.slot * (Cfg::KV_BYTES >> 4));
            const bool v_done = !b_dual || (b_u & 1);
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < KT / 16; ++kk) umma_bf16_ts(d, pt + (kk >> 2) * 64 + (kk & 3) * 8, v + (uint64_t)(kk * (2048 >> 4)), ID_PV, kk > 0 ? 1 : add);
                if (v_done) commit_to(bar(B_KV_EMPTY, vb.slot));
                if (NS == 1 || b_u + 2 >= b_n) commit_to(bar(B_O_FULL, o));
            }
            __syncwarp();
            if (v_done) {
                vb.step(2, n_slots);
                okb.step(1, n_slots);
            }
            --ahead;
            ++b_U;
            if (++b_u == b_n) {
                b_u = 0;
                ok = next_segment(b_seg, b_par, b_n, b_dual, true);
            }
        }
    } else if (warp == 2) {
        // ---------------- value tiles: rows that no key stands for become zeros ----------------
        Segment w;
        Ring kv{0, 0}, done{0, 0};
        bool ok = true;
        while (ok && (ok = seg.take(w, ctx, 47)) && w.n > 0) {
#pragma unroll 1
            for (int t = 0; t < w.n && ok; ++t) {
                const KeyTile k = key_tile(p, w, w.t0 + t);
                if (!(ok = warp_wait(bar(B_KV_FULL, kv.slot), kv.parity, ctx, 56))) break;
                kv.step(1, n_slots);
                if (!(ok = warp_wait(bar(B_KV_FULL, kv.slot), kv.parity, ctx, 56))) break;
                const int valid = k.len - k.k0;
                if (valid < KT) {
                    uint8_t *const tile = s_kv + kv.slot * Cfg::KV_BYTES;
#pragma unroll 1
                    for (int i = lane; i < (KT - valid) * 8 * CB; i += 32) {
                        const int c = i % CB, r = valid + i / CB / 8, e = i / CB % 8;
                        *reinterpret_cast<uint4 *>(tile + c * (KT * 128) + r * 128 + e * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                if (lane == 0) bar_arrive(bar(B_V_OK, done.slot));
                kv.step(1, n_slots);
                done.step(1, n_slots);
            }
        }
    } else if (warp == 3) {
        // ---------------- schedule ----------------
        if (lane == 0) {
            int g = shares.first(blockIdx.x);
            const int g_end = shares.first(blockIdx.x + 1);
            AttnJob j = attn_find(p, bases, g);
            attn_note_cut(p, shares, j, g, min(g_end, j.g1));
            Ring sg{0, 0};
            for (uint32_t k = 0;; ++k) {
                if (k >= ATC_SEGS && !bar_try(bar(B_SEG_EMPTY, sg.slot), sg.parity ^ 1u) &&
                    !wait_slow(bar(B_SEG_EMPTY, sg.slot), sg.parity ^ 1u, ctx.abort, ctx.ws, 46))
                    break;
                const int stop = min(g_end, j.g1);
                Segment w;
                w.t0 = g - j.g0;
                w.n = stop - g;
                w.pre_tiles = j.seq < 0 || p.fused ? p.prefix_tiles : 0;
                w.head = j.head;
                w.seq = j.seq;
                w.tok0 = j.tok0;
                w.rows = j.rows;
                w.seen0 = j.seen0;
                w.own_len = j.own_len;
                w.alt = j.alt;
                w.first = g == j.g0;
                w.direct = attn_direct(p, j, w.first && stop == j.g1);
                segs[sg.slot] = w;
                bar_arrive(bar(B_SEG_FULL, sg.slot));
                if (w.n == 0) break;
                sg.step(1, ATC_SEGS);
                g = stop;
                if (g < g_end) j = attn_next(p, bases, j);
                else j.g1 = g;  // the last description: no tiles
            }
        }
    } else if (warp >= 4 && (NS == 2 || warp < 8)) {
        // ---------------- softmax ----------------
        const uint32_t grp = (warp - 4) >> 2;
        const int wr = (warp & 3) * 32;                            // the group's rows of this warp: wr .. wr + 31
        const uint32_t lanes = tmem + ((uint32_t)wr << 16);
        const int tile_rows = p.tile_tokens * p.group;
        Segment j;
        uint32_t U0 = 0, n_o = 0;  // units before this segment; segments finished by this group
        bool ok = true;
        while (ok && (ok = seg.take(j, ctx, 45)) && j.n > 0) {
            const bool dual = NS == 2 && !j.alt;
            const uint32_t n = (uint32_t)j.n << (dual ? 1 : 0);
            uint32_t u = NS == 2 ? (U0 ^ grp) & 1 : 0;             // the group's first unit
            const int row0 = dual ? (int)u * tile_rows : 0, r = wr + lane, row = row0 + r;
            const bool valid = r < tile_rows && row < j.rows;
            const bool warp_on = wr < tile_rows && row0 + wr < j.rows;
            const int tok = attn_row_token(p, row), own_seen = j.seen0 + tok;
            const int stream = j.alt ? (int)u : 0;
            const bool has = u < n;
            float m = -INFINITY, l = 0.f;
            bool started = false;
            for (; u < n && ok; u += NS) {
                const uint32_t U = U0 + u, buf = U & 1;
                const KeyTile k = key_tile(p, j, j.t0 + (int)(dual ? u >> 1 : u));
                bool o_seen = u == 0;   // (one accumulator: whether P V of the unit before is known to be done)
                ok = warp_wait(bar(B_S_FULL, buf), (U >> 1) & 1, ctx, 57);
                if (!ok) break;
                tc_fence_after_sync();
                if (warp_on) {
                    const uint32_t ts = lanes + buf * KT;
                    const int lim = (k.prefix ? k.len : min(k.len, own_seen)) - k.k0;   // keys of the tile that the row sees
                    if (__any_sync(0xffffffffu, lim < KT)) mask_tile<KT>(ts, lim);
                    float s[64], mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
                    for (int c = 0; c < KT; c += 64) {
                        tmem_ld64(ts + c, s);
#pragma unroll
                        for (int i = 0; i < 64; i += 8)
#pragma unroll
                            for (int e = 0; e < 4; ++e) mx4[e] = max3_nan(mx4[e], s[i + e], s[i + 4 + e]);
                    }
                    const float mx = max3_nan(max3_nan(mx4[0], mx4[1], mx4[2]), mx4[3], -INFINITY) * p.scale_log2;
                    if (mx != -INFINITY) l += mx - mx;   // a NaN or an infinity among the logits makes the row NaN
                    // the maximum moves only when 2^(c S - m) could grow too large (or there is none yet)
                    const bool move = mx > m + ATC_SLACK || (m == -INFINITY && mx > m);
                    if (__any_sync(0xffffffffu, move)) {
                        const float f = move ? fast_exp2(m - mx) : 1.f;   // (0 for the first)
                        if (move) m = mx;
                        l *= f;
                        if (started) {
                            // (one accumulator: S of this unit was issued before P V of the last one, so its barrier
                            // does not cover it)
                            if (NS == 1) {
                                if (!(ok = warp_wait(bar(B_O_FULL, 0), (U - 1) & 1, ctx, 59))) break;
                                o_seen = true;
                                tc_fence_after_sync();
                            }
                            scale_out<DP>(lanes + Cfg::O_COL + (NS == 2 ? buf : 0) * DP, f);
                        }
                    }
                    const float off = m == -INFINITY ? 0.f : m;
                    const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), off2 = make_float2(-off, -off);
                    float2 sum[2] = {};
                    // (the last 64 keys first: they are still here; the count is hidden from the compiler, and the loop
                    // in this form, so that its body is laid out once)
                    int c = KT - 64;
                    asm volatile("" : "+r"(c));
#pragma unroll 1
                    do {
                        uint32_t pk[32];
                        if (c != KT - 64) tmem_ld64(ts + c, s);
                        exp_pairs(s, scale2, off2, sum, pk);
                        tmem_st32(ts + c, pk);
                        c -= 64;
                    } while (c >= 0);
                    const float2 both = add2(sum[0], sum[1]);
                    l += both.x + both.y;
                    started = true;
                    tmem_wait_st();
                }
                if (NS == 1 && !o_seen && !(ok = warp_wait(bar(B_O_FULL, 0), (U - 1) & 1, ctx, 59))) break;
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(bar(B_P_READY, buf));
            }
            // the segment's result
            if (ok && has) {
                ok = warp_wait(bar(B_O_FULL, NS == 2 ? grp : 0), (NS == 2 ? n_o : U0 + n - 1) & 1, ctx, 58);
                ++n_o;
                if (ok && warp_on) {
                    tc_fence_after_sync();
                    const uint32_t to = lanes + Cfg::O_COL + (NS == 2 ? grp : 0) * DP;
                    __nv_bfloat16 *dst = nullptr;
                    float *part = nullptr;
                    if (j.direct) {
                        dst = static_cast<__nv_bfloat16 *>(prm.out) + (j.tok0 + tok) * prm.ld_out +
                              (j.head * p.group + row - tok * p.group) * p.d;
                    } else if (valid) {
                        const PartPlace at = attn_place(p, PartJob{j.seq, j.head, j.tok0, j.alt != 0}, j.first != 0, stream, row);
                        *reinterpret_cast<float2 *>(at.ml) = make_float2(m, l);
                        part = at.o;
                    }
                    write_out<DP>(to, p.d, valid, m == -INFINITY ? 0.f : 1.0f / l, dst, part);
                    tc_fence_before_sync();
                }
            } else if (ok && valid && j.alt) {  // a segment of one tile leaves the other stream empty
                *reinterpret_cast<float2 *>(attn_place(p, PartJob{j.seq, j.head, j.tok0, j.alt != 0}, j.first != 0, stream, row).ml) = make_float2(-INFINITY, 0.f);
            }
            U0 += n;
        }
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
    const size_t tail = ATC_BARS * 8 + ATC_SEGS * sizeof(Segment) + 8 + ((size_t)plan.n_seq + 1) * 4, fixed = 1024 + Cfg::NS * Cfg::Q_BYTES + tail;
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
