// Attention over the shared prefix and each sequence's own keys on the 5th-generation tensor cores, bf16
// storage, fp32 accumulation:
//   S = Q K^T;  P = 2^(c S - m) with c = scale log2(e) and m the row's running maximum of c S;
//   l += sum P;  O += P V;  when m grows by more than 2^8 can hold, O and l are scaled by 2^(m_old - m_new)
//
// One persistent CTA per SM, each with its share of the call's key tiles (attn_plan.cuh), 384 threads:
//   warp 0      TMA producer: query tiles and, page by page, key and value tiles (128-byte swizzle) into a ring
//   warp 1      MMA issuer: one thread issues tcgen05.mma; it also owns the TMEM allocation
//   warp 2      clears what must not be multiplied with in a value tile, since 0 * NaN would reach the sum: rows that no
//               key stands for, and values that are not finite of keys that not every row sees (add_not_finite)
//   warp 3      scheduler: walks the share, segment by segment (a segment: what the share has of one job), and
//               hands descriptions of the segments to the others through a ring in shared memory
//   warps 4-7, 8-11   two softmax groups, a row per thread: S from TMEM, P (bf16) back to TMEM over S,
//               and at the end of a segment O to the output or the partials
// Over a cache in 4 bits (Q4) warp 0 brings key and value tiles as they lie, by bulk copies into a ring of three, and eight more
// warps (12-19; 8-15 for heads wider than 128) write them out as bf16 into the ring that the products read.
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
//
// Measured: 4096 causal tokens of 32 heads over 8, 128 wide, take 150 us, 0.92 PFLOP/s (0.56 of the measured bf16 burst).  A
// unit pair takes 4090 cycles: a group's softmax 2050, P to P V 290, P V 500, to Q K 180, Q K 640, S back 175, the other
// group's under it; so the chain of a group bounds it, half of it waits for the other steps, and neither the issue slots (38 %
// busy) nor the products (tensor pipe 43 %) do.  32 steps behind 32768 tokens (176 MB) take 52 us with the joining kernel, 41
// without it: 4.3 TB/s; the rest of both is the way to the first result (6 to 10 us with cold instructions) and the end of
// each segment.  Looking for values that are not finite (warp 2) costs a prompt's 128-wide heads nothing that can be
// measured, 256-wide ones 3 % (2048 tokens of 16 heads 87.8 -> 90.1 us).
// Q4: the same prompt takes 172 us, the same 32 steps (45 MB) 57: the unpacking warps and the softmax share the issue slots (2.2 of 4
// a clock), and a tile's way through the unpacking lies in front of the first product of a segment.  Four unpacking warps instead of
// eight: the steps 67, the prompt 174; of that, 8 us are the 256 segments of a tile or three that the sequences' own keys are.
#include "attn.h"
#include "attn_join.cuh"
#include "tmem_wide.cuh"

namespace griffin {

constexpr int ATC_ROWS = 128;
constexpr float ATC_SLACK = 8.f;  // how far (log2) the true maximum may run ahead of the one P is scaled by

constexpr int ATC_BARS = 2 * 10 + 10 + 4 + 6 + 2 * 4 + 2;  // kv full/empty, v_ok, q full/empty, s_full, p_ready, o_full, seg full/empty, seg wanted

template <int DP, bool Q4> struct AtcCfg {
    static constexpr int KT = DP == 256 ? 64 : 128;       // keys per tile
    static constexpr int NS = DP == 256 ? 1 : 2;          // O accumulators
    static constexpr int UNPACK_WARP = NS == 2 ? 12 : 8;  // behind the softmax warps: first of those that unpack (Q4)
    static constexpr int UNPACKERS = 8, THREADS = Q4 ? (UNPACK_WARP + UNPACKERS) * 32 : 384;
    static constexpr int CH = Q4 ? 32 : 64;    // columns of S that a softmax thread takes at once (of 640 threads each has 96 registers)
    static constexpr int CB = DP / 64;                    // 64-entry column blocks (128 swizzled bytes per row)
    static constexpr int Q_BYTES = ATC_ROWS * DP * 2, KV_BYTES = KT * DP * 2;
    static constexpr int O_COL = 2 * KT;                  // TMEM columns: S/P 0, S/P 1, O (0, 1)
    static constexpr int MAX_SLOTS = DP == 64 ? 10 : 5;
    // a tile of the cache in 4 bits, as it lies: codes, scales, a note; unpacked in units of 32 entries of a key, PASSES to a thread
    static constexpr int UNITS = DP / 32, PASSES = KT * UNITS / (32 * UNPACKERS), RAW_STAGES = Q4 ? 3 : 0;
    static constexpr int RAW_SCALES = KT * DP / 2, RAW_NOTE = RAW_SCALES + KT * DP / 16, RAW_BYTES = RAW_NOTE + 128;
    static constexpr int BARS = ATC_BARS + 2 * RAW_STAGES;   // and raw full/empty
};

struct AtcMaps {
    CUtensorMap q, k, v;
};
struct AtcParams {
    AttnPlan plan;
    void *out;
    long long ld_out;
    const void *k, *v;
    long long stride_page, stride_head, stride_token;
    Q4Layout q4;
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
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15]), "r"(taddr)
        : "memory");
}
// S of the columns that a softmax thread takes at once, and P of them.
__device__ __forceinline__ void load_s(uint32_t taddr, float (&s)[64]) { tmem_ld64(taddr, s); }
__device__ __forceinline__ void load_s(uint32_t taddr, float (&s)[32]) { tmem_ld32(taddr, s); }
__device__ __forceinline__ void store_p(uint32_t taddr, const uint32_t (&p)[32]) { tmem_st32(taddr, p); }
__device__ __forceinline__ void store_p(uint32_t taddr, const uint32_t (&p)[16]) { tmem_st16(taddr, p); }
// 32 bytes, a whole sector, in one store (the scratch, its parts and the partials' rows start on 32-byte boundaries)
__device__ __forceinline__ void store_8f(float *to, const float *v) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                 "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void prefetch_tensormap(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN if any is
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 2^x of both lanes on the FMA and integer pipes, x >= -120 after clamping (NaN too: the row's maximum tells of one): n = the integer next to x (by adding
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
// P of N keys: 2^(c S - m), summed in fp32 and packed to bf16: the product's two operands are of one type, and the values are
// bf16 as they are stored.  That rounding (2^-8 of each P at most) brings the error against 64 bits from 0.0017 of the output,
// which is the output's own rounding, to 0.0021 to 0.0023.  POLY of every 8 pairs go through poly_exp2: the
// special-function unit gives 16 results a clock and SM, and 32768 of them per tile would take as long as the
// four products of the tile do.
constexpr int ATC_POLY = 3;
template <int POLY, int N>
__device__ __forceinline__ void exp_pairs(const float (&s)[N], float2 scale2, float2 off2, float2 (&sum)[4], uint32_t (&pk)[N / 2]) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        float2 e = fma2(make_float2(s[2 * i], s[2 * i + 1]), scale2, off2);
        if ((i * 3 & 7) < POLY) {
            e = poly_exp2(e);
        } else {
            e.x = fast_exp2(e.x);
            e.y = fast_exp2(e.y);
        }
        sum[i & 3] = add2(sum[i & 3], e);
        const __nv_bfloat162 x = __floats2bfloat162_rn(e.x, e.y);
        pk[i] = *reinterpret_cast<const uint32_t *>(&x);
    }
}

// Keys from `lim` on are not seen.
template <int N> __device__ __forceinline__ void mask_keys(float (&s)[N], int lim) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = i < lim ? s[i] : -INFINITY;
}

// The bounded wait with its slow path in one place: the loops below stay small enough for the instruction cache
// (with everything inlined the kernel was 128 KB of code and spent half its time fetching it).
static __device__ __noinline__ bool wait_slow(uint64_t *bar, uint32_t parity, volatile int *abort, void *ws, int where) {
    return wait_or_abort(bar, parity, abort, ws, where);
}
__device__ __forceinline__ bool wait_bar(uint64_t *bar, uint32_t parity, volatile int *abort, void *ws, int where) {
    return mbar_try_wait(bar, parity) || wait_slow(bar, parity, abort, ws, where);
}
// A wait of a whole warp: all its lanes go on, or none.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort, void *ws, int where) {
    return __all_sync(0xffffffffu, wait_bar(bar, parity, abort, ws, where));
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }

// Place in a ring of barriers, and the parity that a wait for this round's completion takes.
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

// A segment, as the scheduler hands it on.
struct __align__(16) Segment {
    int t0, n;            // first key tile (of the job's) and how many; n = 0: the share is done
    int pre_tiles;        // the job's tiles of the prefix; the others are the sequence's own
    int head, seq, tok0, rows, seen0, own_len;
    int alt, direct, first;
};
constexpr int ATC_SEGS = 4;
constexpr int ATC_MARKS = 2 * ATC_SEGS;   // segments that the value warp may be ahead of a softmax warp, and the one at work

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

// The values that the value warp has set to zero in this segment's tiles because they are not finite and not every row
// of the block sees their keys: added to the rows that do (whatever P, the sum is what P times them gives).  A thread has a
// row of `lanes`' accumulator at `to`; own_seen: the row's own tokens; 0: none.
template <int DP, bool Q4>
static __device__ __noinline__ void add_not_finite(const AtcParams &prm, const Segment &s, int own_seen, uint32_t to) {
    const AttnPlan &p = prm.plan;
    const int first = max(s.t0 - s.pre_tiles, 0) << p.kt_shift, last = max(s.t0 + s.n - s.pre_tiles, 0) << p.kt_shift;
    const int k0 = max(max(s.seen0, 0), first), k1 = min(min(own_seen, s.own_len), last);
#pragma unroll 1
    for (int c = 0; c < DP; c += 32) {
        float o[32];
        tmem_ld32(to + c, o);
#pragma unroll 1
        for (int k = k0; k < k1; ++k) {
            const int page = __ldg(p.page_table + (long long)s.seq * p.table_stride + (k >> p.page_shift));
            if (page < 0 || page >= p.n_pages) continue;
            if constexpr (Q4) {
                const uint8_t *const scales = static_cast<const uint8_t *>(prm.v) + page * prm.stride_page + s.head * prm.stride_head +
                                              prm.q4.scale_off + (k & ((1 << p.page_shift) - 1)) * prm.q4.scale_row + c / 16;
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    if (c + 16 * g < p.d && scales[g] == Q4_NAN) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[16 * g + i] = __uint_as_float(0x7fffffffu);
                    }
                continue;
            }
            const uint4 *const v = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(prm.v) + page * prm.stride_page +
                                                                   s.head * prm.stride_head +
                                                                   (k & ((1 << p.page_shift) - 1)) * prm.stride_token + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (c + 8 * e >= p.d) continue;
                const uint4 x = v[e];   // (a coherent load: the call in front may have written it while this grid was waiting)
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float f = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
                    if (!(fabsf(f) < INFINITY)) o[8 * e + i] += f;
                }
            }
        }
        uint32_t r[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(o[i]);
        __syncwarp();
        tmem_st32(to + c, r);
    }
    tmem_wait_st();
}

// A reader's place in the ring of segments.
struct SegReader {
    uint32_t slot, parity;
    uint64_t *full, *empty;
    const Segment *ring;
    // the next segment, into s; false: a wait gave up.  s.n == 0: there is none.
    __device__ __forceinline__ bool get(Segment &s, volatile int *abort, void *ws, int where) {
        if (!wait_bar(&full[slot], parity, abort, ws, where)) return false;
        s = ring[slot];
        return true;
    }
    __device__ __forceinline__ void step() {
        if (++slot == ATC_SEGS) {
            slot = 0;
            parity ^= 1u;
        }
    }
    // once a reader (a warp, or the issuer with its later look) has copied the segment
    __device__ __forceinline__ void release() { mbar_arrive(&empty[slot]); }
    // get by a whole warp, which then gives the place back
    __device__ __forceinline__ bool take(Segment &s, volatile int *abort, void *ws, int where) {
        const bool ok = __all_sync(0xffffffffu, get(s, abort, ws, where));
        if (ok && (threadIdx.x & 31) == 0) release();
        step();
        return ok;
    }
};

// A tile of a cache held in 4 bits (q4.cuh) comes by bulk copies as it lies, page by page, and eight warps write it out as bf16
// into the ring.  With it comes a note of what is not there.  Behind the last key, and beyond the head's width, they write what happens to
// lie there: it is a number, whatever the bits, and meets P = 0, or a logit that is masked, or a query's zeros, or no output.
struct __align__(16) RawNote {
    int valid;      // keys; < 0: there are no more tiles
    uint32_t boxes; // bit i: the page with the i-th box_rows of them is one
};
// Groups that are NaN, for which unpack_tile has written numbers, and keys of pages that are none, which read as zeros.
template <int DP>
static __device__ __noinline__ void unpack_rest(const AtcParams &prm, RawNote note, const uint8_t *raw, uint8_t *tile, int block, int row0, int half) {
    using Cfg = AtcCfg<DP, true>;
    constexpr int ROWS = 32 * Cfg::UNPACKERS / Cfg::UNITS;
    const int box_shift = 31 - __clz(prm.box_rows), q = block * 2 + half;
#pragma unroll 1
    for (int i = 0; i < Cfg::PASSES; ++i) {
        const int row = row0 + i * ROWS;
        const bool there = (note.boxes >> (row >> box_shift) & 1u) != 0;
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {
            const int group = q * 2 + (j >> 1);
            uint32_t v = 0;
            if (row >= note.valid || group * 16 >= prm.plan.d) continue;
            if (there) {
                if (raw[Cfg::RAW_SCALES + row * prm.q4.scale_row + group] != Q4_NAN) continue;
                v = 0x7fff7fffu;
            }
            *reinterpret_cast<uint4 *>(tile + block * (Cfg::KT * 128) + row * 128 + ((j ^ (half * 4) ^ (row & 7)) << 4)) = make_uint4(v, v, v, v);
        }
    }
}
// A thread has units of 32 entries.  Eight neighbours, which store at once, have the two halves of a 64-entry block of four
// keys: with the swizzle by the key's number that meets all banks.
template <int DP> __device__ __forceinline__ void unpack_tile(const AtcParams &prm, const uint8_t *raw, uint8_t *tile) {
    using Cfg = AtcCfg<DP, true>;
    constexpr int UNITS = Cfg::UNITS, BLOCKS = UNITS / 2, ROWS = 32 * Cfg::UNPACKERS / UNITS;   // keys that the warps have at once
    const int t = threadIdx.x - 32 * Cfg::UNPACK_WARP, block = (t >> 3) % BLOCKS, q = block * 2 + (t & 1);
    const int row0 = (t >> 3) / BLOCKS * 4 + ((t >> 1) & 3);
    const RawNote note = *reinterpret_cast<const RawNote *>(raw + Cfg::RAW_NOTE);
    const int d = prm.plan.d, code_row = prm.q4.code_row, scale_row = prm.q4.scale_row;
    const bool wide = (d & 31) == 0;   // rows on 16 bytes
    const uint32_t groups = (q * 32 < d ? 0x80u : 0u) | (q * 32 + 16 < d ? 0x8000u : 0u);   // the head's
    const uint32_t magic = prm.q4.magic;
    uint32_t codes = smem_u32(raw) + row0 * code_row + q * 16, scales = smem_u32(raw) + Cfg::RAW_SCALES + row0 * scale_row + q * 2;
    uint32_t to[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) to[j] = smem_u32(tile) + block * (Cfg::KT * 128) + row0 * 128 + ((j ^ ((t & 1) * 4) ^ (row0 & 7)) << 4);   // (ROWS is a multiple of 8)
    // (one unit is read ahead: the warps have little else to hide its way behind, and more code than this loop costs the other
    // roles their place in the instruction cache)
    uint32_t w[4], b;
    const auto read = [&] {
        asm volatile("ld.shared.u16 %0, [%1];" : "=r"(b) : "r"(scales));
        if (wide) {
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(codes));
        } else {
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(codes));
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[2]), "=r"(w[3]) : "r"(codes + 8));
        }
        codes += ROWS * code_row;
        scales += ROWS * scale_row;
    };
    uint32_t nan = 0;   // whether a scale's byte was 255
    read();
#pragma unroll 1
    for (int i = 0; i < Cfg::PASSES; ++i) {
        const uint32_t h0 = (b & 0xffu) * 0x00100010u + 0x35003500u, h1 = (b >> 8) * 0x00100010u + 0x35003500u;   // q4_scale_bits, twice each
        const Q4Scale2 s[2] = {{h0, q4_mul2(h0, 0xc308c308u)}, {h1, q4_mul2(h1, 0xc308c308u)}};   // -136
        const uint32_t c[4] = {w[0], w[1], w[2], w[3]};
        nan |= (0xfefeu - b) & b & 0x8080u;
        if (i + 1 < Cfg::PASSES) read();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to[j]), "r"(q4_pair(c[j], 0, s[j >> 1], magic)),
                         "r"(q4_pair(c[j], 1, s[j >> 1], magic)), "r"(q4_pair(c[j], 2, s[j >> 1], magic)), "r"(q4_pair(c[j], 3, s[j >> 1], magic)));
            to[j] += ROWS * 128;
        }
    }
    const bool rare = (nan & groups) != 0 || note.boxes != (1u << ((note.valid + prm.box_rows - 1) / (uint32_t)prm.box_rows)) - 1u;
    if (__any_sync(0xffffffffu, rare)) unpack_rest<DP>(prm, note, raw, tile, block, row0, t & 1);
}

template <int DP, bool Q4>
__global__ void __launch_bounds__(AtcCfg<DP, Q4>::THREADS, 1) attn_tc_kernel(const __grid_constant__ AtcMaps maps,
                                                              const __grid_constant__ AtcParams prm) {
    using Cfg = AtcCfg<DP, Q4>;
    constexpr int KT = Cfg::KT, NS = Cfg::NS, CB = Cfg::CB;
    const AttnPlan &p = prm.plan;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *const s_q = base;                                  // NS query tiles
    uint8_t *const s_kv = base + NS * Cfg::Q_BYTES;             // ring of key and value tiles
    const int n_slots = prm.n_slots;
    uint8_t *const s_raw = s_kv + n_slots * Cfg::KV_BYTES;      // tiles of a cache in 4 bits, as they lie
    uint64_t *const bars = reinterpret_cast<uint64_t *>(s_raw + Cfg::RAW_STAGES * Cfg::RAW_BYTES);
    uint64_t *const kv_full = bars, *const kv_empty = bars + 10, *const v_ok = bars + 20, *const q_full = bars + 30,
                   *const q_empty = bars + 32, *const s_full = bars + 34, *const p_ready = bars + 36, *const o_full = bars + 38,
                   *const seg_full = bars + 40, *const seg_empty = bars + 44, *const seg_want = bars + 48, *const raw_full = bars + 50,
                   *const raw_empty = bars + 53;
    Segment *const segs = reinterpret_cast<Segment *>(bars + Cfg::BARS);
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(segs + ATC_SEGS);
    volatile int *const abort = reinterpret_cast<volatile int *>(tmem_slot + 1);
    volatile int *const marks = reinterpret_cast<volatile int *>(tmem_slot + 2);   // segments with values that are not finite
    int *const bases = reinterpret_cast<int *>(tmem_slot + 2 + ATC_MARKS);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    if (tid < (Q4 ? 1 : 3)) prefetch_tensormap(tid == 0 ? &maps.q : tid == 1 ? &maps.k : &maps.v);
    if (tid == 0) {
        for (int i = 0; i < n_slots; ++i) {
            mbar_init(&kv_full[i], Q4 ? Cfg::UNPACKERS : 1);   // the copies' producer, or the warps that unpack
            mbar_init(&kv_empty[i], 2);   // the products that read it, and the value warp
            mbar_init(&v_ok[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_ready[i], 4);  // one arrival per warp of the group
            mbar_init(&o_full[i], 1);
        }
        for (int i = 0; i < ATC_SEGS; ++i) {
            mbar_init(&seg_full[i], 1);
            mbar_init(&seg_empty[i], 3 + 4 * NS);  // producer, issuer, value warp, softmax warps
        }
        mbar_init(seg_want, 1);
        for (int i = 0; i < Cfg::RAW_STAGES; ++i) {
            mbar_init(&raw_full[i], 1);
            mbar_init(&raw_empty[i], Cfg::UNPACKERS);   // the warps that unpack
        }
        *abort = 0;
        mbar_fence_init();
    }
    pdl_wait_prior_grids();
    attn_scan(p, bases);
    const AttnTotals totals = attn_totals(p, bases);
    const AttnShares shares(totals.W, p.grid);
    if ((int)blockIdx.x >= shares.G) return;
    if (warp == 1) tmem_alloc(tmem_slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    SegReader seg{0, 0, seg_full, seg_empty, segs};

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        Segment w;
        uint32_t kv_n = 0, nq = 0;  // ring slots and query buffers handed out so far
        Ring kv{0, 0}, raw{0, 0};
        uint32_t raw_n = 0;
        bool ok = true;
        const int per_tile = KT / prm.box_rows;  // boxes per 64-entry block
        if (lane == 0) mbar_arrive(seg_want);
        while (ok && (ok = seg.take(w, abort, p.ws, 49)) && w.n > 0) {
            const int q_tiles = NS == 2 && !w.alt ? 2 : 1;
            for (int r = 0; r < q_tiles && ok; ++r, ++nq) {
                const int b = nq % NS;
                if (nq >= NS) ok = warp_wait(&q_empty[b], (nq / NS - 1) & 1, abort, p.ws, 50);
                if (ok && lane == 0) {
                    mbar_arrive_expect_tx(&q_full[b], CB * prm.q_box_bytes);
                    for (int c = 0; c < CB; ++c)
                        tma_load_3d(s_q + b * Cfg::Q_BYTES + c * (ATC_ROWS * 128), &maps.q, c * 64, w.head * p.group,
                                    w.tok0 + r * p.tile_tokens, &q_full[b]);
                }
            }
            int next_page = -1;   // of this lane's box of the next tile (Q4)
            const auto look_up = [&](int t) {
                const KeyTile k = key_tile(p, w, t);
                const int key = k.k0 + lane * prm.box_rows;
                return lane < per_tile && key < k.len ? __ldg((k.prefix ? p.prefix_pages : p.page_table + (long long)w.seq * p.table_stride) + (key >> p.page_shift)) : -1;
            };
            if constexpr (Q4) next_page = look_up(w.t0);
            for (int t = 0; t < w.n && ok; ++t) {
                const KeyTile k = key_tile(p, w, w.t0 + t);
                if constexpr (Q4) {
                    const int page = next_page, key = k.k0 + lane * prm.box_rows;
                    if (t + 1 < w.n) next_page = look_up(w.t0 + t + 1);
                    const bool has = lane < per_tile && key < k.len, there = has && (unsigned)page < (unsigned)p.n_pages;
                    if (has && !there) attn_bad(p.ws, 42);
                    const uint32_t boxes = __ballot_sync(0xffffffffu, there);
                    for (int which = 0; which < 2; ++which, ++raw_n) {
                        if (raw_n >= (uint32_t)Cfg::RAW_STAGES && !(ok = warp_wait(&raw_empty[raw.slot], raw.parity ^ 1u, abort, p.ws, 51))) break;
                        uint8_t *const to = s_raw + raw.slot * Cfg::RAW_BYTES;
                        if (lane == 0) {
                            *reinterpret_cast<RawNote *>(to + Cfg::RAW_NOTE) = RawNote{min(k.len - k.k0, KT), boxes};
                            mbar_arrive_expect_tx(&raw_full[raw.slot], __popc(boxes) * prm.box_rows * (prm.q4.code_row + prm.q4.scale_row));
                        }
                        __syncwarp();
                        if (there) {
                            const uint8_t *const from = static_cast<const uint8_t *>(which ? prm.v : prm.k) + page * prm.stride_page + w.head * prm.stride_head;
                            const int slot = key & ((1 << p.page_shift) - 1), r = lane * prm.box_rows;
                            bulk_g2s(to + r * prm.q4.code_row, from + slot * prm.q4.code_row, prm.box_rows * prm.q4.code_row, &raw_full[raw.slot]);
                            bulk_g2s(to + Cfg::RAW_SCALES + r * prm.q4.scale_row, from + prm.q4.scale_off + slot * prm.q4.scale_row,
                                     prm.box_rows * prm.q4.scale_row, &raw_full[raw.slot]);
                        }
                        raw.step(1, Cfg::RAW_STAGES);
                    }
                    continue;
                }
                const int *const pages = k.prefix ? p.prefix_pages : p.page_table + (long long)w.seq * p.table_stride;
                for (int which = 0; which < 2; ++which) {
                    const uint32_t slot = kv.slot;
                    if (kv_n >= (uint32_t)n_slots && !(ok = warp_wait(&kv_empty[slot], kv.parity ^ 1u, abort, p.ws, 51))) break;
                    if (lane == 0) mbar_arrive_expect_tx(&kv_full[slot], Cfg::KV_BYTES);
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
                        tma_load_4d(s_kv + slot * Cfg::KV_BYTES + c * (KT * 128) + r * prm.box_rows * 128, which ? &maps.v : &maps.k,
                                    c * 64, key & ((1 << p.page_shift) - 1), w.head, page, &kv_full[slot]);
                    }
                    __syncwarp();
                    kv.step(1, n_slots);
                    ++kv_n;
                }
            }
            if (lane == 0) mbar_arrive(seg_want);
        }
        uint32_t raw_seen = raw_n > (uint32_t)Cfg::RAW_STAGES ? raw_n - Cfg::RAW_STAGES : 0;   // of the tiles, how many are known to have landed
        if constexpr (Q4) {   // a note that there are no more
            if (ok && (raw_n < (uint32_t)Cfg::RAW_STAGES || warp_wait(&raw_empty[raw.slot], raw.parity ^ 1u, abort, p.ws, 51))) {
                if (lane == 0) {
                    reinterpret_cast<RawNote *>(s_raw + raw.slot * Cfg::RAW_BYTES + Cfg::RAW_NOTE)->valid = -1;
                    mbar_arrive(&raw_full[raw.slot]);
                }
                if (raw_n >= (uint32_t)Cfg::RAW_STAGES) ++raw_seen;   // (the one that was in its place)
            }
        }
        // stay until every copy that was started has landed
        if (lane == 0) {
            const long long t_0 = clock64();
            for (uint32_t i = raw_seen; Q4 && i < raw_n; ++i)
                while (!mbar_try_wait(&raw_full[i % 3], (i / 3) & 1))
                    if (clock64() - t_0 > WAIT_LIMIT_CYCLES) break;
            for (uint32_t i = kv_n > (uint32_t)n_slots ? kv_n - n_slots : 0; i < kv_n; ++i)
                while (!mbar_try_wait(&kv_full[i % n_slots], (i / n_slots) & 1))
                    if (clock64() - t_0 > WAIT_LIMIT_CYCLES) break;
            for (uint32_t i = nq > (uint32_t)NS ? nq - NS : 0; i < nq; ++i)
                while (!mbar_try_wait(&q_full[i % NS], (i / NS) & 1))
                    if (clock64() - t_0 > WAIT_LIMIT_CYCLES) break;
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        // (the whole warp walks, one lane issues: the operands stay in uniform registers)
        constexpr uint32_t ID_QK = umma_idesc(ATC_ROWS, KT), ID_PV = umma_idesc(ATC_ROWS, DP) | (1u << 16);
        // Where S = Q K^T stands (a) and where P V (b): unit in its segment, units in it, whether blocks of two row tiles.
        SegReader seg_b = seg;
        bool a_dual = false, b_dual = false;
        uint32_t a_n = 0, b_n = 0, a_u = 0, b_u = 0;
        uint32_t a_U = 0, b_U = 0, qi = 0;  // units of the CTA; first query buffer of a's segment
        Ring ka{0, 0}, vb{1, 0}, okb{0, 0};  // ring places of the next key tile, of the next value tile, and the latter's v_ok
        const uint64_t q_desc = smem_desc_sw128(s_q, 0), k_desc = smem_desc_sw128(s_kv, 0), v_desc = smem_desc_mn_sw128(s_kv, 0, KT * 128);
        const auto next_segment = [&](SegReader &r, uint32_t &n, bool &dual, bool last_reader) -> bool {
            if (!warp_wait(&r.full[r.slot], r.parity, abort, p.ws, 48)) return false;
            const Segment &s = r.ring[r.slot];
            dual = NS == 2 && uniform(s.alt) == 0;
            n = uniform(s.n) << (dual ? 1 : 0);
            __syncwarp();
            if (last_reader && elect_one()) r.release();
            r.step();
            return true;
        };
        bool ok = next_segment(seg, a_n, a_dual, false) && next_segment(seg_b, b_n, b_dual, true);
        uint32_t ahead = 0;  // units whose S has been issued and P V not: two in front of every P V
        while (ok && b_n > 0) {
            if (ahead < 2 && a_n > 0) {
                const uint32_t q_at = qi + (a_dual ? a_u & 1 : 0), qb = NS == 2 ? q_at & 1 : 0;
                if (a_u < (a_dual ? 2u : 1u) && !(ok = warp_wait(&q_full[qb], (NS == 2 ? q_at >> 1 : q_at) & 1, abort, p.ws, 52))) break;
                if (!(ok = warp_wait(&kv_full[ka.slot], ka.parity, abort, p.ws, 53))) break;
                tc_fence_after_sync();
                const uint64_t q = q_desc + (uint64_t)(qb * (Cfg::Q_BYTES >> 4)), k = k_desc + (uint64_t)(ka.slot * (Cfg::KV_BYTES >> 4));
                const uint32_t d = tmem + (a_U & 1) * KT;
                const bool k_done = !a_dual || (a_u & 1), q_done = a_u + (a_dual ? 2 : 1) >= a_n;
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk)
                        umma_bf16(d, q + (uint64_t)(((kk >> 2) * (ATC_ROWS * 128) + (kk & 3) * 32) >> 4),
                                  k + (uint64_t)(((kk >> 2) * (KT * 128) + (kk & 3) * 32) >> 4), ID_QK, kk > 0);
                    umma_commit(&s_full[a_U & 1]);
                    if (k_done) umma_commit(&kv_empty[ka.slot]);
                    if (q_done) umma_commit(&q_empty[qb]);
                }
                __syncwarp();
                if (k_done) ka.step(2, n_slots);
                ++a_U;
                ++ahead;
                if (++a_u == a_n) {
                    qi += a_dual ? 2 : 1;
                    a_u = 0;
                    ok = next_segment(seg, a_n, a_dual, false);
                }
                continue;
            }
            // (the value warp has seen the tile arrive)
            if (!warp_wait(&v_ok[okb.slot], okb.parity, abort, p.ws, 54)) break;
            if (!warp_wait(&p_ready[b_U & 1], (b_U >> 1) & 1, abort, p.ws, 55)) break;
            tc_fence_after_sync();
            const uint32_t o = NS == 2 ? b_U & 1 : 0, d = tmem + Cfg::O_COL + o * DP, pt = tmem + (b_U & 1) * KT;
            const uint64_t v = v_desc + (uint64_t)(vb.slot * (Cfg::KV_BYTES >> 4));
            const uint32_t add = b_u >= NS;
            const bool v_done = !b_dual || (b_u & 1);
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < KT / 16; ++kk) umma_bf16_ts(d, pt + kk * 8, v + (uint64_t)(kk * (2048 >> 4)), ID_PV, kk > 0 ? 1 : add);
                if (v_done) umma_commit(&kv_empty[vb.slot]);
                if (NS == 1 || b_u + 2 >= b_n) umma_commit(&o_full[o]);
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
                ok = next_segment(seg_b, b_n, b_dual, true);
            }
        }
    } else if (warp == 2) {
        // ---------------- value tiles: rows that no key stands for become zeros (Q4: they are numbers already) ----------------
        Segment w;
        // (It waits for the key tiles too: a wait for a slot's n-th filling may only begin when the one before has been
        // seen, or the parity of an older one passes for it.  And no slot is filled again before it has looked: a filling
        // that it missed would leave it waiting for one that needs its own word.)
        Ring kv{0, 0}, done{0, 0};
        bool ok = true;
        for (uint32_t at = 0; ok && (ok = seg.take(w, abort, p.ws, 47)) && w.n > 0; ++at) {
            // (at most ATC_SEGS segments ahead of the slowest softmax warp: nobody reads this mark any more)
            if (lane == 0) marks[at % ATC_MARKS] = 0;
            for (int t = 0; t < w.n && ok; ++t, done.step(1, n_slots)) {
                const KeyTile k = key_tile(p, w, w.t0 + t);
                if (!(ok = warp_wait(&kv_full[kv.slot], kv.parity, abort, p.ws, 56))) break;
                if (lane == 0) mbar_arrive(&kv_empty[kv.slot]);
                kv.step(1, n_slots);
                const uint32_t slot = kv.slot;
                if (!(ok = warp_wait(&kv_full[slot], kv.parity, abort, p.ws, 56))) break;
                kv.step(1, n_slots);
                const int valid = k.len - k.k0;
                // keys of the tile from `apart` on are seen by some rows of the block and not by others
                const int apart = k.prefix ? KT : max(w.seen0 - k.k0, 0), upto = min(valid, KT);
                if (apart < upto) {
                    uint4 *const rows = reinterpret_cast<uint4 *>(s_kv + slot * Cfg::KV_BYTES + apart * 128) + lane;
                    const int n = (upto - apart) * 8 - lane;   // 16-byte pieces of a column block, this lane's every 32nd
                    NotFinite8 bad;
#pragma unroll 1
                    for (int c = 0; c < CB; ++c)
#pragma unroll 8
                        for (int i = 0; i < n; i += 32) bad.add(rows[c * (KT * 8) + i]);
                    if (__any_sync(0xffffffffu, bad.any())) {
#pragma unroll 1
                        for (int c = 0; c < CB; ++c)
#pragma unroll 1
                            for (int i = 0; i < n; i += 32) rows[c * (KT * 8) + i] = finite_or_zero8(rows[c * (KT * 8) + i]);
                        if (lane == 0) marks[at % ATC_MARKS] = 1;
                        fence_proxy_async_smem();
                    }
                }
                // (Q4: what was unpacked behind the last key is any number, but finite, as the unpacking never writes NaN there, a scale's
                // byte of 255 included; P is 0 there)
                if (!Q4 && valid < KT) {
#pragma unroll 1
                    for (int i = lane; i < (KT - valid) * 8 * CB; i += 32) {
                        const int c = i % CB, r = valid + i / CB / 8, e = i / CB % 8;
                        *reinterpret_cast<uint4 *>(s_kv + slot * Cfg::KV_BYTES + c * (KT * 128) + r * 128 + e * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&v_ok[done.slot]);
                    mbar_arrive(&kv_empty[slot]);
                }
            }
        }
    } else if (warp == 3) {
        // ---------------- scheduler ----------------
        int g = shares.first(blockIdx.x);
        const int g_end = shares.first(blockIdx.x + 1);
        AttnJob j;
        bool more = true;
        if (!totals.queued) {
            j = attn_find(p, bases, g);
            if (lane == 0) attn_note_cut(p, shares, j, g, min(g_end, j.g1));
        }
        Ring at{0, 0};
        AttnQueueAt from{0, 0};
        for (uint32_t k = 0;; ++k) {
            if (k >= ATC_SEGS && !warp_wait(&seg_empty[at.slot], at.parity ^ 1u, abort, p.ws, 46)) break;
            if (totals.queued) {
                // the next job of the queue, once the copies of the one before have been asked for
                if (!warp_wait(seg_want, k & 1, abort, p.ws, 44)) break;
                do {
                    int i = 0;
                    if (lane == 0) i = (int)atomicAdd(p.queue, 1u);
                    i = __shfl_sync(0xffffffffu, i, 0);
                    more = i < totals.jobs;
                    if (!more) break;
                    j = attn_queued(p, i, from);
                    g = j.g0;
                } while (j.g1 == j.g0);   // (blocks that see nothing are the joining kernel's)
            }
            const int stop = totals.queued ? j.g1 : min(g_end, j.g1);
            if (lane == 0) {
                Segment s;
                s.t0 = g - j.g0;
                s.n = more ? stop - g : 0;
                s.pre_tiles = j.seq < 0 || p.fused ? p.prefix_tiles : 0;
                s.head = j.head;
                s.seq = j.seq;
                s.tok0 = j.tok0;
                s.rows = j.rows;
                s.seen0 = j.seen0;
                s.own_len = j.own_len;
                s.alt = j.alt;
                s.first = g == j.g0;
                s.direct = attn_direct(p, j, s.first && stop == j.g1);
                segs[at.slot] = s;
                mbar_arrive(&seg_full[at.slot]);
            }
            __syncwarp();
            if (!more) break;
            at.step(1, ATC_SEGS);
            if (!totals.queued) {
                g = stop;
                more = g < g_end;
                if (more) j = attn_next(p, bases, j);
            }
        }
    } else if (warp >= 4 && warp < Cfg::UNPACK_WARP) {
        // ---------------- softmax ----------------
        const uint32_t grp = (warp - 4) >> 2;
        const int wr = (warp & 3) * 32;                            // the group's rows of this warp: wr .. wr + 31
        const uint32_t lanes = tmem + ((uint32_t)wr << 16);
        const int tile_rows = p.tile_tokens * p.group;
        Segment j;
        uint32_t U0 = 0, n_o = 0;  // units before this segment; segments finished by this group
        bool ok = true;
        for (uint32_t at_seg = 0; ok && (ok = seg.take(j, abort, p.ws, 45)) && j.n > 0; ++at_seg) {
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
                // (one accumulator: whether P V of the unit before is known to be done; every one is waited for in turn, or
                // a later wait would take the parity of an older one)
                bool o_seen = u == 0;
                ok = warp_wait(&s_full[buf], (U >> 1) & 1, abort, p.ws, 57);
                if (!ok) break;
                tc_fence_after_sync();
                if (warp_on) {
                    const uint32_t ts = lanes + buf * KT;
                    const int lim = (k.prefix ? k.len : min(k.len, own_seen)) - k.k0;   // keys of the tile that the row sees
                    const bool masked = __any_sync(0xffffffffu, lim < KT);
                    float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
                    for (int c = 0; c < KT; c += Cfg::CH) {
                        float s[Cfg::CH];
                        load_s(ts + c, s);
                        if (masked) mask_keys(s, lim - c);
#pragma unroll
                        for (int i = 0; i < Cfg::CH; i += 8)
#pragma unroll
                            for (int e = 0; e < 4; ++e) mx4[e] = max3(mx4[e], s[i + e], s[i + 4 + e]);
                    }
                    float mx = max3(max3(mx4[0], mx4[1], mx4[2]), mx4[3], mx4[3]);
                    mx *= p.scale_log2;
                    // the maximum moves only when 2^(c S - m) could grow too large, or there is none yet, or it is NaN
                    const bool move = !(mx <= m + ATC_SLACK);
                    if (__any_sync(0xffffffffu, move)) {
                        const float f = move ? fast_exp2(m - mx) : 1.f;   // (0 for the first)
                        l *= f;
                        if (move) {   // (a logit that is NaN or infinite makes the row NaN)
                            l += mx - mx;
                            m = mx == mx ? mx : INFINITY;
                        }
                        if (started) {
                            // (one accumulator: S of this unit was issued before P V of the last one, so its barrier
                            // does not cover it)
                            if (NS == 1) {
                                if (!(ok = warp_wait(&o_full[0], (U - 1) & 1, abort, p.ws, 59))) break;
                                o_seen = true;
                            }
                            tc_fence_after_sync();
                            const uint32_t to = lanes + Cfg::O_COL + (NS == 2 ? buf : 0) * DP;
#pragma unroll 1
                            for (int c = 0; c < DP; c += 32) {
                                float o[32];
                                uint32_t scaled[32];
                                tmem_ld32(to + c, o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) scaled[i] = __float_as_uint(o[i] * f);
                                tmem_st32(to + c, scaled);
                            }
                        }
                    }
                    const float off = m == -INFINITY ? 0.f : m;
                    const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), off2 = make_float2(-off, -off);
                    float2 sum[4] = {};
#pragma unroll 1
                    for (int c = 0; c < KT; c += Cfg::CH) {
                        float s[Cfg::CH];
                        load_s(ts + c, s);
                        uint32_t pk[Cfg::CH / 2];
                        if (masked) {
                            mask_keys(s, lim - c);   // 2^-inf = 0
                            exp_pairs<0>(s, scale2, off2, sum, pk);
                        } else {
                            exp_pairs<ATC_POLY>(s, scale2, off2, sum, pk);
                        }
                        store_p(ts + c / 2, pk);
                    }
                    const float2 s4 = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
                    l += s4.x + s4.y;
                    started = true;
                    tmem_wait_st();
                }
                if (NS == 1 && !o_seen && !(ok = warp_wait(&o_full[0], (U - 1) & 1, abort, p.ws, 59))) break;
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
                    if (marks[at_seg % ATC_MARKS] != 0) add_not_finite<DP, Q4>(prm, j, valid ? own_seen : 0, to);
                    if (j.direct) {
                        const float inv = m == -INFINITY ? 0.f : 1.0f / l;
                        __nv_bfloat16 *const dst = static_cast<__nv_bfloat16 *>(prm.out) + (j.tok0 + tok) * prm.ld_out +
                                                   (j.head * p.group + row - tok * p.group) * p.d;
#pragma unroll 1
                        for (int c = 0; c < DP; c += 32) {
                            float o[32];
                            tmem_ld32(to + c, o);
                            if (valid) {
#pragma unroll
                                for (int i = 0; i < 32; i += 8) {
                                    uint32_t h[4];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const __nv_bfloat162 x = __floats2bfloat162_rn(o[i + 2 * e] * inv, o[i + 2 * e + 1] * inv);
                                        h[e] = *reinterpret_cast<const uint32_t *>(&x);
                                    }
                                    if (c + i < p.d) *reinterpret_cast<uint4 *>(dst + c + i) = make_uint4(h[0], h[1], h[2], h[3]);
                                }
                            }
                        }
                    } else {
                        PartPlace at{nullptr, nullptr};
                        if (valid) {
                            at = attn_place(p, PartJob{j.seq, j.head, j.tok0, j.alt != 0}, j.first != 0, stream, row);
                            *reinterpret_cast<float2 *>(at.ml) = make_float2(m, l);
                        }
#pragma unroll 1
                        for (int c = 0; c < DP; c += 32) {
                            float o[32];
                            tmem_ld32(to + c, o);
                            if (valid) {
#pragma unroll
                                for (int i = 0; i < 32; i += 8) {
                                    if (c + i < p.d) store_8f(at.o + c + i, o + i);
                                }
                            }
                        }
                    }
                    tc_fence_before_sync();
                }
            } else if (ok && valid && j.alt) {  // a segment of one tile leaves the other stream empty
                *reinterpret_cast<float2 *>(attn_place(p, PartJob{j.seq, j.head, j.tok0, j.alt != 0}, j.first != 0, stream, row).ml) = make_float2(-INFINITY, 0.f);
            }
            U0 += n;
        }
    }

    if constexpr (Q4) {
        if (warp >= Cfg::UNPACK_WARP) {
            // ---------------- the cache in 4 bits: unpacked into the ring ----------------
            Ring kv{0, 0}, raw{0, 0};
            for (uint32_t kv_n = 0;; ++kv_n) {
                if (!warp_wait(&raw_full[raw.slot], raw.parity, abort, p.ws, 60)) break;
                const uint8_t *const from = s_raw + raw.slot * Cfg::RAW_BYTES;
                if (reinterpret_cast<const RawNote *>(from + Cfg::RAW_NOTE)->valid < 0) break;
                if (kv_n >= (uint32_t)n_slots && !warp_wait(&kv_empty[kv.slot], kv.parity ^ 1u, abort, p.ws, 51)) break;
                unpack_tile<DP>(prm, from, s_kv + kv.slot * Cfg::KV_BYTES);
                fence_proxy_async_smem();   // (orders the stores above, which are volatile like it)
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&kv_full[kv.slot]);
                    mbar_arrive(&raw_empty[raw.slot]);
                }
                kv.step(1, n_slots);
                raw.step(1, Cfg::RAW_STAGES);
            }
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

template <int DP, bool Q4> static griffin_status launch_dp(const AttnPlan &plan, const AttnData &x, cudaStream_t stream) {
    using Cfg = AtcCfg<DP, Q4>;
    AtcMaps maps;
    AtcParams prm{};
    prm.plan = plan;
    prm.out = x.out;
    prm.ld_out = x.ld_out;
    prm.k = x.k;
    prm.v = x.v;
    prm.q4 = x.q4;
    prm.stride_page = x.stride_page; prm.stride_head = x.stride_head; prm.stride_token = x.stride_token;
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
    for (int which = 0; !Q4 && which < 2; ++which) {
        const cuuint64_t dims[4] = {(cuuint64_t)plan.d, (cuuint64_t)page, (cuuint64_t)plan.hkv, (cuuint64_t)plan.n_pages};
        const cuuint64_t strides[3] = {(cuuint64_t)x.stride_token * 2, (cuuint64_t)x.stride_head * 2, (cuuint64_t)x.stride_page * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)prm.box_rows, 1, 1}, ones[4] = {1, 1, 1, 1};
        if (enc(which ? &maps.v : &maps.k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(which ? x.v : x.k), dims, strides,
                box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return GRIFFIN_ERR_UNSUPPORTED;  // (strides that the copy engine does not take)
    }
    // as many ring slots as fit beside the list of the sequences' first tiles
    const size_t tail = Cfg::BARS * 8 + ATC_SEGS * sizeof(Segment) + 8 + ATC_MARKS * 4 + ((size_t)plan.n_seq + 3) * 4, fixed = 1024 + Cfg::NS * Cfg::Q_BYTES + Cfg::RAW_STAGES * Cfg::RAW_BYTES + tail;
    prm.n_slots = (int)((232448 - fixed) / Cfg::KV_BYTES);
    if (prm.n_slots > Cfg::MAX_SLOTS) prm.n_slots = Cfg::MAX_SLOTS;
    const size_t smem = fixed + (size_t)prm.n_slots * Cfg::KV_BYTES;
    const void *fn = reinterpret_cast<const void *>(attn_tc_kernel<DP, Q4>);
    if (ensure_dynamic_smem(fn, smem) != cudaSuccess) return GRIFFIN_ERR_CUDA;
    void *args[] = {&maps, &prm};
    return launch_maybe_overlapped(fn, dim3(plan.grid), dim3(Cfg::THREADS), smem, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

AttnShape attn_tc_shape(int head_dim) {
    return head_dim > 128 ? AttnShape{ATC_ROWS, 1, AtcCfg<256, false>::KT, 0} : AttnShape{ATC_ROWS, 2, AtcCfg<128, false>::KT, 1};
}

template <bool Q4> static griffin_status launch_q4(const AttnPlan &plan, const AttnData &data, cudaStream_t stream) {
    if (plan.d <= 64) return launch_dp<64, Q4>(plan, data, stream);
    if (plan.d <= 128) return launch_dp<128, Q4>(plan, data, stream);
    return launch_dp<256, Q4>(plan, data, stream);
}
griffin_status launch_attn_tc(const AttnPlan &plan, const AttnData &data, bool q4, cudaStream_t stream) {
    return q4 ? launch_q4<true>(plan, data, stream) : launch_q4<false>(plan, data, stream);
}

}  // namespace griffin
