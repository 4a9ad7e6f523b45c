// Attention over a cache held in 4 bits (q4.cuh), bf16 or fp32 queries, blocks of up to 8 query rows.  The mathematics is attn_few.cu's:
// S^T = K Q^T and O^T = V^T P^T on m16n8k16, a warp with its own m, l and O.
//
// The keys are unpacked between shared memory and the matrix instruction: codes become bf16 values, exactly, with a
// shift, a logical operation and an fma for two of them, so nothing but the codes is ever written anywhere.
//   K: the order of the entries in a product is free, so lane t of four takes the t-th quarter of a key's codes as they lie,
//      and the queries are read in that order.
//   V: a register holds two keys' values of one entry, the lower halves of the two keys' words put side by side (entries 2i of
//      a word are in its lower half, 2i + 1 in the upper); lane / 4 has an eighth of the entries.
// Key r of eight is row 2 (r mod 4) + r / 4 of the products (fq_row): so the keys whose values four lanes load at once lie
// side by side, and with their pieces turned (fq_turn) on different banks.
//
// The CTA's share of the call's tiles, of 32 keys here (attn_plan.cuh), is dealt out evenly to its warps, and each works its
// own off by itself: it brings the keys by cp.async through a ring of two buffers, from segment to segment without a pause.  No barrier is
// met but one at the end, behind which the pieces of jobs that went to several warps are put together, and one partial of
// a job is left to the joining kernel at most.  (Sixteen warps that worked on one segment together, as in attn_few.cu, spent as
// long on its end as on 512 keys: 256 sequences of 512 keys under 8 heads 140 us, 48 of 2560 61.  Warps that each left their
// partials to the joining kernel gave it 148 a row: 4 tokens behind 9000 keys, 8 heads, 104 us.)  The loads' addresses, the pages,
// the walk and the look for a new maximum (which is not exchanged while the sums, in fp32, stay below 2^8) cost as much
// as the products for 16 keys, so a warp takes 32 at a time.  What bounds it are the instructions: of 4 issue slots a clock 2.30
// are used, the integer pipe for 56 % of the time, the matrix pipe for 21 %, and with three warps to a scheduler their fixed latencies
// (1.1 warps at an issue) and the integer pipe (0.75) are what the rest waits for, not memory (0.2 each for device and shared memory): 16 sequences of 4096 keys under
// 32 heads of their own.  (With 16 warps, which spilled, it was 2.35, 58 % and 20 %.)
//
// With few jobs (attn_whole, attn.cu) a cluster of 1, 2, 4 or 8 CTAs takes a job whole instead: the CTAs' sums meet in distributed
// shared memory, each adds up and stores its share of the entries, and there is no second launch.
//
// Measured: 48 sequences of 1024 to 4096 keys, 32 heads over 8, 128 wide (154 MB of codes and scales), 51.2 us, 3.0 TB/s, with
// the joining kernel (from the cache in bf16, 547 MB, 95), all of 4096 (227 MB) 64.9 (139); 1 sequence of 32 heads behind 512
// tokens 8.0, of which 2 are the launch; 8 sequences of 40 heads behind 2048 21.0.
// fp32 calls run on the same instruction: keys and values are exact in bf16, a query's entry and P are sums of three bf16 numbers, so
// three products of each kind replace one; the unpacking is shared.  Prompts too: 1000 causal tokens of 8 heads of 64 41 us (over the
// cache in fp32 72), 2048 of 32 over 8, 128 wide, 590 (1409), 64 behind 4096 69 (194).
#include "attn.h"
#include "attn_join.cuh"
#include "decode_mma.cuh"

namespace griffin {

constexpr int FQ_ROWS = 8, FQ_KEYS = 32;  // query rows of a block; keys of a tile
constexpr float FQ_SLACK = 8.f;  // how far (log2) the true maximum may run ahead of the one P is scaled by

// DP: the head's width rounded up to 64, 128 or 256.  T: of queries and output.
template <int DP, typename T> struct FqCfg {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int PARTS = F32 ? 3 : 1;   // bf16 numbers that a query's entry, or P, is the sum of
    // (as many warps as have the registers that the kernel wants in bf16: 16 of 128-wide bf16 spill 104 bytes, 48 sequences of 4096 keys
    // each 67.6 us, 12 64.2, 8 69.4, and 1 sequence behind 512 tokens 9.9, 8.1, 7.9; 256 wide 8 warps 119, 6 146; 3 stages no faster.  256-wide
    // fp32 spills 64 to 80 bytes at 255 registers, bf16 of 80 to 112 entries 4)
    static constexpr int WARPS = DP == 256 || (F32 && DP == 128) ? 8 : 12, THREADS = 32 * WARPS, STAGES = 2;
    // rows of codes and scales in shared memory
    static constexpr int KROW = DP == 256 ? 144 : DP / 2, VROW = DP / 2, SROW = DP / 16;
    static constexpr int V_AT = FQ_KEYS * KROW, KS_AT = V_AT + FQ_KEYS * VROW, VS_AT = KS_AT + FQ_KEYS * SROW, STAGE = VS_AT + FQ_KEYS * SROW;
    // A warp's pieces of jobs that it shares with others, row by row: m and l of the rows, then the results.  That of its first
    // segment has room of its own, that of its last one lies in the ring.
    static constexpr int LDO = DP + 4, PIECE = FQ_ROWS * (LDO + 2) * 4;
    static constexpr int PIECES_AT = WARPS * STAGES * STAGE, SEGS_AT = PIECES_AT + WARPS * PIECE;
    static_assert(PIECE <= STAGES * STAGE && PIECE % 16 == 0 && STAGE % 128 == 0, "");
    static size_t smem(int n_seq);
};
// Row of the products for key r of eight, and the key for row g.
__device__ __forceinline__ int fq_row(int r) { return (r & 3) * 2 + (r >> 2); }
__device__ __forceinline__ int fq_key(int g) { return (g >> 1) + (g & 1) * 4; }
// By what the 16-byte pieces of key r's values are turned (xor): the eight-byte (128 wide) or 16-byte (256 wide) loads of keys
// r .. r + 3 then meet all banks once.
template <int DP> __device__ __forceinline__ int fq_turn(int r) { return DP == 128 ? (r >> 1 & 1) * 2 : DP == 256 ? (r & 3) * 2 : 0; }

__device__ __forceinline__ uint32_t fq_movmatrix(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t fq_pack(float a, float b) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}
template <int BYTES> __device__ __forceinline__ void fq_copy(uint32_t dst, const void *src) {   // 4, 8 or 16
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
template <int N> __device__ __forceinline__ void fq_lds(uint32_t (&w)[N], uint32_t at) {   // N words, N = 1, 2, 4 or 8
    if constexpr (N == 1) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
    else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
    else
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3])
                         : "r"(at + 4 * i)
                         : "memory");
}
// BYTES = 1, 2 or 4 bytes, in the last bits
template <int BYTES> __device__ __forceinline__ uint32_t fq_lds_bytes(uint32_t at) {
    uint32_t v;
    if constexpr (BYTES == 1) asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    else if constexpr (BYTES == 2) asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
// Two scales' bytes, in bits 0-7 and 16-23, for q4_pair (a byte of 255 for a number: what it spoils is set to NaN later).
__device__ __forceinline__ Q4Scale2 fq_scale2(uint32_t bytes) {
    const uint32_t s = bytes * 16u + 0x35003500u;
    return {s, q4_mul2(s, 0xc308c308u)};   // -136
}
// Bit 7 of a byte of 255 in y (and perhaps of the bytes above it).
__device__ __forceinline__ uint32_t fq_nan_bytes(uint32_t y) { return (0xfefefefeu - y) & y & 0x80808080u; }

// A segment: what a warp's share has of one job.  Its keys are some of the prefix's, then some of the sequence's own.
struct FqSegment {
    AttnJob j;
    int pre0, pre1, own0, own1;
    int tiles;           // 0: the share is done
    int at, stop;        // the tiles, of the call's
};
constexpr int FQ_SEGS = 4;   // the one at work, and two that the copies may be ahead
// A segment that has to be put together with those of other warps: the CTA's share of its job begins with it, or not.
struct FqPiece {
    PartJob job;
    int rows, begin, end;   // rows 0: none; begin: whether it is the first; end: whether it is the last
    int first, whole;       // of what the CTA has of the job: it has the job's first tile; all of them
};
template <int DP, typename T> size_t FqCfg<DP, T>::smem(int n_seq) {
    return SEGS_AT + WARPS * (FQ_SEGS * sizeof(FqSegment) + 2 * sizeof(FqPiece)) + ((size_t)n_seq + 3) * 4;
}

// Tiles at .. stop - 1 (of the call's) of job j, by one warp.
__device__ __forceinline__ void fq_fill(const AttnPlan &p, FqSegment &s, const AttnJob &j, int at, int stop) {
    const int pre = j.seq < 0 || p.fused ? p.prefix_tiles : 0, t0 = at - j.g0, t1 = stop - j.g0;
    __syncwarp();
    if ((threadIdx.x & 31) == 0) {
        s.j = j;
        s.pre0 = min(t0, pre) * FQ_KEYS;
        s.pre1 = min(min(t1, pre) * FQ_KEYS, p.prefix_len);
        s.own0 = max(t0 - pre, 0) * FQ_KEYS;
        s.own1 = min(max(t1 - pre, 0) * FQ_KEYS, j.own_len);
        s.tiles = t1 - t0;
        s.at = at;
        s.stop = stop;
    }
    __syncwarp();
}
// The segment behind `last` of a share that ends at at_end.
static __device__ __noinline__ void fq_next(const AttnPlan &p, const int *bases, const FqSegment &last, int at_end, FqSegment &to) {
    const AttnJob j = last.j;
    if (j.g1 < at_end) {
        const AttnJob next = attn_next(p, bases, j);
        fq_fill(p, to, next, j.g1, min(at_end, next.g1));
    } else {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) to.tiles = 0;
        __syncwarp();
    }
}

// A walk over the tiles of a segment: the first key, where the keys end.
struct FqWalk {
    int key0, end;
    bool pre;
    __device__ __forceinline__ void begin(const FqSegment &s) {   // (of a segment that has tiles)
        pre = s.pre1 > s.pre0;
        key0 = pre ? s.pre0 : s.own0;
        end = pre ? s.pre1 : s.own1;
    }
    __device__ __forceinline__ void step(int own0, int own1) {
        key0 += FQ_KEYS;
        if (pre && key0 >= end) {
            pre = false;
            key0 = own0;
            end = own1;
        }
    }
};

// Eight keys of a page that is not there read as zeros; by the eight lanes that bring them.
template <int DP, typename T> static __device__ __noinline__ void fq_no_page(void *ws, uint32_t buf, int first) {
    using Cfg = FqCfg<DP, T>;
    raise_status(ws, DEV_STATUS_BAD_INDEX, 42);
    const auto put = [](uint32_t at, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); };
    for (int i = threadIdx.x & 7; i < 8 * (DP / 8); i += 8) {
        const int r = first + i / (DP / 8), w = i % (DP / 8);
        put(buf + r * Cfg::KROW + w * 4, Q4_ZEROS);
        put(buf + Cfg::V_AT + r * Cfg::VROW + w * 4, Q4_ZEROS);
    }
    for (int i = threadIdx.x & 7; i < 2 * Cfg::SROW; i += 8) {
        put(buf + Cfg::KS_AT + first * Cfg::SROW + i * 4, 0u);
        put(buf + Cfg::VS_AT + first * Cfg::SROW + i * 4, 0u);
    }
}

// What brings a warp's keys, STAGES - 1 tiles ahead of the products, from segment to segment.  Eight lanes have eight of the 32
// keys, which are of one page.  The pages are looked up a tile earlier still.
// EXACT: the head is DP wide, so that the rows' distances are constants.
template <int DP, bool EXACT, typename T> struct FqCopies {
    using Cfg = FqCfg<DP, T>;
    static constexpr int PPR = DP / 32, RP = 8 / PPR;     // 16-byte pieces of a key's codes; keys that 8 lanes bring at once
    static constexpr int WPR = DP / 64, RS = 8 / WPR;     // 4-byte pieces of a key's scales; keys at once
    const AttnPlan &p;
    const AttnData &x;
    FqSegment *const segs;                 // a ring of FQ_SEGS
    const int *const bases;
    const int at_end;                      // where the share ends
    int code_row, scale_row;
    int code_at, scale_at;                 // where the lane's first pieces are behind the codes and the scales of its first key
    uint32_t k_to, v_to, ks_to, vs_to;     // and in a buffer
    FqWalk at;                             // the tile that is next, and the page of the lane's keys
    int seg, left, page;                   // its segment, tiles of that from it on; -1: no page
    const int *own_pages;
    int own0, own1;
    long long head;

    __device__ __forceinline__ FqCopies(const AttnPlan &p_, const AttnData &x_, FqSegment *segs_, const int *bases_, int at_end_)
        : p(p_), x(x_), segs(segs_), bases(bases_), at_end(at_end_) {
        const int lane = threadIdx.x & 31, i = lane & 7, e = i % PPR, r = i / PPR, ws = i % WPR, rs = i / WPR, first = lane & 24;
        code_row = EXACT ? DP / 2 : x.q4.code_row;
        scale_row = EXACT ? DP / 16 : x.q4.scale_row;
        code_at = r * code_row + e * 16;
        scale_at = x.q4.scale_off + rs * scale_row + ws * 4;
        // (the rows of the keys that a lane brings are its first one's plus a constant)
        k_to = (first + fq_row(r)) * Cfg::KROW + e * 16;
        v_to = Cfg::V_AT + (first + r) * Cfg::VROW + (e ^ fq_turn<DP>(r)) * 16;
        ks_to = Cfg::KS_AT + (first + fq_row(rs)) * Cfg::SROW + ws * 4;
        vs_to = Cfg::VS_AT + (first + rs) * Cfg::SROW + ws * 4;
        seg = 0;
        enter();
    }
    __device__ __forceinline__ int first() const { return threadIdx.x & 24; }
    __device__ __forceinline__ void enter() {
        const FqSegment &s = segs[seg % FQ_SEGS];
        left = s.tiles;
        page = -1;
        if (left == 0) return;
        own_pages = p.page_table + (long long)s.j.seq * p.table_stride;
        own0 = s.own0;
        own1 = s.own1;
        head = (s.j.head / x.heads_per_key) * x.stride_head;
        at.begin(s);
        look_up();
    }
    __device__ __forceinline__ void look_up() {
        const int key = at.key0 + first();
        page = -1;
        if (key < at.end) page = __ldg((at.pre ? p.prefix_pages : own_pages) + (key >> p.page_shift));
    }
    // Asks for the tile that is next.  What lies in the page behind the last key comes with it, and is dealt with when it is read.
    __device__ __forceinline__ void ask(uint32_t buf) {
        const int key = at.key0 + first();
        if ((unsigned)page < (unsigned)p.n_pages) {
            const int slot = key & ((1 << p.page_shift) - 1);
            const long long block = page * x.stride_page + head;
            const long long codes = block + (slot * code_row + code_at), scales = block + (slot * scale_row + scale_at);
            const uint8_t *const k = static_cast<const uint8_t *>(x.k), *const v = static_cast<const uint8_t *>(x.v);
            const uint8_t *const kc = k + codes, *const vc = v + codes, *const ks = k + scales, *const vs = v + scales;
            if (EXACT || (p.d & 31) == 0) {
                if (EXACT || (int)(threadIdx.x & 7) % PPR * 32 < p.d) {
#pragma unroll
                    for (int r = 0; r < 8; r += RP) {
                        fq_copy<16>(buf + k_to + fq_row(r) * Cfg::KROW, kc + r * code_row);
                        fq_copy<16>(buf + (v_to ^ (fq_turn<DP>(r) * 16)) + r * Cfg::VROW, vc + r * code_row);
                    }
                }
            } else {   // (rows of codes are on 8-byte boundaries; the last piece may have one group)
                const int e = (int)(threadIdx.x & 7) % PPR * 32;
#pragma unroll
                for (int r = 0; r < 8; r += RP)
#pragma unroll
                    for (int h = 0; h < 16; h += 8)
                        if (e + 2 * h < p.d) {
                            fq_copy<8>(buf + k_to + fq_row(r) * Cfg::KROW + h, kc + r * code_row + h);
                            fq_copy<8>(buf + (v_to ^ (fq_turn<DP>(r) * 16)) + r * Cfg::VROW + h, vc + r * code_row + h);
                        }
            }
            if (EXACT || (int)(threadIdx.x & 7) % WPR * 64 < p.d) {
#pragma unroll
                for (int r = 0; r < 8; r += RS) {
                    fq_copy<4>(buf + ks_to + fq_row(r) * Cfg::SROW, ks + r * scale_row);
                    fq_copy<4>(buf + vs_to + r * Cfg::SROW, vs + r * scale_row);
                }
            }
        } else if (key < at.end) {
            fq_no_page<DP, T>(p.ws, buf, first());
        }
    }
    // Asks for the tile that is next, if there is one, and goes on to the one behind it.
    __device__ __forceinline__ void go(uint32_t buf) {
        if (left > 0) {
            ask(buf);
            if (--left > 0) {
                at.step(own0, own1);
                look_up();
            } else {
                fq_next(p, bases, segs[seg % FQ_SEGS], at_end, segs[(seg + 1) % FQ_SEGS]);
                ++seg;
                enter();
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
};

// The scales of values that must not be multiplied with, since 0 * NaN would reach the sum, become finite: of keys from `from`
// on (none of the block's rows sees them, or not all do).  Whether any of the latter was NaN.
template <int DP, typename T> static __device__ __noinline__ bool fq_clear_scales(uint8_t *scales, int from, int end, bool all) {
    using Cfg = FqCfg<DP, T>;
    bool found = false;
    __syncwarp();
    for (int i = threadIdx.x & 31; i < FQ_KEYS * Cfg::SROW; i += 32) {
        const int r = i / Cfg::SROW;
        if (r < from) continue;
        if (r >= end || all) {
            scales[i] = 0;
        } else if (scales[i] == Q4_NAN) {
            scales[i] = 0;
            found = true;
        }
    }
    __syncwarp();
    return __any_sync(0xffffffffu, found);
}
// An fp32 number as a sum of bf16 ones, each the rest of those before to the nearest: 24 bits in three.
template <int PARTS> __device__ __forceinline__ void fq_split(float a, float b, uint32_t (&to)[PARTS]) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        to[i] = fq_pack(a, b);
        a -= __uint_as_float(to[i] << 16);
        b -= __uint_as_float(to[i] & 0xffff0000u);
    }
}
// The queries of a job as the first product takes them: row lane / 4, entries of quarter lane % 4.
template <int DP, typename T>
__device__ __forceinline__ void fq_queries(const AttnPlan &p, const AttnData &x, const AttnJob &j, uint32_t (&q)[DP / 16][2][FqCfg<DP, T>::PARTS]) {
    const int lane = threadIdx.x & 31, r = lane >> 2, tok = attn_row_token(p, r);
    const T *const at = static_cast<const T *>(x.q) + (j.tok0 + tok) * x.ld_q + (j.head * p.group + r - tok * p.group) * p.d;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const int e = (lane & 3) * (DP / 4) + 4 * c;
        const bool on = r < j.rows && e < p.d;
        if constexpr (sizeof(T) == 2) {
            uint2 v = make_uint2(0u, 0u);
            if (on) v = *reinterpret_cast<const uint2 *>(at + e);
            q[c][0][0] = v.x;
            q[c][1][0] = v.y;
        } else {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (on) v = *reinterpret_cast<const float4 *>(at + e);
            fq_split(v.x, v.y, q[c][0]);
            fq_split(v.z, v.w, q[c][1]);
        }
    }
}
// Four entries of a row to the output.
template <typename T> __device__ __forceinline__ void fq_store4(T *to, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(to) = make_uint2(fq_pack(a, b), fq_pack(c, d));
    else *reinterpret_cast<float4 *>(to) = make_float4(a, b, c, d);
}

// One warp's share, tiles at .. at_end - 1 of the call's (the CTA's are cta_at .. cta_end - 1), the first of them of job j.
// to_piece: whatever it has of a job is put together with others'.
template <int DP, bool EXACT, typename T>
__device__ __forceinline__ void fq_work(const AttnPlan &p, const AttnData &x, const int *bases, const AttnJob &j, int cta_at, int cta_end,
                                        int at, int at_end, bool to_piece, uint8_t *mine, FqSegment *segs, uint8_t *piece, FqPiece *pieces) {
    using Cfg = FqCfg<DP, T>;
    constexpr int NC = DP / 16, PARTS = Cfg::PARTS;
    constexpr int KW = DP / 32, KG = DP / 64;        // words of codes and scales of a lane's quarter of a key
    constexpr int VW = DP / 64, VG = DP == 256 ? 2 : 1;   // and of its eighth of a value
    const int lane = threadIdx.x & 31;
    const uint32_t ring = smem_u32(mine);
    // queries lie by row lane / 4, S and the results by rows ra and ra + 1
    const int g = lane >> 2, t4 = lane & 3, ra = t4 * 2;
    // scales of groups beyond the head's width may be anything (their codes meet queries of zero, and results that nobody reads)
    uint32_t k_groups = 0;
#pragma unroll
    for (int i = 0; i < KG; ++i)
        if ((t4 * KG + i) * 16 < p.d) k_groups |= 0xffu << (8 * i);
    const uint32_t v_groups = (DP == 64 ? g >> 1 : g * VG) * 16 < p.d ? 0x80808080u : 0u;

    fq_fill(p, segs[0], j, at, min(at_end, j.g1));
    FqCopies<DP, EXACT, T> copies(p, x, segs, bases, at_end);
    int slot = 0;   // buffer of the tile at work
#pragma unroll
    for (int i = 0; i < Cfg::STAGES - 1; ++i) copies.go(ring + i * Cfg::STAGE);
    // a lane's places in a buffer: rows g and g + 8 of K; keys t and t + 4 (the products' 2t and 2t + 1) and those plus 8 of V
    const uint32_t k_from = g * Cfg::KROW + t4 * (DP / 8), ks_from = Cfg::KS_AT + g * Cfg::SROW + t4 * KG;
    uint32_t v_from[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = t4 + 4 * h, byte = g * (DP / 16);
        v_from[h] = Cfg::V_AT + r * Cfg::VROW + (((byte >> 4) ^ fq_turn<DP>(r)) << 4) + (byte & 15);
    }
    const uint32_t vs_from = Cfg::VS_AT + t4 * Cfg::SROW + (DP == 64 ? g >> 1 : g * VG);
    const uint32_t magic = x.q4.magic;
    uint32_t q[NC][2][PARTS];
    fq_queries<DP, T>(p, x, segs[0].j, q);
#pragma unroll 1
    for (int at_seg = 0;; ++at_seg) {
        const FqSegment &seg = segs[at_seg % FQ_SEGS];
        const int seen0 = seg.j.seen0, tiles = seg.tiles;
        float m_a = -INFINITY, m_b = -INFINITY, b_a = 0.f, b_b = 0.f, l_a = 0.f, l_b = 0.f, o[NC][4];   // b: -m, 0 while there is none
#pragma unroll
        for (int i = 0; i < NC; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

        bool marked = false;   // whether values were cleared, and have to be added to the rows that see them
        FqWalk t;
        t.begin(seg);
#pragma unroll 1
        for (int i = 0; i < tiles; ++i, t.step(seg.own0, seg.own1)) {
            __syncwarp();   // the buffer of the tile before is done with
            copies.go(ring + (slot == 0 ? Cfg::STAGES - 1 : slot - 1) * Cfg::STAGE);
            asm volatile("cp.async.wait_group %0;" ::"n"(Cfg::STAGES - 1) : "memory");
            __syncwarp();   // the keys of this one have come, for every lane
            const uint32_t buf = ring + slot * Cfg::STAGE;
            slot = slot + 1 == Cfg::STAGES ? 0 : slot + 1;
            // keys that some rows see and some do not, or that are not there
            const bool edge = t.key0 + FQ_KEYS > (t.pre ? t.end : min(t.end, seen0));
            if (edge) {
                const bool apart = !t.pre && seen0 < t.end;
                marked |= fq_clear_scales<DP, T>(mine + (buf - ring) + Cfg::VS_AT, apart ? max(seen0 - t.key0, 0) : t.end - t.key0, t.end - t.key0, !apart);
            }
            float s[2][4];      // 16 keys each
            uint32_t bad = 0;   // bytes of 255 among the keys' scales
            uint32_t kscale[4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t kw[2][KW], ks[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    fq_lds(kw[h], buf + k_from + (16 * u + 8 * h) * Cfg::KROW);
                    ks[h] = fq_lds_bytes<KG>(buf + ks_from + (16 * u + 8 * h) * Cfg::SROW) & k_groups;
                    kscale[2 * u + h] = ks[h];
                }
                bad |= KG == 4 ? fq_nan_bytes(ks[0]) | fq_nan_bytes(ks[1]) : fq_nan_bytes(ks[0] | ks[1] << 16);
                s[u][0] = s[u][1] = s[u][2] = s[u][3] = 0.f;
                Q4Scale2 a, b;
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    if (w % 2 == 0) {   // (a byte, twice)
                        const uint32_t sel = 0x4040u + (w / 2) * 0x0101u;
                        a = fq_scale2(__byte_perm(ks[0], 0u, sel));
                        b = fq_scale2(__byte_perm(ks[1], 0u, sel));
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t k0 = q4_pair(kw[0][w], 2 * e, a, magic), k1 = q4_pair(kw[1][w], 2 * e, b, magic),
                                       k2 = q4_pair(kw[0][w], 2 * e + 1, a, magic), k3 = q4_pair(kw[1][w], 2 * e + 1, b, magic);
#pragma unroll
                        for (int i = PARTS - 1; i >= 0; --i) mma_bf16(s[u], k0, k1, k2, k3, q[2 * w + e][0][i], q[2 * w + e][1][i]);
                    }
                }
            }
            if (__any_sync(0xffffffffu, bad != 0)) {   // a group of a key is NaN, and so is the logit
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    bool nan = false;
#pragma unroll
                    for (int i = 0; i < KG; ++i) nan = nan || (kscale[h] >> (8 * i) & 0xffu) == Q4_NAN;
                    if (__ballot_sync(0xffffffffu, nan) >> (lane & 28) & 15u) s[h >> 1][(h & 1) * 2] = s[h >> 1][(h & 1) * 2 + 1] = __uint_as_float(0x7fffffffu);
                }
            }
            if (edge) {   // keys of the 32 that the two rows see
                const int see_a = (t.pre ? t.end : min(t.end, seen0 + attn_row_token(p, ra))) - t.key0 - fq_key(g),
                          see_b = (t.pre ? t.end : min(t.end, seen0 + attn_row_token(p, ra + 1))) - t.key0 - fq_key(g);
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    if (8 * h >= see_a) s[h >> 1][(h & 1) * 2] = -INFINITY;
                    if (8 * h >= see_b) s[h >> 1][(h & 1) * 2 + 1] = -INFINITY;
                }
            }
            float x_a = max_nan(max_nan(s[0][0], s[0][2]), max_nan(s[1][0], s[1][2])) * p.scale_log2;
            float x_b = max_nan(max_nan(s[0][1], s[0][3]), max_nan(s[1][1], s[1][3])) * p.scale_log2;
            // the maximum moves only when 2^(S - m) could grow too large, or there is none yet, or it is NaN
            if (__any_sync(0xffffffffu, !(x_a <= m_a + FQ_SLACK) || !(x_b <= m_b + FQ_SLACK))) {
#pragma unroll
                for (int w = 4; w < 32; w *= 2) {
                    x_a = max_nan(x_a, __shfl_xor_sync(0xffffffffu, x_a, w));
                    x_b = max_nan(x_b, __shfl_xor_sync(0xffffffffu, x_b, w));
                }
                float f_a = 1.f, f_b = 1.f;
                if (!(x_a <= m_a)) {   // (a logit that is NaN or infinite makes the row NaN: x - x)
                    f_a = fast_exp2(m_a - x_a);
                    l_a = l_a * f_a + (x_a - x_a);
                    m_a = x_a == x_a ? x_a : INFINITY;
                    b_a = -m_a;
                }
                if (!(x_b <= m_b)) {
                    f_b = fast_exp2(m_b - x_b);
                    l_b = l_b * f_b + (x_b - x_b);
                    m_b = x_b == x_b ? x_b : INFINITY;
                    b_b = -m_b;
                }
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    o[c][0] *= f_a;
                    o[c][1] *= f_b;
                    o[c][2] *= f_a;
                    o[c][3] *= f_b;
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[u][2 * h] = fast_exp2(fmaf(s[u][2 * h], p.scale_log2, b_a));
                    s[u][2 * h + 1] = fast_exp2(fmaf(s[u][2 * h + 1], p.scale_log2, b_b));
                    l_a += s[u][2 * h];
                    l_b += s[u][2 * h + 1];
                }
                // keys t, t + 4, t + 8, t + 12 of the 16
                uint32_t vw[4][VW], vs[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    fq_lds(vw[h], buf + v_from[h & 1] + (16 * u + (h >> 1) * 8) * Cfg::VROW);
                    vs[h] = fq_lds_bytes<VG>(buf + vs_from + (16 * u + 4 * h) * Cfg::SROW);
                }
                // (P in bf16, as the values are: 2^-8 of each at most; fp32 calls in three parts)
                uint32_t w0[PARTS], w1[PARTS];
                fq_split(s[u][0], s[u][1], w0);
                fq_split(s[u][2], s[u][3], w1);
#pragma unroll
                for (int i = 0; i < PARTS; ++i) w0[i] = fq_movmatrix(w0[i]), w1[i] = fq_movmatrix(w1[i]);
                Q4Scale2 lo, hi;
                const uint32_t s01 = vs[0] | vs[1] << 16, s23 = vs[2] | vs[3] << 16;
                const uint32_t v_bad = VG == 2 ? fq_nan_bytes(s01) | fq_nan_bytes(s23) : fq_nan_bytes(s01 | s23 << 8);
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    if (w % 2 == 0) {
                        lo = fq_scale2(VG == 2 ? __byte_perm(s01, 0u, 0x4240u + (w / 2) * 0x0101u) : s01);
                        hi = fq_scale2(VG == 2 ? __byte_perm(s23, 0u, 0x4240u + (w / 2) * 0x0101u) : s23);
                    }
                    const uint32_t even0 = __byte_perm(vw[0][w], vw[1][w], 0x5410), odd0 = __byte_perm(vw[0][w], vw[1][w], 0x7632);
                    const uint32_t even1 = __byte_perm(vw[2][w], vw[3][w], 0x5410), odd1 = __byte_perm(vw[2][w], vw[3][w], 0x7632);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {   // entries 2e and 2e + 1 of the word
                        const uint32_t v0 = q4_pair(even0, e, lo, magic), v1 = q4_pair(odd0, e, lo, magic), v2 = q4_pair(even1, e, hi, magic),
                                       v3 = q4_pair(odd1, e, hi, magic);
#pragma unroll
                        for (int i = PARTS - 1; i >= 0; --i) mma_bf16(o[4 * w + e], v0, v1, v2, v3, w0[i], w1[i]);
                    }
                }
                if (__any_sync(0xffffffffu, (v_bad & v_groups) != 0)) {   // a group of values is NaN, for all rows (all of them see it)
#pragma unroll
                    for (int i = 0; i < VG; ++i) {
                        bool nan = false;
#pragma unroll
                        for (int h = 0; h < 4; ++h) nan = nan || (vs[h] >> (8 * i) & 0xffu) == Q4_NAN;
                        if (__ballot_sync(0xffffffffu, nan) >> (lane & 28) & 15u) {
#pragma unroll
                            for (int c = i * (NC / VG); c < (i + 1) * (NC / VG); ++c)
                                o[c][0] = o[c][1] = o[c][2] = o[c][3] = __uint_as_float(0x7fffffffu);
                        }
                    }
                }
            }
        }
        // Values that were cleared, of keys that some rows see and some do not: to the rows that do.
        if (marked) {
            for (int k = max(seen0, seg.own0); k < seg.own1; ++k) {
                const int page = __ldg(p.page_table + (long long)seg.j.seq * p.table_stride + (k >> p.page_shift));
                if ((unsigned)page >= (unsigned)p.n_pages) continue;
                const uint8_t *const scales = static_cast<const uint8_t *>(x.v) + page * x.stride_page + (seg.j.head / x.heads_per_key) * x.stride_head +
                                              x.q4.scale_off + (k & ((1 << p.page_shift) - 1)) * x.q4.scale_row;
                const float nan = __uint_as_float(0x7fffffffu);
                const bool sees_a = k < seen0 + attn_row_token(p, ra), sees_b = k < seen0 + attn_row_token(p, ra + 1);
#pragma unroll
                for (int i = 0; i < VG; ++i) {
                    const int group = DP == 64 ? g >> 1 : g * VG + i;
                    if (group * 16 >= p.d || scales[group] != Q4_NAN) continue;
#pragma unroll
                    for (int c = i * (NC / VG); c < (i + 1) * (NC / VG); ++c) {
                        if (sees_a) o[c][0] = o[c][2] = nan;
                        if (sees_b) o[c][1] = o[c][3] = nan;
                    }
                }
            }
        }
#pragma unroll
        for (int w = 4; w < 32; w *= 2) {
            l_a += __shfl_xor_sync(0xffffffffu, l_a, w);
            l_b += __shfl_xor_sync(0xffffffffu, l_b, w);
        }
        // The result: a lane has an eighth of the entries of two rows.  What the CTA has of the job, all of it here: to the output or
        // the partials; else to the pieces.
        const int job_at = max(seg.j.g0, cta_at), job_end = min(seg.j.g1, cta_end);
        const bool first = job_at == seg.j.g0, whole = first && job_end == seg.j.g1, alone = seg.at == job_at && seg.stop == job_end && !to_piece;
        const bool last_one = seg.stop >= at_end;
        if (!alone) {
            if (last_one && at_seg > 0) {   // (nothing is on its way into the ring any more, and nothing read from it)
                piece = mine;
                ++pieces;
                asm volatile("cp.async.wait_all;" ::: "memory");
            }
            __syncwarp();
            if (lane == 0) *pieces = FqPiece{seg.j, seg.j.rows, seg.at == job_at, seg.stop == job_end, first, whole};
        }
        const bool direct = attn_direct(p, seg.j, whole);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = ra + h, e0 = g * (DP / 8);
            if (r >= seg.j.rows) continue;
            const float m = h ? m_b : m_a, l = h ? l_b : l_a;
            if (alone && direct) {
                const int tok = attn_row_token(p, r);
                const float inv = m == -INFINITY ? 0.f : 1.0f / l;
                T *const to = static_cast<T *>(x.out) + (seg.j.tok0 + tok) * x.ld_out + (seg.j.head * p.group + r - tok * p.group) * p.d + e0;
#pragma unroll
                for (int c = 0; c < NC; c += Cfg::F32 ? 2 : 4)   // (16 bytes)
                    if (EXACT || e0 + 2 * c < p.d) {
                        if constexpr (sizeof(T) == 2)
                            *reinterpret_cast<uint4 *>(to + 2 * c) =
                                make_uint4(fq_pack(o[c][h] * inv, o[c][2 + h] * inv), fq_pack(o[c + 1][h] * inv, o[c + 1][2 + h] * inv),
                                           fq_pack(o[c + 2][h] * inv, o[c + 2][2 + h] * inv), fq_pack(o[c + 3][h] * inv, o[c + 3][2 + h] * inv));
                        else
                            *reinterpret_cast<float4 *>(to + 2 * c) = make_float4(o[c][h] * inv, o[c][2 + h] * inv, o[c + 1][h] * inv, o[c + 1][2 + h] * inv);
                    }
            } else {
                PartPlace to{reinterpret_cast<float *>(piece) + 2 * r, reinterpret_cast<float *>(piece) + 2 * FQ_ROWS + r * Cfg::LDO};
                if (alone) to = attn_place(p, seg.j, first, 0, r);
                if (g == 0) *reinterpret_cast<float2 *>(to.ml) = make_float2(m, l);
#pragma unroll
                for (int c = 0; c < NC; c += 2)
                    if (EXACT || e0 + 2 * c < p.d)
                        *reinterpret_cast<float4 *>(to.o + e0 + 2 * c) = make_float4(o[c][h], o[c][2 + h], o[c + 1][h], o[c + 1][2 + h]);
            }
        }
        if (segs[(at_seg + 1) % FQ_SEGS].tiles == 0) return;
        fq_queries<DP, T>(p, x, segs[(at_seg + 1) % FQ_SEGS].j, q);
    }
}

// The pieces of jobs that went to several warps of the CTA, put together in their order: the output, or its partial.  As many
// warps to a job as there are for each.
template <int DP, typename T>
static __device__ __noinline__ void fq_join_pieces(const AttnPlan &p, const AttnData &x, const uint8_t *smem_raw, const FqPiece *pieces) {
    using Cfg = FqCfg<DP, T>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // (lane i: piece i, in the order of the keys; a warp's first, then its last)
    const FqPiece mine = lane < 2 * Cfg::WARPS ? pieces[lane] : FqPiece{};
    const unsigned there = __ballot_sync(0xffffffffu, mine.rows > 0), begins = __ballot_sync(0xffffffffu, mine.rows > 0 && mine.begin != 0);
    const int jobs = __popc(begins);
    if (jobs == 0) return;
    int per = Cfg::WARPS;   // warps to a job
    while (per > 1 && per * jobs > Cfg::WARPS) per >>= 1;
    const auto at = [&](int i) {
        return reinterpret_cast<const float *>(i & 1 ? smem_raw + (i >> 1) * (Cfg::STAGES * Cfg::STAGE) : smem_raw + Cfg::PIECES_AT + (i >> 1) * Cfg::PIECE);
    };
    for (int n = warp / per; n < jobs; n += Cfg::WARPS / per) {
        const int i0 = __fns(begins, 0, n + 1);
        const FqPiece a = pieces[i0];
        // its pieces: up to the next one that ends a job
        unsigned which = there & ~((1u << i0) - 1u);
        for (int i = threadIdx.x - (warp - warp % per) * 32; i < a.rows * (DP / 4); i += per * 32) {
            const int r = i / (DP / 4), e = i % (DP / 4) * 4;
            if (e >= p.d) continue;
            float M = -INFINITY, sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (unsigned left = which; left != 0; left &= left - 1) {
                const int k = __ffs(left) - 1;
                const float *const from = at(k);
                const float2 ml = *reinterpret_cast<const float2 *>(from + 2 * r);
                const float4 v = *reinterpret_cast<const float4 *>(from + 2 * FQ_ROWS + r * Cfg::LDO + e);
                const float m = fmaxf(M, ml.x), f = m == -INFINITY ? 0.f : fast_exp2(M - m), w = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m);
                M = m;
                sum = fmaf(sum, f, w * ml.y);
                acc.x *= f, acc.y *= f, acc.z *= f, acc.w *= f;
                if (ml.x != -INFINITY) {   // (a weight of 0 counts: it keeps NaN)
                    acc.x = fmaf(w, v.x, acc.x);
                    acc.y = fmaf(w, v.y, acc.y);
                    acc.z = fmaf(w, v.z, acc.z);
                    acc.w = fmaf(w, v.w, acc.w);
                }
                if (pieces[k].end) break;
            }
            if (p.fused && a.whole != 0) {
                const int tok = attn_row_token(p, r);
                const float inv = M == -INFINITY ? 0.f : 1.0f / sum;
                fq_store4(static_cast<T *>(x.out) + (a.job.tok0 + tok) * x.ld_out + (a.job.head * p.group + r - tok * p.group) * p.d + e, acc.x * inv,
                          acc.y * inv, acc.z * inv, acc.w * inv);
            } else {
                const PartPlace to = attn_place(p, a.job, a.first != 0, 0, r);
                if (e == 0) *reinterpret_cast<float2 *>(to.ml) = make_float2(M, sum);
                *reinterpret_cast<float4 *>(to.o + e) = acc;
            }
        }
    }
}

// A call whose jobs go to the CTAs, or clusters of them, whole, so that nothing is left to join.  First job of every sequence into bases[0 .. n_seq], by all threads.
static __device__ __noinline__ void fq_scan_jobs(const AttnPlan &p, int *bases) {
    const int lane = threadIdx.x & 31;
    for (int s = threadIdx.x; s < p.n_seq; s += blockDim.x) bases[s] = ceil_div(attn_seq(p, s).nq, p.block_tokens) * p.hkv;
    __syncthreads();
    if (threadIdx.x < 32) {
        int sum = 0;
        for (int s0 = 0; s0 < p.n_seq; s0 += 32) {
            const int mine = s0 + lane < p.n_seq ? bases[s0 + lane] : 0;
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            if (s0 + lane < p.n_seq) bases[s0 + lane] = sum + upto - mine;
            sum += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (lane == 0) bases[p.n_seq] = sum;
    }
    __syncthreads();
}
// Job i of such a call; its tiles begin at 0.
static __device__ __noinline__ AttnJob fq_whole_job(const AttnPlan &p, const int *bases, int i) {
    int lo = 0, hi = p.n_seq;  // bases[lo] <= i < bases[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (bases[mid] <= i) lo = mid; else hi = mid;
    }
    const int of = i - bases[lo], block = (int)((uint32_t)of / (uint32_t)p.hkv);
    return attn_own_job(p, attn_seq(p, lo), lo, of - block * p.hkv, block, 0);
}


// (not the .aligned forms: the loops in front of a meeting let the lanes of a warp go different ways)
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// m and l of a row and four entries of its results, from a piece of any CTA of the cluster.
struct FqPart {
    float2 ml;
    float4 o;
};
__device__ __forceinline__ FqPart fq_remote(uint32_t ml, uint32_t o, int rank) {
    FqPart v;
    asm volatile("{\n\t.reg .u32 a, b;\n\tmapa.shared::cluster.u32 a, %6, %8;\n\tmapa.shared::cluster.u32 b, %7, %8;\n\t"
                 "ld.shared::cluster.v2.f32 {%0, %1}, [a];\n\tld.shared::cluster.v4.f32 {%2, %3, %4, %5}, [b];\n\t}"
                 : "=f"(v.ml.x), "=f"(v.ml.y), "=f"(v.o.x), "=f"(v.o.y), "=f"(v.o.z), "=f"(v.o.w)
                 : "r"(ml), "r"(o), "r"(rank)
                 : "memory");
    return v;
}
// A running sum of parts, scaled by the largest m so far.
struct FqSum {
    float M = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(const FqPart &v) {
        const float m = fmaxf(M, v.ml.x), f = m == -INFINITY ? 0.f : fast_exp2(M - m), w = v.ml.x == -INFINITY ? 0.f : fast_exp2(v.ml.x - m);
        M = m;
        l = fmaf(l, f, w * v.ml.y);
        o.x *= f, o.y *= f, o.z *= f, o.w *= f;
        if (v.ml.x != -INFINITY) {   // (a part in which the row sees nothing has no results; a weight of 0 counts, which keeps NaN)
            o.x = fmaf(w, v.o.x, o.x);
            o.y = fmaf(w, v.o.y, o.y);
            o.z = fmaf(w, v.o.z, o.z);
            o.w = fmaf(w, v.o.w, o.w);
        }
    }
};
template <typename T> __device__ __forceinline__ void fq_output(const AttnPlan &p, const AttnData &x, const PartJob &j, int r, int e, const FqSum &s) {
    const int tok = attn_row_token(p, r);
    const float inv = s.M == -INFINITY ? 0.f : 1.0f / s.l;
    fq_store4(static_cast<T *>(x.out) + (j.tok0 + tok) * x.ld_out + (j.head * p.group + r - tok * p.group) * p.d + e, s.o.x * inv, s.o.y * inv,
              s.o.z * inv, s.o.w * inv);
}
// A whole job's pieces put together: those of the CTA's first n warps, then the sums of the cluster's CTAs, which are left in the ring.
template <int DP, typename T>
static __device__ __noinline__ void fq_join_whole(const AttnPlan &p, const AttnData &x, uint8_t *smem_raw, const AttnJob &j, int n, int cluster, int rank) {
    using Cfg = FqCfg<DP, T>;
    const int items = j.rows * (DP / 4);
    // (a part of the pieces to each of four neighbouring threads, where there are enough)
    const int per = 4 * items <= Cfg::THREADS ? 4 : 1;
    for (int i = threadIdx.x; i < items * per; i += Cfg::THREADS) {
        const int item = i / per, r = item / (DP / 4), e = item % (DP / 4) * 4;
        FqSum s;
#pragma unroll 4
        for (int w = i % per; w < n; w += per) {
            const float *const from = reinterpret_cast<const float *>(smem_raw + Cfg::PIECES_AT + w * Cfg::PIECE);
            s.add(FqPart{*reinterpret_cast<const float2 *>(from + 2 * r), *reinterpret_cast<const float4 *>(from + 2 * FQ_ROWS + r * Cfg::LDO + e)});
        }
        for (int o = 1; o < per; o *= 2) {   // (one turn, of whole warps)
            FqPart v;
            v.ml = make_float2(__shfl_xor_sync(0xffffffffu, s.M, o), __shfl_xor_sync(0xffffffffu, s.l, o));
            v.o = make_float4(__shfl_xor_sync(0xffffffffu, s.o.x, o), __shfl_xor_sync(0xffffffffu, s.o.y, o), __shfl_xor_sync(0xffffffffu, s.o.z, o),
                              __shfl_xor_sync(0xffffffffu, s.o.w, o));
            s.add(v);
        }
        if (i % per != 0) continue;
        if (cluster == 1) {
            if (e < p.d) fq_output<T>(p, x, j, r, e, s);
        } else {
            float *const to = reinterpret_cast<float *>(smem_raw);
            if (e == 0) *reinterpret_cast<float2 *>(to + 2 * r) = make_float2(s.M, s.l);
            *reinterpret_cast<float4 *>(to + 2 * FQ_ROWS + r * Cfg::LDO + e) = s.o;
        }
    }
    if (cluster == 1) return;
    cluster_meet();
    const uint32_t base = smem_u32(smem_raw);
    for (int i = threadIdx.x * cluster + rank; i < items; i += Cfg::THREADS * cluster) {
        const int r = i / (DP / 4), e = i % (DP / 4) * 4;
        if (e >= p.d) continue;
        FqSum s;
#pragma unroll 4
        for (int c = 0; c < cluster; ++c) s.add(fq_remote(base + 8 * r, base + 4 * (2 * FQ_ROWS + r * Cfg::LDO + e), c));
        fq_output<T>(p, x, j, r, e, s);
    }
    cluster_meet();   // (nobody leaves, or writes again, while its sum is read)
}

// cluster: 0: the call's tiles are dealt out evenly to the CTAs; else so many CTAs, side by side, take a job whole.
template <int DP, bool EXACT, typename T>
__global__ void __launch_bounds__(FqCfg<DP, T>::THREADS, 1) attn_few_q4_kernel(const __grid_constant__ AttnPlan p,
                                                                          const __grid_constant__ AttnData x, const int cluster) {
    using Cfg = FqCfg<DP, T>;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *const mine = smem_raw + warp * (Cfg::STAGES * Cfg::STAGE), *const piece = smem_raw + Cfg::PIECES_AT + warp * Cfg::PIECE;
    FqSegment *const segs = reinterpret_cast<FqSegment *>(smem_raw + Cfg::SEGS_AT) + warp * FQ_SEGS;
    FqPiece *const all_pieces = reinterpret_cast<FqPiece *>(smem_raw + Cfg::SEGS_AT + Cfg::WARPS * FQ_SEGS * sizeof(FqSegment));
    int *const bases = reinterpret_cast<int *>(all_pieces + 2 * Cfg::WARPS);
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    if (cluster != 0) {
        fq_scan_jobs(p, bases);
        const int rank = blockIdx.x % cluster;
#pragma unroll 1
        for (int i = blockIdx.x / cluster; i < bases[p.n_seq]; i += gridDim.x / cluster) {
            const AttnJob j = fq_whole_job(p, bases, i);
            // the CTA's tiles, and this warp's of them
            const AttnShares of_cta(j.g1, cluster);
            const int cta_at = rank < of_cta.G ? of_cta.first(rank) : 0, cta_end = rank < of_cta.G ? of_cta.first(rank + 1) : 0;
            const AttnShares of_warp(cta_end - cta_at, Cfg::WARPS);
            if (warp < of_warp.G)
                fq_work<DP, EXACT, T>(p, x, bases, j, cta_at, cta_end, cta_at + of_warp.first(warp), cta_at + of_warp.first(warp + 1), true, mine, segs,
                                   piece, all_pieces + 2 * warp);
            __syncthreads();
            fq_join_whole<DP, T>(p, x, smem_raw, j, of_warp.G, cluster, rank);
            __syncthreads();   // the pieces may be written again
        }
        return;
    }
    attn_scan(p, bases);
    const AttnShares shares(bases[p.n_seq], p.grid);
    if ((int)blockIdx.x >= shares.G) return;
    const int cta_at = shares.first(blockIdx.x), cta_end = shares.first(blockIdx.x + 1);
    const AttnShares of_warp(cta_end - cta_at, Cfg::WARPS);
    if (lane < 2) all_pieces[2 * warp + lane].rows = 0;
    if (warp < of_warp.G) {
        const int at = cta_at + of_warp.first(warp);
        const AttnJob j = attn_find(p, bases, at);
        if (threadIdx.x == 0) attn_note_cut(p, shares, j, at, min(cta_end, j.g1));
        fq_work<DP, EXACT, T>(p, x, bases, j, cta_at, cta_end, at, cta_at + of_warp.first(warp + 1), false, mine, segs, piece, all_pieces + 2 * warp);
    }
    __syncthreads();
    fq_join_pieces<DP, T>(p, x, smem_raw, all_pieces);
}

AttnShape attn_few_q4_shape() {
    return {FQ_ROWS, 1, FQ_KEYS, 0};
}

template <int DP, typename T> static griffin_status launch_dp(AttnPlan p, AttnData x, int jobs, int cluster, cudaStream_t stream) {
    const void *fn = p.d == DP ? reinterpret_cast<const void *>(attn_few_q4_kernel<DP, true, T>)
                               : reinterpret_cast<const void *>(attn_few_q4_kernel<DP, false, T>);
    const size_t smem = FqCfg<DP, T>::smem(p.n_seq);
    if (ensure_dynamic_smem(fn, smem) != cudaSuccess) return GRIFFIN_ERR_CUDA;
    void *args[] = {&p, &x, &cluster};
    const dim3 block(FqCfg<DP, T>::THREADS);
    const cudaError_t e = cluster > 1 ? launch_clusters(fn, dim3(jobs * cluster), block, cluster, smem, stream, args)
                                      : launch_maybe_overlapped(fn, dim3(cluster == 1 ? jobs : p.grid), block, smem, stream, true, args);
    return e == cudaSuccess ? GRIFFIN_OK : GRIFFIN_ERR_CUDA;
}

template <typename T> static griffin_status launch_type(const AttnPlan &p, const AttnData &data, int jobs, int cluster, cudaStream_t stream) {
    if (p.d <= 64) return launch_dp<64, T>(p, data, jobs, cluster, stream);
    if (p.d <= 128) return launch_dp<128, T>(p, data, jobs, cluster, stream);
    return launch_dp<256, T>(p, data, jobs, cluster, stream);
}
griffin_status launch_attn_few_q4(const AttnPlan &plan, const AttnData &data, int dtype, int jobs, int cluster, cudaStream_t stream) {
    AttnPlan p = plan;
    if (cluster > 0) {   // (a job has the prefix's keys and the sequence's own)
        p.fused = 1;
        p.prefix_blocks = 0;
    }
    return dtype == GRIFFIN_DT_F32 ? launch_type<float>(p, data, jobs, cluster, stream) : launch_type<__nv_bfloat16>(p, data, jobs, cluster, stream);
}

}  // namespace griffin
