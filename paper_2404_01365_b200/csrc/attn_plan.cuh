// How one griffin_attn_prefix call is cut up, shared by the attention kernels and the joining kernel.
//
// A JOB is a block of query rows under one key head (row = token * group + query head of the group) and the
// keys that they see; its work is counted in TILES of KT keys.  All jobs' tiles, laid end to end, are dealt
// out in equal shares to G CTAs (one per SM, or one per tile where there are fewer): W / G each, the first W mod G of them one more.  So every SM has
// the same number of tiles to within one, however ragged the lengths, without any word from the host about
// them; a share that ends inside a job leaves a PARTIAL (running maximum m, sum l, unnormalised output, all
// fp32), and the joining kernel adds a row's partials in the order of the keys.
//
// Order of the jobs: first those of the shared prefix (by key head, then row block over all the call's
// tokens), then sequence by sequence its own keys (by key head, then row block).  When the call is FUSED
// (see attn_fused) there are no prefix jobs and every job walks the prefix's tiles before its own.
//
// A block is `tiles_per_block` row tiles of `tile_rows` rows.  With ALT, a block that fits in one row tile
// is worked on by two groups of warps that take its key tiles in turn, each with its own m, l and output:
// two partials (streams 0 and 1) per segment.
#pragma once

#include "common.cuh"

namespace griffin {

struct AttnPlan {
    const int *q_start, *seq_len, *page_table, *prefix_pages;
    int n_seq, n_tokens, table_stride, prefix_len, n_pages;
    int page_shift;
    int hq, hkv, group, d;
    int may_queue;         // whether the kernel takes jobs from a queue (and the call is fused)
    int fused, alt, by_token;  // by_token: how partials by row are numbered (attn_part_row)
    int tile_tokens;       // tokens per row tile
    int tiles_per_block;   // row tiles per block
    int block_tokens;      // tile_tokens * tiles_per_block
    int kt_shift;          // keys per tile: 1 << kt_shift
    uint32_t group_inv;    // ceil(2^16 / group): x / group = x * group_inv >> 16 for x * group < 2^16
    int prefix_tiles;      // ceil(prefix_len / keys per tile)
    int prefix_blocks;     // row blocks per key head of the prefix jobs (0 when fused or without a prefix)
    int grid;
    float scale_log2;      // scale * log2(e): logits in units of log2
    void *ws;
    // scratch (see attn_scratch)
    int *bases;            // [n_seq + 3]: first own tile of each sequence, W, jobs, longest job
    unsigned int *queue;   // how many jobs of a queued call have been taken (in the workspace's header; 0 between calls)
    struct CutJob *cuts;   // [grid]: the cut block that ends in the CTA's first segment, for the joining kernel
    float *own, *pre;      // partials by row: [2 streams][rows]: m and l, then the outputs
    float *cta;            // partials by CTA: [grid][2: continued from before / going on behind][2 * tile_rows]
    long long own_rows;
    int cta_rows;          // 2 * tile_rows
};

// Rows of one partial array: (m, l) pairs for all rows, then D outputs for all rows.
__host__ __device__ inline float *part_ml(float *base, long long row) { return base + 2 * row; }
__host__ __device__ inline float *part_o(float *base, long long rows, long long row, int d) { return base + 2 * rows + row * d; }

// Whether the call's rows are fewer than 128 per sequence and key head.
__host__ __device__ inline bool attn_by_token(int n_seq, int n_tokens, int group) {
    return (long long)n_tokens * group <= (long long)n_seq * 128;
}

// Whether each sequence walks the prefix itself.  Read once for the batch, the prefix costs two partials per
// row; read by each sequence it costs its bytes n_seq times.  With 128 rows or more per sequence and key head
// the second reading is no longer what bounds the call (the matrix unit's tiles are full either way), and
// nothing has to be joined.
__host__ __device__ inline bool attn_fused(int n_seq, int n_tokens, int group, int prefix_len) {
    return n_seq == 1 || prefix_len == 0 || !attn_by_token(n_seq, n_tokens, group);
}

// row (of a block) / query heads per key head
__device__ __forceinline__ int attn_row_token(const AttnPlan &p, int row) { return (int)(((uint32_t)row * p.group_inv) >> 16); }

__host__ __device__ inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

static __device__ __noinline__ void attn_bad(void *ws, int where) { raise_status(ws, DEV_STATUS_BAD_INDEX, where); }

struct AttnSeq {
    int q0, nq, len;  // first new token, how many, own tokens
};
// A sequence's lengths as the arrays q_start (a, b) and seq_len have them, held to what the call can hold (and to 2^30 own
// tokens, as a prefix is: places and tile counts stay in 32 bits).
__device__ __forceinline__ AttnSeq attn_seq_of(const AttnPlan &p, int a, int b, int len) {
    AttnSeq r;
    const long long cap = min((long long)p.table_stride << p.page_shift, (long long)GRIFFIN_MAX_ATTN_TOKENS);
    const bool bad = a < 0 || b < a || b > p.n_tokens || len < 0 || len > cap;
    a = min(max(a, 0), p.n_tokens);
    b = min(max(b, a), p.n_tokens);
    if (bad) attn_bad(p.ws, 41);
    r.q0 = a;
    r.nq = b - a;
    r.len = (int)min((long long)max(len, 0), cap);
    return r;
}
__device__ __forceinline__ AttnSeq attn_seq(const AttnPlan &p, int s) {
    return attn_seq_of(p, __ldg(p.q_start + s), __ldg(p.q_start + s + 1), __ldg(p.seq_len + s));
}
// Key tiles of row block b of a sequence: the prefix's (fused) and its own up to the last row's place.
__device__ __forceinline__ int attn_block_tiles(const AttnPlan &p, const AttnSeq &q, int b) {
    const int last = q.len - q.nq + min(q.nq, (b + 1) * p.block_tokens);  // own tokens that the block's last row sees
    return (p.fused ? p.prefix_tiles : 0) + ((max(last, 0) + (1 << p.kt_shift) - 1) >> p.kt_shift);
}

// The shares: G CTAs have work (every one of them at least a tile), the first `more` of them each a tile more.
struct AttnShares {
    int W, G, each, more;
    __device__ __forceinline__ AttnShares(int W_, int grid) : W(W_), G(W_ < grid ? W_ : grid), each(0), more(0) {
        if (G > 0) {
            each = (int)((uint32_t)W / (uint32_t)G);
            more = W - each * G;
        }
    }
    __device__ __forceinline__ int first(int c) const { return c * each + min(c, more); }   // first tile of CTA c
    __device__ __forceinline__ int cta_of(int g) const {                                    // the CTA that has tile g
        const int lead = more * (each + 1);
        return g < lead ? (int)((uint32_t)g / (uint32_t)(each + 1)) : more + (int)((uint32_t)(g - lead) / (uint32_t)each);
    }
};

// What says where a job's partials are.
struct PartJob {
    int seq;              // -1: prefix job
    int head;             // key head
    int tok0;             // first token of its rows
    bool alt;
};
struct AttnJob : PartJob {
    int g0, g1;           // its tiles
    int n_tok;            // its rows' tokens
    int block;            // row block of its sequence
    int seen0;            // own tokens that the first of them sees (the next one sees one more)
    int rows;             // n_tok * group
    int own_len;          // own tokens of the sequence that any row sees
};

__device__ __forceinline__ AttnJob attn_prefix_job(const AttnPlan &p, int head, int b) {
    AttnJob j;
    j.seq = -1;
    j.head = head;
    j.block = b;
    j.tok0 = b * p.block_tokens;
    j.n_tok = min(p.block_tokens, p.n_tokens - j.tok0);
    j.g0 = (head * p.prefix_blocks + b) * p.prefix_tiles;
    j.g1 = j.g0 + p.prefix_tiles;
    j.seen0 = 0;
    j.own_len = 0;
    j.rows = j.n_tok * p.group;
    j.alt = p.alt && j.n_tok <= p.tile_tokens;
    return j;
}

__device__ __forceinline__ AttnJob attn_own_job(const AttnPlan &p, const AttnSeq &q, int s, int head, int b, int g0) {
    AttnJob j;
    j.g0 = g0;
    j.g1 = g0 + attn_block_tiles(p, q, b);
    j.seq = s;
    j.head = head;
    j.block = b;
    j.tok0 = q.q0 + b * p.block_tokens;
    j.n_tok = min(p.block_tokens, q.nq - b * p.block_tokens);
    j.seen0 = q.len - q.nq + b * p.block_tokens + 1;
    j.own_len = max(j.seen0 + j.n_tok - 1, 0);
    j.rows = j.n_tok * p.group;
    j.alt = p.alt && j.n_tok <= p.tile_tokens;
    return j;
}

// Sum over blocks b0 .. b1 - 1 of a sequence of their key tiles, by a whole warp.
__device__ __forceinline__ long long attn_sum_tiles(const AttnPlan &p, const AttnSeq &q, int b0, int b1) {
    long long n = 0;
#pragma unroll 1
    for (int b = b0 + (threadIdx.x & 31); b < b1; b += 32) n += attn_block_tiles(p, q, b);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    return n;
}

// What the CTAs know of a call after the scan.
struct AttnTotals {
    int W;         // tiles; -1: more than the kernels can count
    int jobs;      // of the sequences
    bool queued;   // whether jobs are handed out whole, from a queue
};
constexpr int ATTN_QUEUE_JOBS = 3;   // jobs per CTA from which a call is queued

// First tile of every sequence into bases[0 .. n_seq] (shared memory), by all threads of the CTA; bases[n_seq] is
// the number of tiles of the call, and the two entries behind it say how many jobs there are and how long the longest is.
// The first CTA also leaves them in the scratch for the joining kernel.  A call of 2^31 tiles or more is not run: its
// number of tiles is -1, at which the kernels return, and the status word is raised.  (Tiles are counted by key head and row
// block: one prompt of 32 heads over 8, 128 wide, gets there with 2.1 million tokens in bf16, with 0.74 million in fp32.)
__device__ __forceinline__ void attn_scan(const AttnPlan &p, int *bases) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const long long most = 1ll << 31;
    // sequences of one row block (steps of a generation): a thread each; the others: a warp each
#pragma unroll 1
    for (int s = threadIdx.x; s < p.n_seq; s += blockDim.x) {
        const AttnSeq q = attn_seq(p, s);
        if (q.nq <= p.block_tokens) {
            const long long n = q.nq > 0 ? (long long)attn_block_tiles(p, q, 0) * p.hkv : 0;
            bases[s] = n < most ? (int)n : -1;
        }
    }
    if (p.n_tokens > p.block_tokens) {
#pragma unroll 1
        for (int s = warp; s < p.n_seq; s += warps) {
            const AttnSeq q = attn_seq(p, s);
            if (q.nq <= p.block_tokens) continue;
            const long long n = attn_sum_tiles(p, q, 0, ceil_div(q.nq, p.block_tokens)) * p.hkv;
            if (lane == 0) bases[s] = n < most ? (int)n : -1;
        }
    }
    __syncthreads();
    if (warp == 0) {
        long long sum = (long long)p.hkv * p.prefix_blocks * p.prefix_tiles;
        bool bad = false;
        int jobs = 0, longest = 0;
#pragma unroll 1
        for (int s0 = 0; s0 < p.n_seq; s0 += 32) {
            const int s = s0 + lane;
            const long long mine = s < p.n_seq ? bases[s] : 0;
            bad |= mine < 0;
            if (mine > 0 && p.n_tokens > p.block_tokens) {  // (a call of one row block has nothing to queue)
                const AttnSeq q = attn_seq(p, s);
                const int nb = ceil_div(q.nq, p.block_tokens);
                jobs += nb;
                longest = max(longest, attn_block_tiles(p, q, nb - 1));
            }
            long long upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            if (s < p.n_seq) bases[s] = (int)(sum + upto - mine);
            sum += __shfl_sync(0xffffffffu, upto, 31);
        }
        bad = __any_sync(0xffffffffu, bad) || sum >= most;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            jobs += __shfl_xor_sync(0xffffffffu, jobs, o);
            longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
        }
        if (lane == 0) {
            bases[p.n_seq] = bad ? -1 : (int)sum;
            bases[p.n_seq + 1] = jobs * p.hkv;
            bases[p.n_seq + 2] = longest;
            if (bad) attn_bad(p.ws, 43);
        }
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int s = threadIdx.x; s <= p.n_seq + 2; s += blockDim.x) p.bases[s] = bases[s];
}
// Whether a call's jobs are handed out whole.  Cut shares are even to a tile, but every cut costs two partials of a
// block, written and read again.  With several jobs per CTA and none of them longer than a fair share, whole jobs are taken
// from a queue, the longest of a sequence first: with one sequence that comes within a short job of even, with several
// within the last sequence's longest.  Queue / cut shares, us a pass, 32 heads over 8: a 4096-token prompt 150 / 215, 8 of 2048
// tokens 275 / 358, 64 of 256 110 / 171, 512 of 64 192 / 239.  Only fused calls: the others have partials to join anyway.
__device__ __forceinline__ AttnTotals attn_totals(const AttnPlan &p, const int *bases) {
    AttnTotals t;
    t.W = bases[p.n_seq];
    t.jobs = bases[p.n_seq + 1];
    t.queued = p.may_queue && t.jobs >= ATTN_QUEUE_JOBS * p.grid && (long long)bases[p.n_seq + 2] * p.grid <= t.W;
    return t;
}

// (Not inlined: the schedule's code would otherwise be most of a kernel's, and instruction fetches its time.)
// The job that has tile g (one exists: g < bases[n_seq]); by a whole warp.
static __device__ __noinline__ AttnJob attn_find(const AttnPlan &p, const int *bases, int g) {
    if (g < bases[0]) {
        const int hb = (int)((uint32_t)g / (uint32_t)p.prefix_tiles), head = (int)((uint32_t)hb / (uint32_t)p.prefix_blocks);
        return attn_prefix_job(p, head, hb - head * p.prefix_blocks);
    }
    int lo = 0, hi = p.n_seq;  // bases[lo] <= g < bases[hi]
#pragma unroll 1
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (bases[mid] <= g) lo = mid; else hi = mid;
    }
    const AttnSeq q = attn_seq(p, lo);
    const int per_head = (int)((uint32_t)(bases[lo + 1] - bases[lo]) / (uint32_t)p.hkv);
    const int head = (int)((uint32_t)(g - bases[lo]) / (uint32_t)per_head);
    const int lane = threadIdx.x & 31;
    int at = bases[lo] + head * per_head;
#pragma unroll 1
    for (int b0 = 0;; b0 += 32) {   // 32 blocks at a time
        const int b = b0 + lane, n = b * p.block_tokens < q.nq ? attn_block_tiles(p, q, b) : 0;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned here = __ballot_sync(0xffffffffu, g < at + upto);
        if (here != 0) {
            const int first = __ffs(here) - 1;
            return attn_own_job(p, q, lo, head, b0 + first, at + __shfl_sync(0xffffffffu, upto - n, first));
        }
        at += __shfl_sync(0xffffffffu, upto, 31);
    }
}
// Where a CTA's last job from the queue was: its sequence, and the jobs of the sequences in front of it.
struct AttnQueueAt {
    int seq, before;
};
// Job i of a queued call: sequence by sequence, its row blocks from the last (the longest) to the first, each under
// every key head; by a whole warp.  A CTA's jobs ascend, so it goes on from its last one's sequence, 32 sequences at a time:
// it passes each of them once, not once a job.
static __device__ __noinline__ AttnJob attn_queued(const AttnPlan &p, int i, AttnQueueAt &at) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (;;) {
        AttnSeq q{};
        int nb = 0;   // (a sequence that sees nothing has no jobs)
        if (at.seq + lane < p.n_seq) {
            q = attn_seq(p, at.seq + lane);
            nb = ceil_div(q.nq, p.block_tokens);
            if (nb > 0 && attn_block_tiles(p, q, nb - 1) == 0) nb = 0;
        }
        int upto = nb * p.hkv;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned here = __ballot_sync(0xffffffffu, i < at.before + upto);
        if (here != 0) {
            const int f = __ffs(here) - 1;
            at.before += __shfl_sync(0xffffffffu, upto - nb * p.hkv, f);
            at.seq += f;
            nb = __shfl_sync(0xffffffffu, nb, f);
            q = AttnSeq{__shfl_sync(0xffffffffu, q.q0, f), __shfl_sync(0xffffffffu, q.nq, f), __shfl_sync(0xffffffffu, q.len, f)};
            const int of = i - at.before, k = (int)((uint32_t)of / (uint32_t)p.hkv);
            AttnJob j = attn_own_job(p, q, at.seq, of - k * p.hkv, nb - 1 - k, 0);
            j.alt = false;   // (its result is not joined with another)
            return j;
        }
        at.before += __shfl_sync(0xffffffffu, upto, 31);
        at.seq += 32;
    }
}
// The job behind j, whose first tile is j.g1 < bases[n_seq].
static __device__ __noinline__ AttnJob attn_next(const AttnPlan &p, const int *bases, const AttnJob &j) {
    int s = j.seq, head = j.head, b = j.block + 1;
    if (s < 0) {
        if (j.g1 < bases[0]) return b < p.prefix_blocks ? attn_prefix_job(p, head, b) : attn_prefix_job(p, head + 1, 0);
        s = 0;
        head = b = 0;
        while (bases[s + 1] == bases[s]) ++s;
    }
    AttnSeq q = attn_seq(p, s);
    if (b * p.block_tokens >= q.nq) {
        b = 0;
        if (++head == p.hkv) {
            head = 0;
            do ++s; while (bases[s + 1] == bases[s]);
            q = attn_seq(p, s);
        }
    }
    while (attn_block_tiles(p, q, b) == 0) ++b;  // (only in front of blocks that have some)
    return attn_own_job(p, q, s, head, b, j.g1);
}

// Whether a whole job's result goes straight to the output (no other partial of its rows exists).
__device__ __forceinline__ bool attn_direct(const AttnPlan &p, const AttnJob &j, bool whole) {
    return whole && !j.alt && p.fused;
}
// Row of `own` / `pre` for row r of a job.  Either every row (token and query head) has a place, or, where that
// is less, 128 rows of every sequence and key head: then only one-tile blocks are kept there, of which a
// sequence has one at most.  (A call that is not fused is by token: that is the same comparison.)
__device__ __forceinline__ long long attn_part_row(const AttnPlan &p, const PartJob &j, int r) {
    if (!p.by_token) return (long long)(j.seq * p.hkv + j.head) * 128 + r;
    return (long long)(j.tok0 + attn_row_token(p, r)) * p.hq + j.head * p.group + (r - attn_row_token(p, r) * p.group);
}

// Where the first segment of a job (the one with its first tile) leaves its partials: by row, or with the
// CTA when a block of several row tiles is cut in a fused call.
__device__ __forceinline__ bool attn_first_by_row(const AttnPlan &p, const PartJob &j) { return j.alt || !p.fused; }

// A block of several row tiles that was cut in a fused call, noted by the CTA that has its last tile.
struct __align__(16) CutJob {
    int head, tok0, rows, c0;   // rows 0: none; c0: the CTA with its first tile
};
__device__ __forceinline__ void attn_note_cut(const AttnPlan &p, const AttnShares &sh, const AttnJob &j, int g, int stop) {
    const bool cut = g > j.g0 && stop == j.g1 && !attn_first_by_row(p, j);
    p.cuts[blockIdx.x] = CutJob{j.head, j.tok0, cut ? j.rows : 0, cut ? sh.cta_of(j.g0) : 0};
}

}  // namespace griffin
