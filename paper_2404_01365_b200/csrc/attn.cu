// griffin_attn_prefix on the host: the plan's sizes, the scratch, the two launches.
#include <math.h>

#include "attn.h"
#include "attn_join.cuh"

namespace griffin {

constexpr int ATTN_MAX_GRID = 148;  // CTAs at most (one per SM of a B200)

// Whether the kernel for blocks of 8 rows (attn_few.cu) takes a call rather than the tcgen05 one: a CTA has about two of
// the sequences' key heads at most, and the rows that a sequence has on average, and those of a shared prefix, fit one such
// block, or two whose second reading of the keys finds them in L2.
// Both sides, us a pass, few / tcgen05.  One block: 1 sequence of 32 heads behind 512 tokens 12.4 / 14.6, behind 20000 61.3 /
// 65.2; 32 query heads over 8 behind 2048 11.4 / 14.2; 8 sequences of 32 heads behind 2048 (256 key heads) 25.8 / 27.1, of 40
// (320) 31.5 / 30.6; 64 sequences of 32 heads of their own (2048) 90 / 83: the end of a block costs this kernel more.
// Two blocks of a sequence's keys: 4 sequences of 16 tokens of 8 heads 11.7 / 14.6; 4 tokens, 32 heads over 8, 9000 keys (37 MB)
// 20.9 / 21.8, 16000 (66 MB) 27.6 / 26.5; 16 tokens of 32 heads, 2600 keys (43 MB) 23.4 / 22.7.  Two blocks of a shared prefix: 2
// sequences of 2 tokens, 16 heads over 4, 3000 tokens (6 MB) 12.4 / 14.9; 4 sequences, 32 over 8, 2048 (8 MB) 15.2 / 15.1.
// The lengths are on the device, so the rule for two blocks goes by what the page table could hold: with tables that are as
// long as the sequences, as they were for these figures, the limit is where the two kernels meet; with a table for a longer
// context the tcgen05 kernel takes such calls earlier than it need.  (The limit for a prefix stands on these two calls alone.)
constexpr long long FEW_OWN_TWICE = 36ll << 20, FEW_PREFIX_TWICE = 7ll << 20;   // bytes
static bool attn_few(const griffin_attn_desc *desc, const griffin_attn_batch *batch) {
    const long long rows = (long long)batch->n_tokens * (desc->n_q_heads / desc->n_kv_heads), n = batch->n_seq;
    if (desc->dtype != GRIFFIN_DT_BF16 || desc->n_q_heads > 8 * desc->n_kv_heads || n * desc->n_kv_heads > 2 * ATTN_MAX_GRID) return false;
    const long long token = 4ll * desc->n_kv_heads * desc->head_dim, prefix = batch->prefix_len * token;
    const double own = (double)n * batch->table_stride * desc->page_size * token;   // (what the table could hold; past 64 bits for the widest)
    if (n > 1 && prefix > 0 && rows > 8 && (rows > 16 || prefix > FEW_PREFIX_TWICE)) return false;
    return rows <= 8 * n || (rows <= 16 * n && own + (double)prefix <= (double)FEW_OWN_TWICE);
}
// Over a cache held in 4 bits the kernel for blocks of up to 8 rows (attn_few_q4.cu) may give its jobs (a block under a key head, with the
// prefix's keys and the sequence's own) to clusters of CTAs whole: then nothing is left to the joining kernel, which is 4 us, but the
// call waits for its longest job.  us a pass by cluster, - more than are resident at once; cut: the call's tiles dealt out evenly, and joined:
//   jobs  keys   cut     1     2     4     8       jobs  keys   cut     1     2     4
//      1   200  10.7   8.4   9.3   9.3   9.9         40   500  13.1  10.9  10.6     -
//      1  1000  12.7  12.9  11.9  10.2   9.7         40  4000  22.6  27.8  20.1     -
//      1  4000  19.2  26.1  19.0  14.5  12.4         40 16000  38.3  85.9  51.0     -
//      8   500  12.3  10.5  10.3   9.6   9.9         72  1000  16.6  13.6  12.9     -
//      8 16000  21.0  83.0  48.0  29.3  20.3         72  4000  26.4  28.3  21.3     -
//     16  4000  16.0  27.0  19.4  14.9  24.0         80  4000  27.8  28.2     -     -
//     32  1000  13.5  13.4  12.6  10.6     -        128  1000  21.4  14.4     -     -
//     32 16000  33.4  84.8  49.7  32.2     -        128  4000  34.0  30.2     -     -
// (With 16 warps to a CTA; with the 12 that it has now all are 1 to 2 us less.)
// Fitted over 150 calls drawn at random, each timed in every form: base + slope * keys (128 wide) for each cluster, to 1.1 us, and for cut
// calls 13 + 0.0048 * keys * jobs / 148, and 3 more where a prefix is walked apart, to 3.  What is chosen by these takes 0.4 % more than the best
// form on average, 1.16 times as long at worst, where the tables are about as wide as the sequences are long.
// The sequences' lengths are on the device; what the page table could hold stands for them, here and below.  Short sequences in tables for
// a long context are taken by the forms for long ones.  us a pass, tables as wide as need be / for 4096 keys / for 32768: 1 sequence of 32
// heads behind 512, 128 own 8.0 / 8.0 / 12.6; 5 of 8 heads, 500 keys 8.1 / 8.1 / 12.4; 16 of 32 over 8, 200 keys 7.4 / 7.4 / 13.1; fp32, 5
// of 16 over 4 behind 1003 8.6 / 8.6 / 13.7; 6 drafted tokens, 32 over 8, behind 1000 9.5 / 9.5 / 15.2; 6 x 5 drafted, 256 wide 21.4 / 21.3 / 26.2; 4
// pieces of 16, 300 keys 15.8 / 18.1 / 18.0; 48 sequences of 4096 50.1 / 50.3 / 50.3.
struct WholeFit {
    int cluster, most_jobs;
    double base, slope, slack;   // slack: how far a cut call with the fewest jobs, of which each has many parts to join, is above its fit
};
constexpr WholeFit WHOLE_FITS[] = {{1, 148, 7.0, 0.0045, 0.0}, {2, 72, 7.7, 0.00236, 0.0}, {4, 32, 7.6, 0.00128, 0.0}, {8, 8, 7.9, 0.0007, 5.0}};
constexpr double CUT_BASE = 13, CUT_SLOPE = 0.0048 / ATTN_MAX_GRID, CUT_APART = 3;
constexpr int FQ_SHORT_PREFIX = 128;   // (a prefix up to which every sequence walks it itself, below)
// Query heads of a block of that kernel: all of a key head, or an even part of them.  (Groups of a prime number above 8 go one by one, and
// each unpacks the keys: 64 steps of 13 heads over 1, 2048 keys 26.2 us, of 12 17.2; over the cache in bf16 both 23.3.)
static int few_group(const griffin_attn_desc *desc) {
    const int group = desc->n_q_heads / desc->n_kv_heads;
    int n = group < 8 ? group : 8;
    while (group % n != 0) --n;
    return n;
}
struct WholeJobs {
    int jobs, cluster;   // cluster 0: not whole
    double us;
};
static WholeJobs attn_whole(const griffin_attn_desc *desc, const griffin_attn_batch *batch) {
    const int group = few_group(desc), block_tokens = 8 / group;
    const long long n = batch->n_seq, blocks = batch->n_tokens <= n ? n : n + batch->n_tokens / block_tokens, jobs = blocks * (desc->n_q_heads / group);
    // Keys 128 wide: of the longest job, and of all blocks of a cut call, which reads a shared prefix once for 8 rows of the batch.
    const double width = desc->head_dim / 128.0, prefix = batch->prefix_len * width, own = (double)batch->table_stride * desc->page_size * width;
    const bool apart = n > 1 && batch->prefix_len > FQ_SHORT_PREFIX;
    const double keys = prefix + own, shared = apart ? (double)(((long long)batch->n_tokens * group + 7) / 8 * (desc->n_q_heads / group)) : (double)jobs;
    const double cut = CUT_BASE + (apart ? CUT_APART : 0.0) + CUT_SLOPE * (jobs * own + shared * prefix);
    WholeJobs best{0, 0, 0.0};
    for (const WholeFit &f : WHOLE_FITS) {
        const double us = f.base + f.slope * keys;
        if (jobs > f.most_jobs || (best.cluster > 0 && us >= best.us)) continue;
        best = WholeJobs{(int)jobs, us <= cut + f.slack ? f.cluster : 0, us};
    }
    return best;
}
// Whether that kernel takes a call over a cache in 4 bits rather than the tcgen05 one.  It unpacks the keys once for every 8 rows, the
// other once for every 128 (a row tile; two of them share a key tile, but not the softmax).  In keys of a 128-wide head, over
// all jobs, few rows take 2.5e-5 us each on 148 SMs and row tiles 6.5e-5 (of 64-wide heads not less: their softmax is the same); the
// tcgen05 kernel's way to the first and from the last result takes 2 us more, and blocks that are cut, which the joining kernel has
// too few CTAs for, 0.4 us a part (of 128 entries).  500 calls drawn at random (1 to 128 sequences of 1 to 128 tokens, up to 32000 shared and
// 30000 own keys, 64 to 256 wide, 1 to 32 key heads with 1 to 64 query heads each), each timed with both kernels, take 1.0 % more by
// this rule than with the better one each time, at worst 1.5 times as long (with tables that fit, as above).  us a pass, few / tcgen05, query heads over key heads (the
// 128-wide figures of the former with 16 warps to a CTA; 12 take 5 to 15 % less):
//   1 sequence of 1 token, 64 over 8, 5000 keys 14.3 / 19.7;  4 of 4 tokens 38.0 / 32.9;  16 tokens, 32 over 16 28.0 / 24.5
//   24 sequences of 1 token, 64 over 8, 12000 keys 93 / 235;  of 32 tokens, 5000 keys 945 / 190
//   32 over 8 behind 1000 shared, 600 keys, 8 sequences 14.3 / 20.5;  8 over 8 behind 2000, 64 keys, 48 sequences 24.7 / 27.2
//   16 over 2 behind 2000 shared, 5000 keys, 48 sequences 41.9 / 83.3;  8 over 4 behind 8000, 64 keys 36.7 / 26.2
//   256 wide: 64 over 8 behind 2000, 5000 keys, 64 sequences 246 / 558;  16 over 8, 2 tokens behind 2000, 200 keys 69.0 / 55.8
//   cut blocks: 16 tokens, 16 over 1, 12000 keys 31.6 / 54.8, 30000 keys of 64 over 4 143 / 59;  4 tokens, 8 over 1, 5000 keys 256 wide 17.0 / 51.5
// More than 8 query heads a key head go in even parts, each of which unpacks the keys (they are read from L2 but once):
//   32 over 2, 1 sequence, 200 keys 8.6 / 14.5, 12000 18.2 / 19.1;  48 over 4 behind 1000, 2000 keys, 8 sequences 18.1 / 22.3
//   128 over 8, 2000 keys, 64 sequences 89.7 / 172;  9 over 1 behind 8000, 64 keys, 64 sequences 55.8 / 30.5
// In keys of 8 rows: a key of a row tile, the tcgen05 kernel's start, a part of a cut block.
constexpr double FQ_TILE_KEY = 2.5, FQ_START = 80000, FQ_PART = 16500;
static bool attn_few_q4(const griffin_attn_desc *desc, const griffin_attn_batch *batch) {
    const int group = desc->n_q_heads / desc->n_kv_heads;
    if (desc->dtype != GRIFFIN_DT_BF16) return true;   // (the only one for fp32)
    const int part = few_group(desc);
    const double n = batch->n_seq, tokens = batch->n_tokens, rows = tokens * group, prefix = batch->prefix_len, parts = group / part, most = 8 / part;
    const double own = (double)batch->table_stride * desc->page_size, heads = desc->n_kv_heads, width = desc->head_dim / 128.0;
    const double own8 = n * parts * ceil(tokens / (most * n)), own128 = n * ceil(rows / (128 * n));   // blocks, were the sequences equally long
    const double few = heads * width * ((n == 1 || prefix <= FQ_SHORT_PREFIX ? own8 : parts * ceil(tokens / most)) * prefix + own8 * own);
    const AttnShape tc = attn_tc_shape(desc->head_dim);
    const double own_tiles = ceil(own / tc.kt), pre_tiles = ceil(prefix / tc.kt);
    double tcgen05 = FQ_TILE_KEY * heads * fmax(width, 1.0) * tc.kt * (ceil(rows / 128) * pre_tiles + own128 * own_tiles) + FQ_START;
    if (attn_fused(batch->n_seq, batch->n_tokens, group, batch->prefix_len) && (!tc.alt || rows > 128 * n)) {   // (attn_join.cu)
        const double cut = fmin(own_tiles + pre_tiles, ATTN_MAX_GRID / (heads * n * ceil(rows / (128 * tc.tiles_per_block * n))));
        if (cut > 1) tcgen05 += FQ_PART * fmax(width, 1.0) * cut;
    }
    return few <= tcgen05;
}
static AttnShape shape_of(const griffin_attn_desc *desc, bool few, bool q4) {
    if (few && q4) return attn_few_q4_shape();
    if (desc->dtype == GRIFFIN_DT_F32) return attn_simt_shape(desc->head_dim);
    return few ? attn_few_shape(desc->head_dim) : attn_tc_shape(desc->head_dim);
}

struct AttnScratch {
    size_t cuts_off, own_off, pre_off, cta_off, total;  // the bases are at 0
    long long own_rows;
};
// (every size grows with n_tokens and n_seq, so a workspace for the largest call serves the others)
static AttnScratch attn_scratch(const griffin_attn_desc *desc, const AttnShape &sh, long long n_tokens, long long n_seq) {
    AttnScratch s;
    const size_t row = (size_t)(desc->head_dim + 2) * sizeof(float), streams = sh.alt ? 2 : 1;
    const long long by_token = n_tokens * desc->n_q_heads, by_seq = n_seq * desc->n_kv_heads * 128;
    s.own_rows = ((by_token < by_seq ? by_token : by_seq) + 3) / 4 * 4;  // (what follows the rows' m and l, 8 bytes each, is on a 32-byte boundary again)
    s.cuts_off = ((size_t)(n_seq + 3) * 4 + 255) / 256 * 256;
    s.own_off = s.cuts_off + ATTN_MAX_GRID * sizeof(CutJob);
    s.pre_off = s.own_off + streams * s.own_rows * row;
    s.cta_off = s.pre_off + (n_seq > 1 ? streams * s.own_rows * row : 0);
    s.total = s.cta_off + (size_t)ATTN_MAX_GRID * 2 * (2 * sh.tile_rows) * row;
    return s;
}

// (the kernel for few rows over a cache in 4 bits has the scratch of the other one, less than that of fp32)
size_t attn_scratch_bytes(const griffin_attn_desc *desc, int n_tokens, int n_seq) {
    const size_t a = attn_scratch(desc, shape_of(desc, false, false), n_tokens, n_seq).total, b = attn_scratch(desc, shape_of(desc, true, false), n_tokens, n_seq).total;
    return a > b ? a : b;
}

// group: query heads of a block, a part of those of a key head.
static AttnPlan make_plan(const griffin_attn_desc *desc, const griffin_attn_batch *batch, int n_pages, int sms, const AttnShape &sh, int group,
                          uint8_t *scratch, void *ws) {
    AttnPlan p{};
    p.q_start = batch->q_start; p.seq_len = batch->seq_len; p.page_table = batch->page_table;
    p.prefix_pages = batch->prefix_pages;
    p.n_seq = batch->n_seq; p.n_tokens = batch->n_tokens; p.table_stride = batch->table_stride;
    p.prefix_len = batch->prefix_len; p.n_pages = n_pages;
    while ((1 << p.page_shift) < desc->page_size) ++p.page_shift;
    p.hq = desc->n_q_heads; p.hkv = p.hq / group; p.group = group;
    p.group_inv = (65536u + p.group - 1) / p.group;
    p.d = desc->head_dim;
    // (by all of a key head's rows, as the scratch is; the kernel whose groups are parts keeps partials by row by token only)
    p.fused = attn_fused(p.n_seq, p.n_tokens, desc->n_q_heads / desc->n_kv_heads, p.prefix_len);
    p.by_token = attn_by_token(p.n_seq, p.n_tokens, desc->n_q_heads / desc->n_kv_heads);
    p.alt = sh.alt;
    p.tile_tokens = sh.tile_rows / p.group;
    p.tiles_per_block = sh.tiles_per_block;
    p.block_tokens = p.tile_tokens * p.tiles_per_block;
    while ((1 << p.kt_shift) < sh.kt) ++p.kt_shift;
    p.prefix_tiles = ceil_div(p.prefix_len, sh.kt);
    p.prefix_blocks = p.fused ? 0 : ceil_div(p.n_tokens, p.block_tokens);
    p.grid = sms < ATTN_MAX_GRID ? sms : ATTN_MAX_GRID;
    p.scale_log2 = desc->scale * 1.4426950408889634f;
    p.ws = ws;
    p.may_queue = p.fused && desc->dtype == GRIFFIN_DT_BF16 && sh.tiles_per_block * sh.tile_rows >= 128;   // (attn_tc.cu)
    p.queue = &static_cast<WsHeader *>(ws)->queue_attn;
    const AttnScratch s = attn_scratch(desc, sh, p.n_tokens, p.n_seq);
    p.bases = reinterpret_cast<int *>(scratch);
    p.cuts = reinterpret_cast<CutJob *>(scratch + s.cuts_off);
    p.own = reinterpret_cast<float *>(scratch + s.own_off);
    p.pre = reinterpret_cast<float *>(scratch + s.pre_off);
    p.cta = reinterpret_cast<float *>(scratch + s.cta_off);
    p.own_rows = s.own_rows;
    p.cta_rows = 2 * sh.tile_rows;
    return p;
}

static griffin_status launch(const griffin_attn_desc *desc, const griffin_attn_batch *batch, const AttnData &x, int n_pages, bool few,
                             bool q4, uint8_t *scratch, void *ws, cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms <= 0) return GRIFFIN_ERR_CUDA;
    const int group = few && q4 ? few_group(desc) : desc->n_q_heads / desc->n_kv_heads;
    AttnPlan p = make_plan(desc, batch, n_pages, sms, shape_of(desc, few, q4), group, scratch, ws);
    griffin_status st;
    if (few && q4) {
        const WholeJobs whole = attn_whole(desc, batch);
        // A short prefix is walked by every sequence: most jobs then lie in one warp's share and need no joining.  us a pass, each / once for
        // the batch: 24 sequences, 8 key heads, 64 keys in front of 200 14.9 / 17.2, 128 16.0 / 16.6, 256 19.9 / 17.9; 35, 40 key heads, 256 wide,
        // 64 53 / 80, 128 57 / 68, 256 66 / 66.
        if (p.prefix_len <= FQ_SHORT_PREFIX) p.fused = 1, p.prefix_blocks = 0;
        st = launch_attn_few_q4(p, x, desc->dtype, whole.jobs, whole.cluster, stream);
        if (whole.cluster > 0) return st;
    } else {
        st = desc->dtype == GRIFFIN_DT_F32 ? launch_attn_simt(p, x, stream)
             : few                         ? launch_attn_few(p, x, stream)
                                           : launch_attn_tc(p, x, q4, stream);
    }
    return st != GRIFFIN_OK ? st : launch_attn_join(p, desc->dtype, x.out, x.ld_out, stream);
}

griffin_status launch_attn_prefix(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                  const griffin_kv_cache *cache, const void *q, int64_t ld_q, void *out, int64_t ld_out,
                                  uint8_t *scratch, void *ws, cudaStream_t stream) {
    const AttnData x{q, cache->k, cache->v, out, ld_q, ld_out, cache->stride_page, cache->stride_head, cache->stride_token, {}, 1};
    return launch(desc, batch, x, cache->n_pages, attn_few(desc, batch), false, scratch, ws, stream);
}

griffin_status launch_attn_prefix_q4(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                     const griffin_kv_cache_q4 *cache, const void *q, int64_t ld_q, void *out, int64_t ld_out,
                                     uint8_t *scratch, void *ws, cudaStream_t stream) {
    const AttnData x{q, cache->k, cache->v, out, ld_q, ld_out, cache->stride_page, cache->stride_head, 0,
                     q4_layout(desc->head_dim, desc->page_size), desc->n_q_heads / desc->n_kv_heads / few_group(desc)};
    return launch(desc, batch, x, cache->n_pages, attn_few_q4(desc, batch), true, scratch, ws, stream);
}

}  // namespace griffin
