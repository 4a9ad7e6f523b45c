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
static AttnShape shape_of(const griffin_attn_desc *desc, bool few) {
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

size_t attn_scratch_bytes(const griffin_attn_desc *desc, int n_tokens, int n_seq) {
    const size_t a = attn_scratch(desc, shape_of(desc, false), n_tokens, n_seq).total, b = attn_scratch(desc, shape_of(desc, true), n_tokens, n_seq).total;
    return a > b ? a : b;
}

griffin_status launch_attn_prefix(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                  const griffin_kv_cache *cache, const void *q, int64_t ld_q, void *out, int64_t ld_out,
                                  uint8_t *scratch, void *ws, cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms <= 0) return GRIFFIN_ERR_CUDA;
    const bool few = attn_few(desc, batch);
    const AttnShape sh = shape_of(desc, few);
    AttnPlan p{};
    p.q_start = batch->q_start; p.seq_len = batch->seq_len; p.page_table = batch->page_table;
    p.prefix_pages = batch->prefix_pages;
    p.n_seq = batch->n_seq; p.n_tokens = batch->n_tokens; p.table_stride = batch->table_stride;
    p.prefix_len = batch->prefix_len; p.n_pages = cache->n_pages;
    while ((1 << p.page_shift) < desc->page_size) ++p.page_shift;
    p.hq = desc->n_q_heads; p.hkv = desc->n_kv_heads; p.group = p.hq / p.hkv;
    p.group_inv = (65536u + p.group - 1) / p.group;
    p.d = desc->head_dim;
    p.fused = attn_fused(p.n_seq, p.n_tokens, p.group, p.prefix_len);
    p.by_token = attn_by_token(p.n_seq, p.n_tokens, p.group);
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
    p.may_queue = p.fused && desc->dtype == GRIFFIN_DT_BF16 && !few;
    p.queue = &static_cast<WsHeader *>(ws)->queue_attn;
    const AttnScratch s = attn_scratch(desc, sh, p.n_tokens, p.n_seq);
    p.bases = reinterpret_cast<int *>(scratch);
    p.cuts = reinterpret_cast<CutJob *>(scratch + s.cuts_off);
    p.own = reinterpret_cast<float *>(scratch + s.own_off);
    p.pre = reinterpret_cast<float *>(scratch + s.pre_off);
    p.cta = reinterpret_cast<float *>(scratch + s.cta_off);
    p.own_rows = s.own_rows;
    p.cta_rows = 2 * sh.tile_rows;
    const AttnData x{q, cache->k, cache->v, out, ld_q, ld_out, cache->stride_page, cache->stride_head, cache->stride_token};
    const griffin_status st = desc->dtype == GRIFFIN_DT_F32 ? launch_attn_simt(p, x, stream)
                              : few                         ? launch_attn_few(p, x, stream)
                                                            : launch_attn_tc(p, x, stream);
    return st != GRIFFIN_OK ? st : launch_attn_join(p, desc->dtype, out, ld_out, stream);
}

}  // namespace griffin
