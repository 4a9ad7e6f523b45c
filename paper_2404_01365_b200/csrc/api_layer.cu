// C ABI entry points of the operators around the FF block: host-side validation, then the launchers.
#include <math.h>

#include "common.cuh"
#include "layer.h"

using namespace griffin;

static inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// The attention scratch begins at the first 32-byte boundary behind the header (partials are stored 32 bytes at a time); a
// workspace may begin on any 16-byte boundary.
static inline uint8_t *scratch_of(void *ws) {
    return reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(ws) + WS_HEADER_BYTES + 31) & ~uintptr_t(31));
}
static inline size_t attn_ws_bytes(const griffin_attn_desc *desc, int n_tokens, int n_seq) {
    return WS_HEADER_BYTES + 16 + attn_scratch_bytes(desc, n_tokens, n_seq);
}
static inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static inline int elem_bytes(int dtype) { return dtype == GRIFFIN_DT_F32 ? 4 : 2; }
static inline bool is_dtype(int t) { return t == GRIFFIN_DT_F32 || t == GRIFFIN_DT_BF16; }

static griffin_status check_attn_desc(const griffin_attn_desc *d) {
    if (d == nullptr || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads % d->n_kv_heads != 0) return GRIFFIN_ERR_INVALID_ARG;
    if (!(d->scale > 0.f) || !isfinite(d->scale)) return GRIFFIN_ERR_INVALID_ARG;
    if (!is_dtype(d->dtype) || d->n_q_heads / d->n_kv_heads > GRIFFIN_MAX_HEAD_GROUP) return GRIFFIN_ERR_UNSUPPORTED;
    if (d->head_dim < 64 || d->head_dim > 256) return GRIFFIN_ERR_UNSUPPORTED;
    if (d->head_dim % 8 != 0) return GRIFFIN_ERR_ALIGNMENT;
    if (d->page_size < 8 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)) != 0) return GRIFFIN_ERR_UNSUPPORTED;
    if ((long long)d->n_q_heads * d->head_dim > (1 << 24)) return GRIFFIN_ERR_UNSUPPORTED;
    return GRIFFIN_OK;
}

static griffin_status check_batch(const griffin_attn_batch *b) {
    if (b == nullptr || b->n_seq < 1 || b->n_tokens < 0 || b->prefix_len < 0 || b->table_stride < 0) return GRIFFIN_ERR_INVALID_ARG;
    if (b->q_start == nullptr || b->seq_len == nullptr) return GRIFFIN_ERR_INVALID_ARG;
    if (b->table_stride > 0 && b->page_table == nullptr) return GRIFFIN_ERR_INVALID_ARG;
    if (b->prefix_len > 0 && b->prefix_pages == nullptr) return GRIFFIN_ERR_INVALID_ARG;
    if (b->n_seq > GRIFFIN_MAX_ATTN_SEQ || b->prefix_len > GRIFFIN_MAX_ATTN_TOKENS || b->n_tokens > (1 << 22)) return GRIFFIN_ERR_UNSUPPORTED;
    if (!aligned4(b->q_start) || !aligned4(b->seq_len) || !aligned4(b->page_table) || !aligned4(b->prefix_pages))
        return GRIFFIN_ERR_ALIGNMENT;
    return GRIFFIN_OK;
}

static griffin_status check_cache(const griffin_attn_desc *d, const griffin_kv_cache *c) {
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->n_pages < 1) return GRIFFIN_ERR_INVALID_ARG;
    if (c->stride_page < 0 || c->stride_head < 0 || c->stride_token < d->head_dim) return GRIFFIN_ERR_INVALID_ARG;
    const int unit = 16 / elem_bytes(d->dtype);
    if (c->stride_page % unit != 0 || c->stride_head % unit != 0 || c->stride_token % unit != 0 || !aligned16(c->k) || !aligned16(c->v))
        return GRIFFIN_ERR_ALIGNMENT;
    return GRIFFIN_OK;
}

// A matrix of n rows of `width` entries, `ld` apart.
static griffin_status check_rows(const void *p, int64_t ld, int64_t width, int dtype) {
    if (ld < width) return GRIFFIN_ERR_INVALID_ARG;
    if (!aligned16(p) || ld % (16 / elem_bytes(dtype)) != 0) return GRIFFIN_ERR_ALIGNMENT;
    return GRIFFIN_OK;
}

extern "C" {

griffin_status griffin_norm_residual(const griffin_norm_desc *desc, const griffin_norm_weights *w, int32_t T,
                                     const void *y, int64_t ld_y, const void *gate, int64_t ld_gate,
                                     const void *res, int64_t ld_res, void *res_out, int64_t ld_res_out,
                                     void *h, int64_t ld_h, void *stream) {
    if (desc == nullptr || w == nullptr || res == nullptr || T < 1 || desc->d < 8) return GRIFFIN_ERR_INVALID_ARG;
    if (desc->d % 8 != 0) return GRIFFIN_ERR_ALIGNMENT;
    if (desc->d > GRIFFIN_MAX_NORM_D || !is_dtype(desc->dtype) || !is_dtype(desc->res_dtype)) return GRIFFIN_ERR_UNSUPPORTED;
    if (desc->dtype == GRIFFIN_DT_F32 && desc->res_dtype != GRIFFIN_DT_F32) return GRIFFIN_ERR_UNSUPPORTED;
    if (desc->pre_norm < GRIFFIN_NORM_NONE || desc->pre_norm > GRIFFIN_NORM_LAYER || desc->post_norm < GRIFFIN_NORM_NONE ||
        desc->post_norm > GRIFFIN_NORM_LAYER || desc->gate_act < GRIFFIN_GATE_LINEAR || desc->gate_act > GRIFFIN_GATE_TANH)
        return GRIFFIN_ERR_UNSUPPORTED;
    if (!(desc->eps > 0.f)) return GRIFFIN_ERR_INVALID_ARG;
    if ((gate != nullptr && y == nullptr) || (h == nullptr && res_out == nullptr)) return GRIFFIN_ERR_INVALID_ARG;
    if (desc->pre_norm != GRIFFIN_NORM_NONE && (w->pre_w == nullptr || h == nullptr)) return GRIFFIN_ERR_INVALID_ARG;
    if (desc->post_norm != GRIFFIN_NORM_NONE && (w->post_w == nullptr || y == nullptr)) return GRIFFIN_ERR_INVALID_ARG;
    if (!aligned16(w->pre_w) || !aligned16(w->pre_b) || !aligned16(w->post_w) || !aligned16(w->post_b)) return GRIFFIN_ERR_ALIGNMENT;
    griffin_status st = check_rows(res, ld_res, desc->d, desc->res_dtype);
    if (st == GRIFFIN_OK && res_out != nullptr) st = check_rows(res_out, ld_res_out, desc->d, desc->res_dtype);
    if (st == GRIFFIN_OK && y != nullptr) st = check_rows(y, ld_y, desc->d, desc->dtype);
    if (st == GRIFFIN_OK && gate != nullptr) st = check_rows(gate, ld_gate == 0 ? desc->d : ld_gate, desc->d, desc->dtype);
    if (st == GRIFFIN_OK && h != nullptr) st = check_rows(h, ld_h, desc->d, desc->dtype);
    if (st != GRIFFIN_OK) return st;
    return launch_norm_residual(desc, w, T, y, ld_y, gate, ld_gate, res, ld_res, res_out, ld_res_out, h, ld_h,
                                static_cast<cudaStream_t>(stream));
}

griffin_status griffin_kv_append(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                 const griffin_kv_cache *cache, const griffin_rope *rope,
                                 const void *q, int64_t ld_q, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                 void *q_out, int64_t ld_q_out, void *workspace, void *stream) {
    griffin_status st = check_attn_desc(desc);
    if (st == GRIFFIN_OK) st = check_batch(batch);
    if (st == GRIFFIN_OK) st = check_cache(desc, cache);
    if (st != GRIFFIN_OK) return st;
    if (k == nullptr || v == nullptr || (q == nullptr) != (q_out == nullptr)) return GRIFFIN_ERR_INVALID_ARG;
    if (rope != nullptr) {
        if (rope->table == nullptr || rope->n_pos < 1 || rope->rot_dim < 16 || rope->rot_dim > desc->head_dim) return GRIFFIN_ERR_INVALID_ARG;
        if (rope->style != GRIFFIN_ROPE_HALF && rope->style != GRIFFIN_ROPE_PAIRS) return GRIFFIN_ERR_UNSUPPORTED;
        if (rope->rot_dim % 16 != 0 || !aligned16(rope->table)) return GRIFFIN_ERR_ALIGNMENT;
    }
    const int64_t wq = (int64_t)desc->n_q_heads * desc->head_dim, wk = (int64_t)desc->n_kv_heads * desc->head_dim;
    if (q != nullptr) st = check_rows(q, ld_q, wq, desc->dtype);
    if (st == GRIFFIN_OK && q != nullptr) st = check_rows(q_out, ld_q_out, wq, desc->dtype);
    if (st == GRIFFIN_OK) st = check_rows(k, ld_k, wk, desc->dtype);
    if (st == GRIFFIN_OK) st = check_rows(v, ld_v, wk, desc->dtype);
    if (st == GRIFFIN_OK && !aligned16(workspace)) st = GRIFFIN_ERR_ALIGNMENT;
    if (st != GRIFFIN_OK || batch->n_tokens == 0) return st;
    return launch_kv_append(desc, batch, cache, rope, q, ld_q, k, ld_k, v, ld_v, q_out, ld_q_out, workspace,
                            static_cast<cudaStream_t>(stream));
}

size_t griffin_attn_workspace_bytes(const griffin_attn_desc *desc, int32_t n_tokens_max, int32_t n_seq_max) {
    if (check_attn_desc(desc) != GRIFFIN_OK || n_tokens_max < 0 || n_seq_max < 1) return 0;
    return attn_ws_bytes(desc, n_tokens_max, n_seq_max);
}

griffin_status griffin_attn_prefix(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                   const griffin_kv_cache *cache, const void *q, int64_t ld_q, void *out, int64_t ld_out,
                                   void *workspace, size_t ws_bytes, void *stream) {
    griffin_status st = check_attn_desc(desc);
    if (st == GRIFFIN_OK) st = check_batch(batch);
    if (st == GRIFFIN_OK) st = check_cache(desc, cache);
    if (st != GRIFFIN_OK) return st;
    if (q == nullptr || out == nullptr) return GRIFFIN_ERR_INVALID_ARG;
    const int64_t wq = (int64_t)desc->n_q_heads * desc->head_dim;
    st = check_rows(q, ld_q, wq, desc->dtype);
    if (st == GRIFFIN_OK) st = check_rows(out, ld_out, wq, desc->dtype);
    if (st != GRIFFIN_OK) return st;
    if (workspace == nullptr) return GRIFFIN_ERR_WORKSPACE;
    if (!aligned16(workspace)) return GRIFFIN_ERR_ALIGNMENT;
    if (ws_bytes < attn_ws_bytes(desc, batch->n_tokens, batch->n_seq)) return GRIFFIN_ERR_WORKSPACE;
    if (batch->n_tokens == 0) return GRIFFIN_OK;
    return launch_attn_prefix(desc, batch, cache, q, ld_q, out, ld_out, scratch_of(workspace), workspace,
                              static_cast<cudaStream_t>(stream));
}

}  // extern "C"
