// Where the tokens of a call are in the paged cache.
#pragma once

#include "common.cuh"

namespace griffin {

// What says so, for kernels that take one CTA (of any grid.y) per TPC tokens.
struct PlaceParams {
    const int *q_start, *seq_len, *page_table;
    void *ws;
    int n_tokens, n_seq, n_pages, table_stride, prefix_len, page_shift;
};
static inline PlaceParams place_params(const griffin_attn_desc *desc, const griffin_attn_batch *batch, int n_pages, void *ws) {
    PlaceParams p{batch->q_start, batch->seq_len, batch->page_table, ws, batch->n_tokens, batch->n_seq, n_pages, batch->table_stride,
                  batch->prefix_len, 0};
    while ((1 << p.page_shift) < desc->page_size) ++p.page_shift;
    return p;
}

struct Place {
    int page;   // -1: none (padding, or it cannot be placed); -2: a row of no sequence
    int slot;   // token of the page
    int pos;    // position: prefix_len + index among the sequence's own tokens
};

// The place of this thread's token, t0 + threadIdx.x of t0 .. t0 + count - 1 (with TPC = 1 every thread's is t0; count <= TPC);
// called by the whole CTA of THREADS threads.  n_pos: positions from there on cannot be placed (-1: all can).
template <int TPC, int THREADS> __device__ __forceinline__ Place place_token(const PlaceParams &p, int t0, int n_pos, int count = TPC) {
    // the first token's sequence: how many sequences end at or before it (empty ones included)
    int seq = 0;
    if (p.n_seq > 1) {
        for (int s0 = 0; s0 < p.n_seq; s0 += THREADS) {
            const int s = s0 + threadIdx.x;
            seq += __syncthreads_count(s < p.n_seq && __ldg(p.q_start + s + 1) <= t0);
        }
    }
    Place r{-2, 0, 0};
    if (TPC > 1 && (int)threadIdx.x >= count) return r;
    const int t = TPC == 1 ? t0 : t0 + threadIdx.x;
    if (TPC > 1 || p.n_seq == 1)  // (otherwise the count above was this token's)
        while (seq < p.n_seq && __ldg(p.q_start + seq + 1) <= t) ++seq;
    int first = t + 1, end = 0, len = 0;   // (three loads in one trip)
    if (seq < p.n_seq && t < p.n_tokens) {
        first = __ldg(p.q_start + seq);
        end = __ldg(p.q_start + seq + 1);
        len = __ldg(p.seq_len + seq);
    }
    if (t >= first) {   // (rows in front of the first sequence's, as those behind the last one's, belong to none)
        const long long own = (long long)len - (end - t);   // index among its own tokens
        const int k = (int)max(min(own, (long long)GRIFFIN_MAX_ATTN_TOKENS), -1ll);
        r.page = -1;
        r.pos = p.prefix_len + k;   // (2^31 - 1 at most for an index below the limit)
        if (k >= 0) {
            const int col = k >> p.page_shift;
            const int page = k < GRIFFIN_MAX_ATTN_TOKENS && col < p.table_stride ? __ldg(p.page_table + (long long)seq * p.table_stride + col) : -1;
            if (page >= 0 && page < p.n_pages && (n_pos < 0 || r.pos < n_pos)) {
                r.page = page;
                r.slot = k & ((1 << p.page_shift) - 1);
            } else if (blockIdx.y == 0 && threadIdx.x < TPC) {
                raise_status(p.ws, DEV_STATUS_BAD_INDEX, 40);
            }
        }
    }
    return r;
}

}  // namespace griffin
