// Partials of rows: who writes them where (attn_plan.cuh says why).
#pragma once

#include "attn_plan.cuh"

namespace griffin {

// Place of the partials of one segment and stream: rows' (m, l) and outputs.
struct PartPlace {
    float *ml, *o;
};
__device__ __forceinline__ PartPlace attn_place_row(const AttnPlan &p, const PartJob &j, int stream, int r) {
    float *base = (j.seq < 0 ? p.pre : p.own) + stream * p.own_rows * (p.d + 2);
    const long long row = attn_part_row(p, j, r);
    return {part_ml(base, row), part_o(base, p.own_rows, row, p.d)};
}
// which: 0 = the CTA's first segment, continued from the CTA before; 1 = its last one, going on in the next
__device__ __forceinline__ PartPlace attn_place_cta(const AttnPlan &p, int cta, int which, int row) {
    float *base = p.cta + (long long)(cta * 2 + which) * p.cta_rows * (p.d + 2);
    return {part_ml(base, row), part_o(base, p.cta_rows, row, p.d)};
}
// r: row of the job; stream: 0, or with ALT 0 and 1
__device__ __forceinline__ PartPlace attn_place(const AttnPlan &p, const PartJob &j, bool first, int stream, int r) {
    if (!first) return attn_place_cta(p, blockIdx.x, 0, j.alt ? stream * (p.cta_rows >> 1) + r : r);
    if (attn_first_by_row(p, j)) return attn_place_row(p, j, stream, r);
    return attn_place_cta(p, blockIdx.x, 1, r);
}

griffin_status launch_attn_join(const AttnPlan &plan, int dtype, void *out, long long ld_out, cudaStream_t stream);

}  // namespace griffin
