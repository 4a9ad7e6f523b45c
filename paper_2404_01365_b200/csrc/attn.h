// What the attention kernels get beside the plan, and their launchers.
#pragma once

#include "attn_plan.cuh"
#include "layer.h"

namespace griffin {

struct AttnData {
    const void *q, *k, *v;
    void *out;
    long long ld_q, ld_out, stride_page, stride_head, stride_token;
};

// How a kernel cuts its work (see attn_plan.cuh).
struct AttnShape {
    int tile_rows, tiles_per_block, kt, alt;
};

AttnShape attn_simt_shape(int head_dim);
AttnShape attn_tc_shape(int head_dim);
griffin_status launch_attn_tc(const AttnPlan &plan, const AttnData &data, cudaStream_t stream);  // bf16
griffin_status launch_attn_simt(const AttnPlan &plan, const AttnData &data, cudaStream_t stream);  // fp32

}  // namespace griffin
