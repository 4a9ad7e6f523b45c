// Host-side launchers of the operators around the FF block (arguments already validated in api_layer.cu).
#pragma once

#include "launch.h"

namespace griffin {

griffin_status launch_norm_residual(const griffin_norm_desc *desc, const griffin_norm_weights *w, int T, const void *y,
                                    int64_t ld_y, const void *gate, int64_t ld_gate, const void *res, int64_t ld_res,
                                    void *res_out, int64_t ld_res_out, void *h, int64_t ld_h, cudaStream_t stream);

griffin_status launch_kv_append(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                const griffin_kv_cache *cache, const griffin_rope *rope, const void *q, int64_t ld_q,
                                const void *k, int64_t ld_k, const void *v, int64_t ld_v, void *q_out, int64_t ld_q_out,
                                void *ws, cudaStream_t stream);

// Scratch of griffin_attn_prefix behind the workspace's header, on a 32-byte boundary.
size_t attn_scratch_bytes(const griffin_attn_desc *desc, int n_tokens, int n_seq);
griffin_status launch_attn_prefix(const griffin_attn_desc *desc, const griffin_attn_batch *batch,
                                  const griffin_kv_cache *cache, const void *q, int64_t ld_q, void *out, int64_t ld_out,
                                  uint8_t *scratch, void *ws, cudaStream_t stream);

}  // namespace griffin
