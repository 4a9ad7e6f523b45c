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

// 2^x to about 2^-22, 0 for -inf
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// two fp32 lanes in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(d)
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)), "l"(*reinterpret_cast<uint64_t *>(&c)));
    return *reinterpret_cast<float2 *>(&d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return *reinterpret_cast<float2 *>(&d);
}
// Whether any of many bf16 is an infinity or NaN: 0 times each, summed, is 0 or NaN.
struct NotFinite8 {
    __nv_bfloat162 sum[4];
    __device__ __forceinline__ NotFinite8() {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = __floats2bfloat162_rn(0.f, 0.f);
    }
    __device__ __forceinline__ void add(uint4 x) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]), __floats2bfloat162_rn(0.f, 0.f), sum[i]);
    }
    __device__ __forceinline__ bool any() const {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= *reinterpret_cast<const uint32_t *>(&sum[i]);
        return (w & 0x7fff7fffu) != 0;
    }
};
// Eight bf16, those that are not finite (their exponent is all ones) set to zero.
__device__ __forceinline__ uint4 finite_or_zero8(uint4 x) {
    const auto two = [](uint32_t w) { return w & ~(((((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu); };
    return make_uint4(two(x.x), two(x.y), two(x.z), two(x.w));
}
// 16 bytes to shared memory, asynchronously; zeros where nothing is there
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

AttnShape attn_simt_shape(int head_dim);
AttnShape attn_tc_shape(int head_dim);
AttnShape attn_few_shape(int head_dim);
griffin_status launch_attn_tc(const AttnPlan &plan, const AttnData &data, cudaStream_t stream);  // bf16
griffin_status launch_attn_few(const AttnPlan &plan, const AttnData &data, cudaStream_t stream);  // bf16, few rows
griffin_status launch_attn_simt(const AttnPlan &plan, const AttnData &data, cudaStream_t stream);  // fp32

}  // namespace griffin
