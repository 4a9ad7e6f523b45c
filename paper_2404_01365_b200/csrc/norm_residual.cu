// The residual stream between two blocks: r' = a res + c act(gate) * post_norm(y), h = pre_norm(r').
//
// A row is held in registers from its one load to its one store: 8 consecutive entries per thread and
// step, fp32.  The mean square of a LayerNorm is taken of the centred values, in a second pass
// over the registers: the one-pass form loses digits when the mean is large.
//
// Bound by memory: 4096 rows of 4096, bf16 with an fp32 residual stream, norms on both sides (201 MB) take 36.5 us, 5.5
// TB/s, where a plain copy of the same bytes takes 33.3; 1001 fp32 rows of 2056 with a gate (41 MB) 10.4 us, one wave of
// CTAs that load, reduce and store in step.  One row of 4096 takes 2.0 us, the launch and four trips to memory.
#include "common.cuh"
#include "layer.h"
#include "vec8.cuh"

namespace griffin {

struct NormParams {
    const void *y, *gate, *res, *pre_w, *pre_b, *post_w, *post_b;
    void *res_out, *h;
    long long ld_y, ld_gate, ld_res, ld_res_out, ld_h;
    int T, d, pre, post, gate_act, wide;  // wide: every row of y, gate, res, res_out and h starts on a 32-byte boundary
    float eps, w0, res_scale, out_scale;
};

// Sum over the row's threads; every one of them gets it.  `red` is a slot of 32 floats that no other
// sum of this kernel uses, so one barrier is enough.
template <bool WARP_ROW> __device__ __forceinline__ float row_sum(float v, float *red) {
    v = warp_sum(v);
    if constexpr (WARP_ROW) {
        return v;
    } else {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = blockDim.x >> 5;
        if (lane == 0) red[warp] = v;
        __syncthreads();
        return warp_sum(lane < n ? red[lane] : 0.f);
    }
}

// x = norm(x), in place.  `mine`: how many of the VPT vectors this thread has.
template <typename T, int VPT, bool WARP_ROW>
__device__ __forceinline__ void norm_row(float (&x)[VPT][8], int kind, const void *w, const void *b, const NormParams &p,
                                         int v0, int step, float (*red)[32]) {
    const int nv = p.d >> 3;
    if (kind == GRIFFIN_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < VPT; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[k][i];  // (vectors beyond the row hold zeros)
        const float mean = row_sum<WARP_ROW>(s, red[0]) / (float)p.d;
#pragma unroll
        for (int k = 0; k < VPT; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] -= mean;
    }
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < VPT; ++k)
        if (v0 + k * step < nv) {
#pragma unroll
            for (int i = 0; i < 8; ++i) q = fmaf(x[k][i], x[k][i], q);
        }
    const float inv = rsqrtf(row_sum<WARP_ROW>(q, red[1]) / (float)p.d + p.eps);
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = v0 + k * step;
        if (v >= nv) continue;
        float f[8];
        load8<T>(w, (long long)v * 8, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[k][i] = x[k][i] * inv * (p.w0 + f[i]);
        if (kind == GRIFFIN_NORM_LAYER && b != nullptr) {
            load8<T>(b, (long long)v * 8, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] += f[i];
        }
    }
}

__device__ __forceinline__ float gate_value(int act, float t) {
    if (act == GRIFFIN_GATE_SIGMOID) return 1.0f / (1.0f + expf(-t));
    if (act == GRIFFIN_GATE_TANH) return tanhf(t);
    return t;
}

// T: storage of y, h, gate, weights; R: of the residual stream.
template <typename T, typename R, int VPT, bool WARP_ROW>
__global__ void __launch_bounds__(WARP_ROW ? 128 : 512, WARP_ROW ? 8 : VPT == 1 ? 4 : VPT == 2 ? 2 : 1) norm_residual_kernel(const __grid_constant__ NormParams p) {
    __shared__ float red[4][32];
    const int row = WARP_ROW ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    const int v0 = WARP_ROW ? threadIdx.x & 31 : threadIdx.x, step = WARP_ROW ? 32 : blockDim.x;
    const int nv = p.d >> 3;
    pdl_launch_dependents();
    pdl_wait_prior_grids();
    if (row >= p.T) return;  // (a whole warp, or nobody)

    float r[VPT][8], u[VPT][8];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = v0 + k * step;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[k][i] = u[k][i] = 0.f;
        if (v >= nv) continue;
        load8<R>(p.res, row * p.ld_res + v * 8, r[k], p.wide);
        if (p.y != nullptr) load8<T>(p.y, row * p.ld_y + v * 8, u[k], p.wide);
    }
    if (p.y != nullptr && p.post != GRIFFIN_NORM_NONE)
        norm_row<T, VPT, WARP_ROW>(u, p.post, p.post_w, p.post_b, p, v0, step, &red[0]);
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = v0 + k * step;
        if (v >= nv) continue;
        if (p.y != nullptr && p.gate != nullptr) {
            float g[8];
            load8<T>(p.gate, row * p.ld_gate + v * 8, g, p.wide);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[k][i] *= gate_value(p.gate_act, g[i]);
        }
        if (p.y != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) r[k][i] = fmaf(p.out_scale, u[k][i], p.res_scale * r[k][i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) r[k][i] *= p.res_scale;
        }
        if (p.res_out != nullptr) store8<R>(p.res_out, row * p.ld_res_out + v * 8, r[k], p.wide);
    }
    if (p.h == nullptr) return;
    if (p.pre != GRIFFIN_NORM_NONE) norm_row<T, VPT, WARP_ROW>(r, p.pre, p.pre_w, p.pre_b, p, v0, step, &red[2]);
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = v0 + k * step;
        if (v < nv) store8<T>(p.h, row * p.ld_h + v * 8, r[k], p.wide);
    }
}

template <typename T, typename R>
static const void *norm_kernel(int nv, int *threads, int *rows_per_cta) {
    // Rows of up to 512 entries belong to a warp each (the statistics are then shuffles only), wider ones to a CTA.  4096
    // bf16 rows of 512: 3.5 us by warps, 4.7 by CTAs (one row: 2.2, 1.8); of 768: 8.4, 5.9; of 1024: 10.3, 7.2.
    *rows_per_cta = nv <= 64 ? 4 : 1;
    if (nv <= 64) {
        *threads = 128;
        if (nv <= 32) return reinterpret_cast<const void *>(norm_residual_kernel<T, R, 1, true>);
        return reinterpret_cast<const void *>(norm_residual_kernel<T, R, 2, true>);
    }
    // as many threads as 512 allow: with half of them and twice the entries each, rows of 4096 take 28.9 us, not 24.5, rows of
    // 8192 41.3, not 31.5 (4096 and 2048 of them, bf16)
    const int vpt = nv <= 512 ? 1 : nv <= 1024 ? 2 : 4;
    *threads = (((nv + vpt - 1) / vpt) + 31) / 32 * 32;
    if (vpt == 1) return reinterpret_cast<const void *>(norm_residual_kernel<T, R, 1, false>);
    if (vpt == 2) return reinterpret_cast<const void *>(norm_residual_kernel<T, R, 2, false>);
    return reinterpret_cast<const void *>(norm_residual_kernel<T, R, 4, false>);
}

griffin_status launch_norm_residual(const griffin_norm_desc *desc, const griffin_norm_weights *w, int T, const void *y,
                                    int64_t ld_y, const void *gate, int64_t ld_gate, const void *res, int64_t ld_res,
                                    void *res_out, int64_t ld_res_out, void *h, int64_t ld_h, cudaStream_t stream) {
    NormParams p{};
    p.y = y; p.gate = gate; p.res = res; p.res_out = res_out; p.h = h;
    p.pre_w = w->pre_w; p.pre_b = w->pre_b; p.post_w = w->post_w; p.post_b = w->post_b;
    p.ld_y = ld_y; p.ld_gate = ld_gate; p.ld_res = ld_res; p.ld_res_out = ld_res_out; p.ld_h = ld_h;
    p.T = T; p.d = desc->d; p.pre = desc->pre_norm; p.post = desc->post_norm; p.gate_act = desc->gate_act;
    const auto on32 = [](const void *q, int64_t ld, int bytes) { return (reinterpret_cast<uintptr_t>(q) & 31) == 0 && ld * bytes % 32 == 0; };
    const int eb = desc->dtype == GRIFFIN_DT_F32 ? 4 : 2, rb = desc->res_dtype == GRIFFIN_DT_F32 ? 4 : 2;
    // (a pointer that is not there is on every boundary)
    p.wide = on32(y, ld_y, eb) && on32(gate, ld_gate, eb) && on32(res, ld_res, rb) && on32(res_out, ld_res_out, rb) && on32(h, ld_h, eb);
    p.eps = desc->eps; p.w0 = desc->weight_offset; p.res_scale = desc->res_scale; p.out_scale = desc->out_scale;
    int threads, rows;
    const void *fn = desc->dtype == GRIFFIN_DT_F32       ? norm_kernel<float, float>(desc->d >> 3, &threads, &rows)
                     : desc->res_dtype == GRIFFIN_DT_F32 ? norm_kernel<__nv_bfloat16, float>(desc->d >> 3, &threads, &rows)
                                                         : norm_kernel<__nv_bfloat16, __nv_bfloat16>(desc->d >> 3, &threads, &rows);
    void *args[] = {&p};
    return launch_maybe_overlapped(fn, dim3((T + rows - 1) / rows), dim3(threads), 0, stream, true, args) == cudaSuccess
               ? GRIFFIN_OK
               : GRIFFIN_ERR_CUDA;
}

}  // namespace griffin
