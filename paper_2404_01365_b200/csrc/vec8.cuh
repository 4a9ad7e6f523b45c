// Eight consecutive elements of a row, as fp32: one 16-byte access (bf16) or two (fp32).
#pragma once

#include "common.cuh"

namespace griffin {

template <typename T> __device__ __forceinline__ void load8(const void *base, long long at, float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        Elem<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4 *>(static_cast<const T *>(base) + at), f);
    } else {
        const float4 *p = reinterpret_cast<const float4 *>(static_cast<const T *>(base) + at);
        const float4 a = p[0], b = p[1];
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
}
template <typename T> __device__ __forceinline__ void store8(void *base, long long at, const float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(static_cast<T *>(base) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        float4 *p = reinterpret_cast<float4 *>(static_cast<T *>(base) + at);
        p[0] = make_float4(f[0], f[1], f[2], f[3]);
        p[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
}

// The same where the caller knows whether the address is on a 32-byte boundary: then fp32 takes one access as well.
template <typename T> __device__ __forceinline__ void load8(const void *base, long long at, float (&f)[8], bool wide) {
    if constexpr (sizeof(T) == 4) {
        if (wide) {
            asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7])
                         : "l"(static_cast<const T *>(base) + at));
            return;
        }
    }
    load8<T>(base, at, f);
}
template <typename T> __device__ __forceinline__ void store8(void *base, long long at, const float (&f)[8], bool wide) {
    if constexpr (sizeof(T) == 4) {
        if (wide) {
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<T *>(base) + at), "f"(f[0]),
                         "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7])
                         : "memory");
            return;
        }
    }
    store8<T>(base, at, f);
}

}  // namespace griffin
