// The cache held in 4 bits: its numbers and its layout.
//
// 16 consecutive entries of a head are a group.  With a = max |x| of the group,
//   s    = a / 7 rounded to 4 significant bits (to nearest, ties to even), held to [2^-21, 1792];
//   b    = 8 (e + 21) + m, the byte that stands for s = 2^e (1 + m / 8); 255: an entry is not finite, the group is NaN;
//   code = rint(x / s) held to [-7, 7], plus 8 (x / s: the fp32 quotient).
// Rounding s down by 1/16 at most leaves a / s below 7.5, so within the range of s no entry is off by more than s / 2.
// Why a scale of 4 bits: code - 8 has 3 and s 4, so their product has 7 at most and is exact in bf16 (8), as are 136 s =
// 17 s 8 (17 times 8 .. 15 is below 256) and the tensor cores' products; reading the cache rounds nothing.
//
// A 32-bit word holds 8 entries: entry 2i in bits 4i .. 4i+3, entry 2i + 1 in the same bits of the upper half, so that
// (w >> 4i) & 0x000f000f is two neighbours, in the two halves of a register.  A page holds, for each head, the codes of
// its tokens (D/2 bytes each) and behind them their scales (D/16 bytes each, padded to a multiple of 4).
#pragma once

#include "common.cuh"

namespace griffin {

// Bytes of one head's part of a page.
struct Q4Layout {
    int code_row, scale_row, scale_off;   // a token's codes, a token's scales, where the scales begin
    uint32_t magic;                       // Q4_MAGIC, for q4_pair
};
constexpr uint32_t Q4_MAGIC = 0x43004300u;   // 128 as bf16, twice
__host__ __device__ inline Q4Layout q4_layout(int d, int page_size) {
    return {d / 2, (d + 63) / 64 * 4, page_size * (d / 2), Q4_MAGIC};
}
__host__ __device__ inline long long q4_block_bytes(int d, int page_size) {
    return (long long)page_size * (d / 2 + (d + 63) / 64 * 4);
}

constexpr uint32_t Q4_NAN = 255;
constexpr uint32_t Q4_ZEROS = 0x88888888u;   // eight codes that stand for 0

__device__ __forceinline__ float q4_scale(uint32_t b) {
    return b == Q4_NAN ? __uint_as_float(0x7fc00000u) : __uint_as_float((b << 20) + (106u << 23));
}

// The scale of a group as bf16 in both halves of a register, and -136 times it, for q4_pair.
struct Q4Scale2 {
    uint32_t s, off;
};
__device__ __forceinline__ uint32_t q4_scale_bits(uint32_t b) { return b == Q4_NAN ? 0x7fc0u : (b << 4) + 0x3500u; }
__device__ __forceinline__ uint32_t q4_mul2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t q4_fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ Q4Scale2 q4_scale2(uint32_t lo, uint32_t hi) {   // two scales' bf16 bits
    const uint32_t s = lo | hi << 16;
    return {s, q4_mul2(s, 0xc308c308u)};   // -136
}
// Entries 2i and 2i + 1 of a word as bf16, i = 0 .. 3: the code in the last bits of 128's mantissa is 128 + code, and
// (128 + code) s - 136 s is exact.  A shift, a logical instruction, an fma.  (The magic number is an argument of the kernel,
// Q4Layout::magic: as a constant it would be an immediate like the mask, of which an instruction takes one, and the logical
// instruction became two; they are half of what a kernel that unpacks issues to the integer pipe.)
__device__ __forceinline__ uint32_t q4_pair(uint32_t w, int i, Q4Scale2 s, uint32_t magic) {
    uint32_t x;
    asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xEA;" : "=r"(x) : "r"(w >> (4 * i)), "r"(magic));   // (a & b) | c
    return q4_fma2(x, s.s, s.off);
}

// 16 entries to two words of codes and the scale's byte.
__device__ __forceinline__ uint32_t q4_quantise(const float (&in)[16], uint2 &codes) {
    float f[16], a = 0.f;   // a: NaN if any entry is
#pragma unroll
    for (int j = 0; j < 16; ++j) f[j] = in[j];
#pragma unroll
    for (int j = 0; j < 16; j += 2) asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(a), "f"(fabsf(f[j])), "f"(fabsf(f[j + 1])));
    const bool finite = a < INFINITY;
    const uint32_t q = __float_as_uint(__fdiv_rn(a, 7.f));
    const int t = (int)((q + 0x7ffffu + ((q >> 20) & 1u)) >> 20) - (106 << 3);
    const uint32_t b = (uint32_t)min(max(t, 0), 254);
    const float s = q4_scale(b), r = __frcp_rn(s);
    if (t > 254) {   // (only then can a quotient be 7.5 or more)
#pragma unroll
        for (int j = 0; j < 16; ++j) f[j] = fminf(fmaxf(f[j], -7.f * s), 7.f * s);
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float half[2] = {0.f, 0.f};   // the codes of a half word, less 8 each, as one number
#pragma unroll
        for (int j = 7; j >= 0; --j) {
            // x / s, rounded to nearest (Markstein's theorem: a quotient from the rounded reciprocal, corrected once by its exact
            // remainder; with the 4-bit divisors here it holds for every x, by trial of all mantissas), then to the nearest
            // integer, ties to even.  Nothing overflows: 1 / s is 2^21 at most, and x then below 2^-18.
            const float x = f[8 * i + j], y = x * r, c = __fadd_rn(__fadd_rn(fmaf(fmaf(-y, s, x), r, y), 12582912.f), -12582912.f);
            half[j & 1] = fmaf(half[j & 1], 16.f, c);
        }
        w[i] = __byte_perm(__float_as_uint(half[0] + (8388608.f + 34952.f)), __float_as_uint(half[1] + (8388608.f + 34952.f)), 0x5410);   // 0x8888
    }
    codes = finite ? make_uint2(w[0], w[1]) : make_uint2(Q4_ZEROS, Q4_ZEROS);
    return finite ? b : Q4_NAN;
}

}  // namespace griffin
