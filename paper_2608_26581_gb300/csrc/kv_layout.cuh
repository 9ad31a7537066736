// kv_layout.cuh -- places in the paged 4-bit cache and the decoding of its
// codes to f16.  The layout is the order in which the lanes of an
// mma.m16n8k16 want their operands (include/rfq.h states it for users):
//   a K row holds the 4-byte words (8 codes) of its 32-element sub-blocks b
//   transposed, word (c, b): lane c of a quad takes its words of all
//   sub-blocks with one load, and every MMA stays inside one scale block;
//   16 V tokens form a tile whose piece (h, g, c, j) is the dimensions
//   g D/8 .. of token 8 h + 2 c + j: lane (g, c) takes two tokens at once.
#pragma once

#include <cuda_fp16.h>
#include <cstdint>

#include "internal.h"
#include "mxfp4_math.cuh"

namespace rfq {

// Bytes per (page, head) of codes and of scales.
__host__ __device__ inline int64_t kv_code_bytes(int page_size, int D) { return (int64_t)page_size * (D / 2); }
__host__ __device__ inline int kv_token_scale_bytes(int fmt, int D) { return fmt == RFQ_FMT_HIF4 ? D / 16 : D / 32; }

// Byte offset, inside its (page, head), of the word of dimensions
// 32 b + 8 c .. + 7 of a token's K row.
__host__ __device__ inline int64_t kv_k_word(int tok, int b, int c, int D)
{
    return (int64_t)tok * (D / 2) + (c * (D / 32) + b) * 4;
}

// Byte offset of the piece (dimensions g D/8 .. + D/8 - 1) of a V token.
__host__ __device__ inline int64_t kv_v_piece(int tok, int g, int D)
{
    return (int64_t)(tok >> 4) * (8 * D) +
           ((((tok >> 3) & 1) * 8 + g) * 4 + ((tok >> 1) & 3)) * (D / 8) + (tok & 1) * (D / 16);
}

// Eight E2M1 codes -> four f16 pairs of their values (exact): pair i holds
// elements 2i, 2i + 1.
__device__ __forceinline__ void e2m1x8_f16(uint32_t w, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}

// An E4M3 byte with exponent field 0 is its three mantissa bits times 2^-9,
// so an S1P2 code (sign, k) spread to a byte (sign at bit 7, k at bits 0..2)
// converts to +-k 2^-9, exactly.
__device__ __forceinline__ uint32_t s1p2_even_bytes(uint32_t w) // elements 0, 2, 4, 6
{
    return (w & 0x07070707u) | ((w << 4) & 0x80808080u);
}
__device__ __forceinline__ uint32_t s1p2_odd_bytes(uint32_t w) // elements 1, 3, 5, 7
{
    return ((w >> 4) & 0x07070707u) | (w & 0x80808080u);
}
__device__ __forceinline__ uint32_t e4m3x2_f16(uint32_t two_bytes) // the low two bytes
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two_bytes));
    return r;
}
// Eight S1P2 codes -> four f16 pairs of k 2^-9: elements (0, 2), (1, 3),
// (4, 6), (5, 7); the first two pairs share a HiF4 sub-group of four, the
// last two the next one.
__device__ __forceinline__ void s1p2x8_f16(uint32_t w, uint32_t (&h)[4])
{
    const uint32_t e = s1p2_even_bytes(w), o = s1p2_odd_bytes(w);
    h[0] = e4m3x2_f16(e);
    h[1] = e4m3x2_f16(o);
    h[2] = e4m3x2_f16(e >> 16);
    h[3] = e4m3x2_f16(o >> 16);
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// 2^(byte - 127), byte 0 the subnormal 2^-127
__device__ __forceinline__ float e8m0_f32(uint32_t byte) { return __uint_as_float(max(byte << 23, 0x00400000u)); }

// Byte j of a word of E8M0 scales as fp32 (byte 0, a block of zeros or of
// values below 2^-124, as 0)
__device__ __forceinline__ float e8m0_byte(uint32_t w, int j)
{
    return __uint_as_float((j < 3 ? w << (23 - 8 * j) : w >> 1) & 0x7F800000u);
}

// HiF4 macro scale of a metadata word: 2^(E - 48) (1 + M / 4)
__device__ __forceinline__ float hif4_macro_f32(uint32_t meta)
{
    return __uint_as_float((((meta >> 2) & 63u) + 79u) << 23 | (meta & 3u) << 21);
}

// Values of eight codes with elements in order.  MXFP4: scale word or half
// word, sub-block b.  HiF4: meta, group gi of its block.
__device__ __forceinline__ void mxfp4_values(uint32_t code, uint32_t scale, float (&x)[8])
{
    e2m1x8_decode(code, x);
    const float s = e8m0_f32(scale);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x[e] *= s;
}
__device__ __forceinline__ void hif4_values(uint32_t code, uint32_t meta, int gi, float (&x)[8])
{
    // S 2^t / 4, and 2^9 that the codes' conversion leaves out
    const float unit = 128.f * hif4_macro_f32(meta);
    const uint32_t e8 = (meta >> (8 + gi)) & 1u, e16 = meta >> (16 + 2 * gi);
    const float s0 = unit * (float)(1 << (e8 + (e16 & 1u)));
    const float s1 = unit * (float)(1 << (e8 + ((e16 >> 1) & 1u)));
    uint32_t h[4];
    s1p2x8_f16(code, h);                     // elements (0, 2), (1, 3), (4, 6), (5, 7)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[j]));
        const int e = (j >> 1) * 4 + (j & 1);
        x[e] = f.x * (j < 2 ? s0 : s1);
        x[e + 2] = f.y * (j < 2 ? s0 : s1);
    }
}

// Two f16 twos-powers (the same in both halves) of the sub-groups 2 gi and
// 2 gi + 1 of group gi of a HiF4 block: 2^(E1_8 + E1_16).
__device__ __forceinline__ void hif4_pow2_pair(uint32_t meta, int gi, uint32_t &t0, uint32_t &t1)
{
    const uint32_t e8 = (meta >> (8 + gi)) & 1u, e16 = meta >> (16 + 2 * gi);
    t0 = 0x3C003C00u + (e8 + (e16 & 1u)) * 0x04000400u;
    t1 = 0x3C003C00u + (e8 + ((e16 >> 1) & 1u)) * 0x04000400u;
}

// D (fp32, 16 x 8) += A (f16, 16 x 16, row) B (f16, 16 x 8, col)
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same with nothing to add to: D = A B
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

} // namespace rfq
