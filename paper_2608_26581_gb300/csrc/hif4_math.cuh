// hif4_math.cuh -- HiF4 quantization arithmetic (Sec. 3.3): the macro scale of
// a 64-element block and the codes of one 8-element group, shared by the
// HiF4 quantizers and the 4-bit cache.
#pragma once

#include <cstdint>

#include "mxfp4_math.cuh"

namespace rfq {

__device__ __forceinline__ float ue6m2_value(int E, int M) // 2^(E-48) (1 + M/4), E in [0, 63]
{
    return __uint_as_float(((uint32_t)(E - 48 + 127) << 23) | ((uint32_t)M << 21));
}

// Smallest UE6M2 byte with 7 * value >= amax (amax > 0), clamped to [0, 255].
// With amax = sig 2^ea (sig in [1, 2)), the candidates 7 (1 + M/4) 2^(E-48)
// in increasing order are, for E - 48 = ea - 3, sig x {0.875, 1.09375,
// 1.3125, 1.53125} and then, for E - 48 = ea - 2, {1.75, 2.1875, ...}; so
// the answer follows from the significand bits of amax alone (thresholds
// 0.09375, 0.3125, 0.53125 and 0.75 of the fraction: 0x0C0000, 0x280000,
// 0x440000, 0x600000 in the 23-bit field), then the E range [0, 63].
__device__ __forceinline__ int hif4_scale_byte(float amax)
{
    const uint32_t b = __float_as_uint(amax);
    if (b < 0x00800000u)   // a subnormal amax is below every 7 S: byte 0
        return 0;
    const uint32_t f = b & 0x7FFFFFu;
    const int e0 = (int)(b >> 23) - 127 - 3 + 48;   // E of the first candidate row
    int E, M;
    if (f <= 0x600000u && e0 >= 0) {
        // first row, M = 1..3, or (E0 + 1, 0)
        M = 1 + (f > 0x0C0000u) + (f > 0x280000u) + (f > 0x440000u);
        E = e0;
        if (M == 4) {
            M = 0;
            E = e0 + 1;
        }
    } else if (e0 >= -1) {
        // second row: (E0 + 1, 0) if sig <= 1.75, else (E0 + 1, 1); with
        // E0 = -1 the first row is out of range and this is the smallest
        E = e0 + 1;
        M = f > 0x600000u ? 1 : 0;
    } else {
        return 0;          // below the smallest macro scale: 2^-48 covers it
    }
    if (E > 63)
        return 255;        // above the largest macro scale: saturate
    return (E << 2) | M;
}

// Quantizes the eight elements x[0..7] of group g (sub-groups 2g, 2g+1) of a
// 64-element block whose macro scale byte sb = (E << 2) | M is given.
// Returns the codes (element i in nibble i) and this group's E1_8 / E1_16
// bits (placed at their final metadata positions); `deq` receives the
// dequantized values.
//
// A sub-group with exponent ex has the step 0.25 S 2^ex = 2^(E - 50 + ex)
// (1 + M/4), formed from its bits, and its reciprocal is 2^(50 - E - ex)
// 4 / (4 + M): rounded to fp32 that is the power of two times RN(4 / (4 + M))
// (scaling by a power of two commutes with rounding in the normal range,
// which every E in [0, 63] and ex in [0, 2] stays in), i.e. exactly the
// correctly rounded reciprocal of the step, from one of four constants.
__device__ __forceinline__ uint32_t hif4_group(const float (&x)[8], int sb, int g, uint32_t &meta_bits,
                                               float (&deq)[8])
{
    const int E = sb >> 2, M = sb & 3;
    const float S = ue6m2_value(E, M);
    const float recip_m = M == 0 ? 1.0f : M == 1 ? 0.8f : M == 2 ? 0.6666666865348816f : 0.5714285969734192f;
    int t[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float a = fmax3(fmaxf(fabsf(x[4 * h]), fabsf(x[4 * h + 1])), fabsf(x[4 * h + 2]), fabsf(x[4 * h + 3]));
        t[h] = a <= 1.75f * S ? 0 : (a <= 3.5f * S ? 1 : 2);
    }
    const int e18 = (t[0] == 2 || t[1] == 2) ? 1 : 0;
    const int e116_0 = max(t[0] - e18, 0), e116_1 = max(t[1] - e18, 0);
    meta_bits = ((uint32_t)e18 << (8 + g)) | ((uint32_t)e116_0 << (16 + 2 * g)) | ((uint32_t)e116_1 << (17 + 2 * g));
    float kf[8];   // the magnitudes k as floats (exact small integers)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int ex = e18 + (h ? e116_1 : e116_0);
        const float step = __uint_as_float(((uint32_t)(E + ex + 77) << 23) | ((uint32_t)M << 21));
        const float inv = __uint_as_float((uint32_t)(177 - E - ex) << 23) * recip_m;   // RN(1 / step)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = x[4 * h + i];
            const float a = fabsf(v);
            // nearest k, ties to even, from the correctly rounded quotient
            // a / step: a * inv is within one ulp of it (inv is the correctly
            // rounded reciprocal), the remainder a - q step is exact (fma),
            // and one correction q + r inv rounds to the correctly rounded
            // quotient (Markstein's division refinement, P. Markstein, IA-64
            // and Elementary Functions, 2000).  A true tie (a half-integer
            // quotient) is then exact, and adding 2^23 rounds it to the even
            // integer; any other quotient lies at least 2^-9 / 7 from every
            // half-integer (a has 8 significant bits, step = D 2^s with D in
            // {4,5,6,7}/4), far beyond the rounding error.  fminf saturates
            // (NaN -> 7) before the rounding.
            float q = a * inv;
            q = fmaf(fmaf(-q, step, a), inv, q);
            const float k = (fminf(q, 7.0f) + 8388608.0f) - 8388608.0f;
            kf[4 * h + i] = k;
            deq[4 * h + i] = copysignf(k * step, v);
        }
    }
    // the eight 3-bit magnitudes into nibbles: two sums of k 16^i (exact
    // below 2^16), their integer bits by adding 2^23, the low halves joined;
    // then the sign bits (bit 3 of each nibble) from the inputs' sign bits
    const float lo = fmaf(kf[3], 4096.0f, fmaf(kf[2], 256.0f, fmaf(kf[1], 16.0f, kf[0])));
    const float hi = fmaf(kf[7], 4096.0f, fmaf(kf[6], 256.0f, fmaf(kf[5], 16.0f, kf[4])));
    uint32_t codes = __byte_perm(__float_as_uint(lo + 8388608.0f), __float_as_uint(hi + 8388608.0f), 0x5410);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        codes |= (__float_as_uint(x[i]) >> (28 - 4 * i)) & (8u << (4 * i));
    return codes;
}

} // namespace rfq
