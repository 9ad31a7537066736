// kv_cache.cu -- keys and values into the paged 4-bit cache (rfq_kv_append)
// and back (rfq_kv_read).  Quantization is that of the activation quantizers
// bit for bit (Sec. 3.2 Eq. 3-4, Sec. 3.3), blocks along the head dimension.
//
// Bound: HBM (2 bytes in, 0.53 or 0.56 out per element; the reverse for the
// read).  One lane takes 32 elements: an MXFP4 block, or half a HiF4 block
// whose amax and metadata two lanes join by a shuffle.  A lane's 16 bytes of
// codes go out as the four words (K) or D/8-dimension pieces (V) of the
// layout; the neighbouring lanes fill the rest of their sectors.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "hif4_math.cuh"
#include "kv_layout.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 256;

// One lane's 32 elements: sub-block b (of D/32) of (token, head) of K or V.
struct Item {
    int64_t t;
    int head, b;
    bool value;
};

template <int D>
__device__ __forceinline__ Item item_of(int64_t i, int heads)
{
    constexpr int NB = D / 32;
    const int b = (int)(i % NB);
    const int64_t r = i / NB;
    const int64_t th = r >> 1;
    return {th / heads, (int)(th % heads), b, (r & 1) != 0};
}

__device__ __forceinline__ bool slot_ok(int64_t slot, const rfq_kv_cache &c)
{
    return slot >= 0 && slot < c.pages * c.page_size;
}

template <int FMT, int D>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const KvAppendArgs a)
{
    constexpr int NB = D / 32;
    const rfq_kv_cache &c = a.cache;
    const int64_t n = a.tokens * 2 * c.heads * NB;
    // every lane of a warp stays to the end (the HiF4 lanes shuffle)
    for (int64_t i0 = (int64_t)blockIdx.x * kThreads; i0 < n; i0 += (int64_t)gridDim.x * kThreads) {
        const int64_t i = i0 + threadIdx.x;
        const Item it = item_of<D>(i < n ? i : n - 1, c.heads);
        const int64_t slot = a.slots[it.t];
        const bool ok = i < n && slot_ok(slot, c);
        const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(it.value ? a.v : a.k) +
                                   it.t * (it.value ? a.v_token : a.k_token) +
                                   (int64_t)it.head * (it.value ? a.v_head : a.k_head) + it.b * 32;
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(src) + j);
            w[4 * j] = u.x, w[4 * j + 1] = u.y, w[4 * j + 2] = u.z, w[4 * j + 3] = u.w;
        }
        float x[32];
        bf16x32_to_f32(w, x);
        uint32_t code[4], scale;
        if (FMT == RFQ_FMT_MXFP4) {
            const Mx32 m = mxfp4_quant32<false>(x);
            code[0] = m.code.x, code[1] = m.code.y, code[2] = m.code.z, code[3] = m.code.w;
            scale = (uint32_t)m.sb;
        } else {
            float am = absmax32(x);
            am = fmaxf(am, __shfl_xor_sync(0xFFFFFFFFu, am, 1));
            const int sb = am > 0.f ? hif4_scale_byte(am) : 0;
            uint32_t bits = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float g[8], deq[8];
                uint32_t m;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    g[e] = x[8 * j + e];
                code[j] = hif4_group(g, sb, 4 * (it.b & 1) + j, m, deq);
                bits |= m;
            }
            bits |= __shfl_xor_sync(0xFFFFFFFFu, bits, 1);
            scale = am > 0.f ? (bits | (uint32_t)sb) : 0u;
        }
        if (!ok)
            continue;
        const int64_t page = slot / c.page_size;
        const int tok = (int)(slot - page * c.page_size);
        const int64_t ph = page * c.heads + it.head;
        uint8_t *const codes =
            static_cast<uint8_t *>(it.value ? c.v_codes : c.k_codes) + ph * kv_code_bytes(c.page_size, D);
        if (it.value) {
            if (D == 128) {   // two pieces of 16 dimensions
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<uint2 *>(codes + kv_v_piece(tok, 2 * it.b + j, D)) =
                        make_uint2(code[2 * j], code[2 * j + 1]);
            } else {          // four of 8
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<uint32_t *>(codes + kv_v_piece(tok, 4 * it.b + j, D)) = code[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<uint32_t *>(codes + kv_k_word(tok, it.b, j, D)) = code[j];
        }
        uint8_t *const sc = static_cast<uint8_t *>(it.value ? c.v_scales : c.k_scales) +
                            (ph * c.page_size + tok) * kv_token_scale_bytes(FMT, D);
        if (FMT == RFQ_FMT_MXFP4)
            sc[it.b] = (uint8_t)scale;
        else if ((it.b & 1) == 0)
            *reinterpret_cast<uint32_t *>(sc + it.b * 2) = scale;
    }
}

template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const rfq_kv_cache c, const int64_t *slots, int64_t tokens,
                                                           void *k, void *v)
{
    constexpr int NB = D / 32;
    const int64_t n = tokens * 2 * c.heads * NB;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
        const Item it = item_of<D>(i, c.heads);
        const int64_t slot = slots[it.t];
        float x[32];
        if (slot_ok(slot, c)) {
            const int64_t page = slot / c.page_size;
            const int tok = (int)(slot - page * c.page_size);
            const int64_t ph = page * c.heads + it.head;
            const uint8_t *const codes =
                static_cast<const uint8_t *>(it.value ? c.v_codes : c.k_codes) + ph * kv_code_bytes(c.page_size, D);
            uint32_t code[4];
            if (!it.value) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    code[j] = *reinterpret_cast<const uint32_t *>(codes + kv_k_word(tok, it.b, j, D));
            } else if (D == 128) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint2 u = *reinterpret_cast<const uint2 *>(codes + kv_v_piece(tok, 2 * it.b + j, D));
                    code[2 * j] = u.x, code[2 * j + 1] = u.y;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    code[j] = *reinterpret_cast<const uint32_t *>(codes + kv_v_piece(tok, 4 * it.b + j, D));
            }
            const uint8_t *const sc = static_cast<const uint8_t *>(it.value ? c.v_scales : c.k_scales) +
                                      (ph * c.page_size + tok) * kv_token_scale_bytes(FMT, D);
            if (FMT == RFQ_FMT_MXFP4) {
                const float s = e8m0_f32(sc[it.b]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float q[8];
                    e2m1x8_decode(code[j], q);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[8 * j + e] = q[e] * s;
                }
            } else {
                const uint32_t meta = *reinterpret_cast<const uint32_t *>(sc + (it.b >> 1) * 4);
                const float quarter = 0.25f * hif4_macro_f32(meta);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int gi = 4 * (it.b & 1) + j;
                    const uint32_t e8 = (meta >> (8 + gi)) & 1u, e16 = meta >> (16 + 2 * gi);
                    const float s0 = quarter * (float)(1 << (e8 + (e16 & 1u)));
                    const float s1 = quarter * (float)(1 << (e8 + ((e16 >> 1) & 1u)));
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t nib = code[j] >> (4 * e);
                        const float m = (float)(nib & 7u) * (e < 4 ? s0 : s1);
                        x[8 * j + e] = (nib & 8u) ? -m : m;
                    }
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 32; ++e)
                x[e] = 0.f;
        }
        const int64_t o = ((it.t * c.heads + it.head) * NB + it.b) * 32;
        if (BF16) {
            uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(it.value ? v : k) + o);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(x[8 * j + 2 * e], x[8 * j + 2 * e + 1]);
                    p[e] = *reinterpret_cast<const uint32_t *>(&h);
                }
                __stcs(dst + j, make_uint4(p[0], p[1], p[2], p[3]));
            }
        } else {
            float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(it.value ? v : k) + o);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                __stcs(dst + j, make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]));
        }
    }
}

unsigned blocks_for(int64_t lanes, const void *kern)
{
    const int64_t want = (lanes + kThreads - 1) / kThreads;
    const int64_t most = (int64_t)num_sms() * resident_blocks_per_sm(kern, kThreads, 0);
    return (unsigned)(want < most ? want : most);
}

} // namespace

cudaError_t launch_kv_append(const KvAppendArgs &a, cudaStream_t st)
{
    const int D = a.cache.head_dim;
    const bool hif4 = a.cache.fmt == RFQ_FMT_HIF4;
    auto *const kern = hif4 ? (D == 128 ? kv_append_kernel<RFQ_FMT_HIF4, 128> : kv_append_kernel<RFQ_FMT_HIF4, 64>)
                            : (D == 128 ? kv_append_kernel<RFQ_FMT_MXFP4, 128> : kv_append_kernel<RFQ_FMT_MXFP4, 64>);
    const int64_t lanes = a.tokens * 2 * a.cache.heads * (D / 32);
    kern<<<blocks_for(lanes, reinterpret_cast<const void *>(kern)), kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_kv_read(const rfq_kv_cache &c, const int64_t *slots, int64_t tokens, void *k, void *v, bool bf16,
                           cudaStream_t st)
{
    const bool wide = c.head_dim == 128;
    using Kern = void (*)(const rfq_kv_cache, const int64_t *, int64_t, void *, void *);
    Kern kern;
    if (c.fmt == RFQ_FMT_HIF4)
        kern = wide ? (bf16 ? kv_read_kernel<RFQ_FMT_HIF4, 128, true> : kv_read_kernel<RFQ_FMT_HIF4, 128, false>)
                    : (bf16 ? kv_read_kernel<RFQ_FMT_HIF4, 64, true> : kv_read_kernel<RFQ_FMT_HIF4, 64, false>);
    else
        kern = wide ? (bf16 ? kv_read_kernel<RFQ_FMT_MXFP4, 128, true> : kv_read_kernel<RFQ_FMT_MXFP4, 128, false>)
                    : (bf16 ? kv_read_kernel<RFQ_FMT_MXFP4, 64, true> : kv_read_kernel<RFQ_FMT_MXFP4, 64, false>);
    const int64_t lanes = tokens * 2 * c.heads * (c.head_dim / 32);
    kern<<<blocks_for(lanes, reinterpret_cast<const void *>(kern)), kThreads, 0, st>>>(c, slots, tokens, k, v);
    return cudaGetLastError();
}

} // namespace rfq
