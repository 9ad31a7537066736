// kv_cache.cu -- keys and values into the paged 4-bit cache (rfq_kv_append)
// and back (rfq_kv_read).  Quantization is that of the activation quantizers
// bit for bit (Sec. 3.2 Eq. 3-4, Sec. 3.3), blocks along the head dimension.
//
// Bound: HBM (2 bytes in, 0.53 or 0.56 out per element; the reverse for the
// read); HiF4's encoder is bound by its arithmetic.  A warp takes 1024
// elements of one head: D / 32 consecutive lanes share a token, each 32 of its
// elements (an MXFP4 block, or half a HiF4 block whose amax and metadata two
// lanes join), and 8 or 16 consecutive tokens fill whole sectors of the cache
// where their slots follow each other.  A K row's word transposition is a
// transposition over the token's lanes, done with shuffles, so that codes go
// out 16 bytes at a time.  Blocks run over the heads first: a token's row of
// all heads is read by blocks that run at the same time.
// 16384 tokens, 8 heads of 128, K and V, appended and read back: MXFP4 32 us,
// 78% of the copy rate; HiF4 44 us, 58%, 28 of them the append, which its
// encoder keeps on the ALUs.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "hif4_math.cuh"
#include "kv_layout.cuh"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 256;

constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ bool slot_ok(int64_t slot, const rfq_kv_cache &c)
{
    return slot >= 0 && slot < c.pages * c.page_size;
}

// Page and token of a slot (a 64-bit division only where it has to be one).
__device__ __forceinline__ int64_t page_of(int64_t slot, int page_size, int &tok)
{
    if ((slot >> 32) == 0) {
        const uint32_t page = (uint32_t)slot / (uint32_t)page_size;
        tok = (int)((uint32_t)slot - page * (uint32_t)page_size);
        return page;
    }
    const int64_t page = slot / page_size;
    tok = (int)(slot - page * page_size);
    return page;
}

// w[c] of lane b -> w[b] of lane c, over a token's four lanes.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4], int lane)
{
#pragma unroll
    for (int d = 1; d <= 2; d <<= 1) {
        const bool up = (lane & d) != 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int lo = d == 1 ? 2 * i : i, hi = lo + d;
            const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, up ? w[lo] : w[hi], d);
            if (up)
                w[lo] = got;
            else
                w[hi] = got;
        }
    }
}

// Block (head of K or V, kWarps warps of tokens).  Four blocks an SM: HiF4's
// encoder waits on its own arithmetic (40 us a 16384 x 8 x 128 append with the
// two that its registers would take, 30 with four).
template <int FMT, int D>
__global__ void __launch_bounds__(kThreads, 4) kv_append_kernel(const KvAppendArgs a)
{
    constexpr int NB = D / 32, TOK = 32 / NB;
    const rfq_kv_cache &c = a.cache;
    const int lane = threadIdx.x & 31, b = lane % NB;
    const bool value = blockIdx.x >= (unsigned)c.heads;
    const int head = blockIdx.x - (value ? c.heads : 0);
    const int64_t token = value ? a.v_token : a.k_token;
    const __nv_bfloat16 *const src = static_cast<const __nv_bfloat16 *>(value ? a.v : a.k) +
                                     (int64_t)head * (value ? a.v_head : a.k_head) + b * 32;
    uint8_t *const codes0 = static_cast<uint8_t *>(value ? c.v_codes : c.k_codes);
    uint8_t *const scales0 = static_cast<uint8_t *>(value ? c.v_scales : c.k_scales);
    wait_for_previous();
    let_next_start();
    // every lane of a warp stays to the end (its lanes shuffle)
    for (int64_t t0 = ((int64_t)blockIdx.y * kWarps + (threadIdx.x >> 5)) * TOK; t0 < a.tokens;
         t0 += (int64_t)gridDim.y * kWarps * TOK) {
        const int64_t t = min(t0 + lane / NB, a.tokens - 1);
        const int64_t slot = a.slots[t];
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 u = reinterpret_cast<const uint4 *>(src + t * token)[j];
            w[4 * j] = u.x, w[4 * j + 1] = u.y, w[4 * j + 2] = u.z, w[4 * j + 3] = u.w;
        }
        const bool ok = t0 + lane / NB < a.tokens && slot_ok(slot, c);
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
                code[j] = hif4_group(g, sb, 4 * (b & 1) + j, m, deq);
                bits |= m;
            }
            bits |= __shfl_xor_sync(0xFFFFFFFFu, bits, 1);
            scale = am > 0.f ? (bits | (uint32_t)sb) : 0u;
        }
        if (!value && D == 128) {
            transpose4(code, lane);
        } else if (!value) {                 // lane 0 takes words c = 0, 1 of both sub-blocks, lane 1 c = 2, 3
            const uint32_t p = __shfl_xor_sync(0xFFFFFFFFu, b ? code[0] : code[2], 1);
            const uint32_t q = __shfl_xor_sync(0xFFFFFFFFu, b ? code[1] : code[3], 1);
            const uint32_t own0 = b ? code[2] : code[0], own1 = b ? code[3] : code[1];
            code[0] = b ? p : own0, code[1] = b ? own0 : p;
            code[2] = b ? q : own1, code[3] = b ? own1 : q;
        }
        if (!ok)
            continue;
        int tok;
        const int64_t ph = page_of(slot, c.page_size, tok) * c.heads + head;
        uint8_t *const codes = codes0 + ph * kv_code_bytes(c.page_size, D);
        if (!value) {
            *reinterpret_cast<uint4 *>(codes + (int64_t)tok * (D / 2) + b * 16) =
                make_uint4(code[0], code[1], code[2], code[3]);
        } else if (D == 128) {               // two pieces of 16 dimensions
#pragma unroll
            for (int j = 0; j < 2; ++j)
                *reinterpret_cast<uint2 *>(codes + kv_v_piece(tok, 2 * b + j, D)) =
                    make_uint2(code[2 * j], code[2 * j + 1]);
        } else {                             // four of 8
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<uint32_t *>(codes + kv_v_piece(tok, 4 * b + j, D)) = code[j];
        }
        uint8_t *const sc = scales0 + (ph * c.page_size + tok) * kv_token_scale_bytes(FMT, D);
        if (FMT == RFQ_FMT_MXFP4)
            sc[b] = (uint8_t)scale;
        else if ((b & 1) == 0)
            *reinterpret_cast<uint32_t *>(sc + b * 2) = scale;
    }
}

template <bool BF16>
__device__ __forceinline__ void store8(void *dst, int64_t at, const float (&x)[8])
{
    if (BF16) {
        uint32_t p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
            p[e] = *reinterpret_cast<const uint32_t *>(&h);
        }
        __stcs(reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(dst) + at), make_uint4(p[0], p[1], p[2], p[3]));
    } else {
        float4 *const d = reinterpret_cast<float4 *>(static_cast<float *>(dst) + at);
        __stcs(d, make_float4(x[0], x[1], x[2], x[3]));
        __stcs(d + 1, make_float4(x[4], x[5], x[6], x[7]));
    }
}

// As above: D / 32 lanes share a token.  Of K lane c takes 16 bytes of the
// row as they lie (D = 128: the words c of all sub-blocks), of V the pieces
// lane, lane + D/32, ... (so that a lane's eight values start a sector's half).
template <int FMT, int D, bool BF16>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const rfq_kv_cache c, const int64_t *slots, int64_t tokens,
                                                           void *k, void *v)
{
    constexpr int NB = D / 32, TOK = 32 / NB;
    const int lane = threadIdx.x & 31, l = lane % NB;
    const bool value = blockIdx.x >= (unsigned)c.heads;
    const int head = blockIdx.x - (value ? c.heads : 0);
    void *const dst = value ? v : k;
    const uint8_t *const codes0 = static_cast<const uint8_t *>(value ? c.v_codes : c.k_codes);
    const uint8_t *const scales0 = static_cast<const uint8_t *>(value ? c.v_scales : c.k_scales);
    wait_for_previous();
    let_next_start();
    for (int64_t t = ((int64_t)blockIdx.y * kWarps + (threadIdx.x >> 5)) * TOK + lane / NB; t < tokens;
         t += (int64_t)gridDim.y * kWarps * TOK) {
        const int64_t slot = slots[t], o = (t * c.heads + head) * D;
        float x[8];
        if (!slot_ok(slot, c)) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                store8<BF16>(dst, o + 32 * l + 8 * j, x);
            continue;
        }
        int tok;
        const int64_t ph = page_of(slot, c.page_size, tok) * c.heads + head;
        const uint8_t *const codes = codes0 + ph * kv_code_bytes(c.page_size, D);
        const uint8_t *const sc = scales0 + (ph * c.page_size + tok) * kv_token_scale_bytes(FMT, D);
        uint32_t code[4], s[2] = {0, 0};
        if (!value) {
            const uint4 u = *reinterpret_cast<const uint4 *>(codes + (int64_t)tok * (D / 2) + l * 16);
            code[0] = u.x, code[1] = u.y, code[2] = u.z, code[3] = u.w;
        } else if (D == 128) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint2 u = *reinterpret_cast<const uint2 *>(codes + kv_v_piece(tok, l + 4 * j, D));
                code[2 * j] = u.x, code[2 * j + 1] = u.y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                code[j] = *reinterpret_cast<const uint32_t *>(codes + kv_v_piece(tok, l + 2 * j, D));
        }
        if (FMT == RFQ_FMT_HIF4) {
            s[0] = *reinterpret_cast<const uint32_t *>(sc);
            s[1] = D == 128 ? *reinterpret_cast<const uint32_t *>(sc + 4) : s[0];
        } else {
            s[0] = D == 128 ? *reinterpret_cast<const uint32_t *>(sc) : *reinterpret_cast<const uint16_t *>(sc);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // first of the word's eight dimensions
            const int d = value ? (D == 128 ? (l + 4 * (j >> 1)) * 16 + (j & 1) * 8 : (l + 2 * j) * 8)
                          : D == 128 ? 32 * j + 8 * l
                                     : 32 * (j & 1) + 8 * (2 * l + (j >> 1));
            if (FMT == RFQ_FMT_HIF4)
                hif4_values(code[j], d < 64 ? s[0] : s[1], (d & 63) >> 3, x);
            else
                mxfp4_values(code[j], (s[0] >> (8 * (d >> 5))) & 0xFFu, x);
            store8<BF16>(dst, o + d, x);
        }
    }
}

dim3 grid_for(int64_t tokens, int heads, int D)
{
    const int64_t per = (int64_t)kWarps * 32 / (D / 32);     // tokens of a block
    const int64_t y = (tokens + per - 1) / per;
    return dim3(2 * heads, (unsigned)(y < 65535 ? y : 65535));
}

} // namespace

cudaError_t launch_kv_append(const KvAppendArgs &a, cudaStream_t st)
{
    const int D = a.cache.head_dim;
    const bool hif4 = a.cache.fmt == RFQ_FMT_HIF4;
    auto *const kern = hif4 ? (D == 128 ? kv_append_kernel<RFQ_FMT_HIF4, 128> : kv_append_kernel<RFQ_FMT_HIF4, 64>)
                            : (D == 128 ? kv_append_kernel<RFQ_FMT_MXFP4, 128> : kv_append_kernel<RFQ_FMT_MXFP4, 64>);
    return launch_early(kern, grid_for(a.tokens, a.cache.heads, D), kThreads, 0, st, 1, a);
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
    return launch_early(kern, grid_for(tokens, c.heads, c.head_dim), kThreads, 0, st, 1, c, slots, tokens, k, v);
}

} // namespace rfq
