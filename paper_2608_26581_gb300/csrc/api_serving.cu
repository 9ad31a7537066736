// api_serving.cu -- the C ABI of the serving entry points declared in
// include/rfq.h (slot maps, rotary positions, the 4-bit cache and the
// attention over it, 4-bit matrix-vector products): argument validation and
// dispatch.  No entry point allocates device memory.
#include <cuda_runtime.h>

#include <cstdint>

#include "internal.h"

using namespace rfq;

namespace {

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

rfq_status from_cuda(cudaError_t e) { return e == cudaSuccess ? RFQ_OK : RFQ_ERR_CUDA; }

// Format and sizes of a cache (not its pointers).
rfq_status check_kv_shape(int32_t fmt, int32_t heads, int32_t head_dim, int32_t page_size, int64_t pages)
{
    if (fmt != RFQ_FMT_MXFP4 && fmt != RFQ_FMT_HIF4)
        return RFQ_ERR_INVALID_ARG;
    if (heads < 1 || page_size < 16 || page_size > 4096 || page_size % 16 != 0 || pages < 0 || pages > INT32_MAX)
        return RFQ_ERR_SHAPE;
    if (head_dim != 64 && head_dim != 128)
        return RFQ_ERR_UNSUPPORTED;
    return RFQ_OK;
}

rfq_status check_kv_cache(const rfq_kv_cache *c)
{
    if (!c)
        return RFQ_ERR_INVALID_ARG;
    if (rfq_status s = check_kv_shape(c->fmt, c->heads, c->head_dim, c->page_size, c->pages))
        return s;
    if (c->pages > 0 && (!c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(c->k_codes, 16) || !aligned(c->k_scales, 16) || !aligned(c->v_codes, 16) || !aligned(c->v_scales, 16))
        return RFQ_ERR_ALIGNMENT;
    return RFQ_OK;
}

} // namespace

extern "C" {

rfq_status rfq_slot_map(const int32_t *cached, const int32_t *added, int32_t requests, int32_t page_size,
                        int32_t *block_table, int32_t table_width, int32_t *free_pages, int32_t free_capacity,
                        const int32_t *free_in, int32_t *free_out, int32_t *lengths, int32_t *token_start,
                        int64_t *slots, int32_t *positions, int64_t tokens, void *workspace, void *stream)
{
    if (requests < 0 || requests > kSlotMapRequests || page_size < 1 || table_width < 1 || free_capacity < 0 ||
        tokens < 0 || (int64_t)requests * table_width > INT32_MAX)
        return RFQ_ERR_SHAPE;
    if (!free_in || !free_out || !token_start || !workspace || (free_capacity > 0 && !free_pages) ||
        (requests > 0 && (!cached || !added || !block_table || !lengths)) || (tokens > 0 && (!slots || !positions)))
        return RFQ_ERR_INVALID_ARG;
    for (const void *p : {(const void *)cached, (const void *)added, (const void *)block_table,
                          (const void *)free_pages, (const void *)free_in, (const void *)free_out,
                          (const void *)lengths, (const void *)token_start, (const void *)positions})
        if (!aligned(p, 4))
            return RFQ_ERR_ALIGNMENT;
    if (!aligned(slots, 8) || !aligned(workspace, 16))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    return from_cuda(launch_slot_map({cached, added, requests, page_size, block_table, table_width, free_pages,
                                      free_capacity, free_in, free_out, lengths, token_start, slots, positions,
                                      tokens, static_cast<int32_t *>(workspace)},
                                     static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_rope(const void *x, int64_t x_token_stride, int64_t x_head_stride, void *out, int64_t out_token_stride,
                    int64_t out_head_stride, int32_t dtype, int64_t tokens, int32_t heads, int32_t head_dim,
                    const int32_t *positions, int32_t axes, const float *inv_freq, const int32_t *axis_of,
                    int32_t pairs, int32_t pairing, int32_t inverse, void *stream)
{
    if (dtype != RFQ_OUT_F32 && dtype != RFQ_OUT_BF16)
        return RFQ_ERR_INVALID_ARG;
    if (pairing != RFQ_ROPE_HALF && pairing != RFQ_ROPE_INTERLEAVED)
        return RFQ_ERR_INVALID_ARG;
    if (tokens < 0 || tokens > INT32_MAX || heads < 1 || head_dim < 1 || head_dim > 1024 || axes < 1 || pairs < 1 ||
        pairs > head_dim / 2 || x_token_stride < 0 || x_head_stride < 0 || out_token_stride < 0 ||
        out_head_stride < 0)
        return RFQ_ERR_SHAPE;
    if (!inv_freq || !axis_of || (tokens > 0 && (!x || !out || !positions)))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned(positions, 4) || !aligned(inv_freq, 4) ||
        !aligned(axis_of, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    if (tokens == 0)
        return RFQ_OK;
    return from_cuda(launch_rope({x, x_token_stride, x_head_stride, out, out_token_stride, out_head_stride,
                                  dtype == RFQ_OUT_BF16, tokens, heads, head_dim, positions, axes, inv_freq, axis_of,
                                  pairs, pairing == RFQ_ROPE_INTERLEAVED, inverse != 0},
                                 static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_kv_cache_bytes(int32_t fmt, int32_t heads, int32_t head_dim, int32_t page_size, int64_t pages,
                              size_t *code_bytes, size_t *scale_bytes)
{
    if (!code_bytes || !scale_bytes)
        return RFQ_ERR_INVALID_ARG;
    if (rfq_status s = check_kv_shape(fmt, heads, head_dim, page_size, pages))
        return s;
    const size_t rows = (size_t)pages * (size_t)heads * (size_t)page_size;
    *code_bytes = rows * (size_t)(head_dim / 2);
    *scale_bytes = rows * (size_t)(fmt == RFQ_FMT_HIF4 ? head_dim / 16 : head_dim / 32);
    return RFQ_OK;
}

rfq_status rfq_kv_append(const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v,
                         int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, const int64_t *slots,
                         const rfq_kv_cache *cache, void *stream)
{
    rfq_status s = check_kv_cache(cache);
    if (s != RFQ_OK)
        return s;
    if (tokens < 0 || tokens > INT32_MAX || k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 ||
        v_head_stride < 0)
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!k || !v || !slots))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8) ||
        (k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 8 != 0)
        return RFQ_ERR_ALIGNMENT;
    if ((s = check_device()) != RFQ_OK)
        return s;
    if (tokens == 0 || cache->pages == 0)
        return RFQ_OK;
    return from_cuda(launch_kv_append({k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, tokens,
                                       slots, *cache},
                                      static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_kv_read(const rfq_kv_cache *cache, const int64_t *slots, int64_t tokens, void *k, void *v,
                       int32_t out_dtype, void *stream)
{
    rfq_status s = check_kv_cache(cache);
    if (s != RFQ_OK)
        return s;
    if (out_dtype != RFQ_OUT_F32 && out_dtype != RFQ_OUT_BF16)
        return RFQ_ERR_INVALID_ARG;
    if (tokens < 0 || tokens > INT32_MAX)
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!k || !v || !slots))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8))
        return RFQ_ERR_ALIGNMENT;
    if ((s = check_device()) != RFQ_OK)
        return s;
    if (tokens == 0)
        return RFQ_OK;
    return from_cuda(launch_kv_read(*cache, slots, tokens, k, v, out_dtype == RFQ_OUT_BF16,
                                    static_cast<cudaStream_t>(stream)));
}

size_t rfq_kv_attention_workspace_bytes(int32_t heads, int32_t head_dim)
{
    if (heads < 1 || (head_dim != 64 && head_dim != 128))
        return 0;
    return kv_attention_workspace_bytes(heads, head_dim);
}

rfq_status rfq_kv_attention(const void *q, int64_t q_token_stride, int64_t q_head_stride, int64_t tokens,
                            int32_t heads, const int32_t *q_start, const int32_t *lengths, int32_t requests,
                            const rfq_kv_cache *cache, const int32_t *block_table, int32_t table_width, float scale,
                            int32_t window, void *out, float *lse, void *workspace, void *stream)
{
    rfq_status s = check_kv_cache(cache);
    if (s != RFQ_OK)
        return s;
    if (tokens < 0 || tokens > INT32_MAX || requests < 0 || heads < 1 || heads % cache->heads != 0 ||
        table_width < 1 || window < 0 || q_token_stride < 0 || q_head_stride < 0 ||
        (!q_start && tokens != requests) || (int64_t)table_width * cache->page_size > INT32_MAX - 4096)
        return RFQ_ERR_SHAPE;
    // (the kernels count rows and units of work in 32 bits)
    if ((double)tokens * heads >= 2147483648.0 ||
        kv_attention_most_units(tokens, heads / cache->heads, q_start != nullptr, requests, cache->heads,
                                (int64_t)table_width * cache->page_size) >= 4294967296.0)
        return RFQ_ERR_SHAPE;
    if (!workspace || !(scale == scale) ||
        (tokens > 0 && (!out || (requests > 0 && (!q || !lengths || !block_table)))))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(q_start, 4) ||
        !aligned(lengths, 4) || !aligned(block_table, 4) || !aligned(lse, 4) ||
        (q_token_stride | q_head_stride) % 8 != 0)
        return RFQ_ERR_ALIGNMENT;
    if ((s = check_device()) != RFQ_OK)
        return s;
    if (tokens == 0)
        return RFQ_OK;
    return from_cuda(launch_kv_attention({q, q_token_stride, q_head_stride, tokens, heads, q_start, lengths, requests,
                                          *cache, block_table, table_width, scale, window, out, lse, workspace},
                                         static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_matvec(const void *x, int64_t x_row_stride, int64_t rows, const rfq_qtensor *wq, void *y,
                      int32_t out_dtype, void *stream)
{
    if (!wq || (out_dtype != RFQ_OUT_F32 && out_dtype != RFQ_OUT_BF16))
        return RFQ_ERR_INVALID_ARG;
    rfq_status s = check_qtensor(wq, wq->rows, wq->k);
    if (s != RFQ_OK)
        return s;
    if (wq->fmt != RFQ_FMT_MXFP4 && wq->fmt != RFQ_FMT_HIF4)
        return RFQ_ERR_UNSUPPORTED;
    if (rows < 0 || rows > kMatvecRows || x_row_stride < 0 || wq->rows > kMatvecWeightRows || wq->k > INT32_MAX)
        return RFQ_ERR_SHAPE;
    if (rows > 0 && wq->rows > 0 && (!x || !y))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(y, 16) || x_row_stride % 8 != 0)
        return RFQ_ERR_ALIGNMENT;
    if ((s = check_device()) != RFQ_OK)
        return s;
    if (rows == 0 || wq->rows == 0)
        return RFQ_OK;
    return from_cuda(launch_matvec({x, x_row_stride, (int32_t)rows, *wq, y, out_dtype == RFQ_OUT_BF16},
                                   static_cast<cudaStream_t>(stream)));
}

} // extern "C"
