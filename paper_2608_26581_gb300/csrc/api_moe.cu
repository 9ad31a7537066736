// api_moe.cu -- the C ABI of the entry points around a mixture-of-experts
// block declared in include/rfq.h (norms, the router, rows brought to the
// experts' groups and back): argument validation and dispatch.  No entry
// point allocates device memory.
#include <cuda_runtime.h>

#include <cstdint>

#include "internal.h"

using namespace rfq;

namespace {

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

rfq_status from_cuda(cudaError_t e) { return e == cudaSuccess ? RFQ_OK : RFQ_ERR_CUDA; }

bool is_dtype(int32_t d) { return d == RFQ_OUT_F32 || d == RFQ_OUT_BF16; }

// A stride along an axis of n elements: of one element it means nothing, and takes no part in any choice.
int64_t used(int64_t stride, int64_t n) { return n > 1 ? stride : 0; }

// n rows of a result, of dim elements, do not lie on top of each other.
bool apart(int64_t stride, int64_t n, int64_t dim) { return n <= 1 || stride >= dim; }

// Sizes of tokens' choices of experts.
bool choices_fit(int64_t tokens, int32_t top_k)
{
    return tokens >= 0 && top_k >= 1 && top_k <= kRouteTopK && tokens <= INT32_MAX / top_k;
}

// Sizes of pairs sorted into groups: every row that a group can have is counted in 31 bits.
bool groups_fit(int64_t tokens, int32_t top_k, int32_t experts, int32_t align)
{
    return choices_fit(tokens, top_k) && experts >= 1 && experts <= kMoeExperts && align >= 1 && align <= kMoeAlign &&
           tokens * top_k + (int64_t)experts * align <= INT32_MAX;
}

// Sizes shared by the calls that move rows.
bool rows_fit(int64_t tokens, int32_t top_k, int64_t rows, int64_t dim, int64_t stride)
{
    return choices_fit(tokens, top_k) && rows >= 0 && rows <= INT32_MAX && dim >= 1 && dim <= kMoeDim && stride >= 0;
}

} // namespace

extern "C" {

rfq_status rfq_norm(const void *x, int64_t x_token_stride, int64_t x_head_stride, void *y, int64_t y_token_stride,
                    int64_t y_head_stride, int32_t dtype, int64_t tokens, int32_t heads, int32_t dim, int32_t kind,
                    float eps, const void *weight, const void *bias, int32_t w_dtype, float *mean, float *rstd,
                    void *stream)
{
    x_token_stride = used(x_token_stride, tokens);
    x_head_stride = used(x_head_stride, heads);
    y_token_stride = used(y_token_stride, tokens);
    y_head_stride = used(y_head_stride, heads);
    if (!is_dtype(dtype) || !is_dtype(w_dtype) || (kind != RFQ_NORM_LAYER && kind != RFQ_NORM_RMS) || !(eps >= 0.f))
        return RFQ_ERR_INVALID_ARG;
    if (tokens < 0 || heads < 1 || tokens > INT32_MAX / heads || dim < 1 || dim > kNormDim || x_token_stride < 0 ||
        x_head_stride < 0 || y_token_stride < 0 || y_head_stride < 0 || !apart(y_token_stride, tokens, dim) ||
        !apart(y_head_stride, heads, dim))
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!x || !y))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(weight, 16) || !aligned(bias, 16) || !aligned(mean, 4) ||
        !aligned(rstd, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    if (tokens == 0)
        return RFQ_OK;
    return from_cuda(launch_norm({x, x_token_stride, x_head_stride, y, y_token_stride, y_head_stride,
                                  dtype == RFQ_OUT_BF16, tokens * heads, heads, dim, kind == RFQ_NORM_RMS, eps, weight,
                                  bias, w_dtype == RFQ_OUT_BF16, mean, rstd},
                                 static_cast<cudaStream_t>(stream)));
}

size_t rfq_norm_grad_workspace_bytes(int32_t dim)
{
    return dim < 1 || dim > kNormDim ? 0 : norm_grad_workspace_bytes(dim);
}

rfq_status rfq_norm_grad(const void *dy, int64_t dy_token_stride, int64_t dy_head_stride, const void *x,
                         int64_t x_token_stride, int64_t x_head_stride, void *dx, int64_t dx_token_stride,
                         int64_t dx_head_stride, int32_t dtype, int64_t tokens, int32_t heads, int32_t dim,
                         int32_t kind, const float *mean, const float *rstd, const void *weight, int32_t w_dtype,
                         float *dweight, float *dbias, void *workspace, void *stream)
{
    dy_token_stride = used(dy_token_stride, tokens);
    dy_head_stride = used(dy_head_stride, heads);
    x_token_stride = used(x_token_stride, tokens);
    x_head_stride = used(x_head_stride, heads);
    dx_token_stride = used(dx_token_stride, tokens);
    dx_head_stride = used(dx_head_stride, heads);
    if (!is_dtype(dtype) || !is_dtype(w_dtype) || (kind != RFQ_NORM_LAYER && kind != RFQ_NORM_RMS))
        return RFQ_ERR_INVALID_ARG;
    if (tokens < 0 || heads < 1 || tokens > INT32_MAX / heads || dim < 1 || dim > kNormDim || dy_token_stride < 0 ||
        dy_head_stride < 0 || x_token_stride < 0 || x_head_stride < 0 || dx_token_stride < 0 || dx_head_stride < 0 ||
        !apart(dx_token_stride, tokens, dim) || !apart(dx_head_stride, heads, dim))
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!dy || !x || !dx || !rstd || (kind == RFQ_NORM_LAYER && !mean)))
        return RFQ_ERR_INVALID_ARG;
    if ((dweight || dbias) && !workspace)
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(dx, 16) || !aligned(weight, 16) || !aligned(workspace, 16) ||
        !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    // (no rows: the weight's gradient is zero, and is written)
    if (tokens == 0 && !dweight && !dbias)
        return RFQ_OK;
    return from_cuda(launch_norm_grad({dy, dy_token_stride, dy_head_stride, x, x_token_stride, x_head_stride, dx,
                                       dx_token_stride, dx_head_stride, dtype == RFQ_OUT_BF16, tokens * heads, heads,
                                       dim, kind == RFQ_NORM_RMS, mean, rstd, weight, w_dtype == RFQ_OUT_BF16, dweight,
                                       dbias, workspace, nullptr},
                                      static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_route(const void *logits, int64_t row_stride, int32_t dtype, int64_t tokens, int32_t experts,
                     int32_t top_k, int32_t normalize, int32_t *ids, float *weights, void *stream)
{
    row_stride = used(row_stride, tokens);
    if (!is_dtype(dtype))
        return RFQ_ERR_INVALID_ARG;
    if (!choices_fit(tokens, top_k) || experts < 1 || experts > kRouteExperts || top_k > experts || row_stride < 0)
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!logits || !ids || !weights))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(logits, 16) || !aligned(ids, 4) || !aligned(weights, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    if (tokens == 0)
        return RFQ_OK;
    return from_cuda(launch_route({logits, row_stride, dtype == RFQ_OUT_BF16, tokens, experts, top_k, normalize != 0,
                                   ids, weights},
                                  static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_route_grad(const void *logits, int64_t row_stride, int32_t dtype, int64_t tokens, int32_t experts,
                          int32_t top_k, int32_t normalize, const int32_t *ids, const float *dweights, void *dlogits,
                          int64_t dlogits_row_stride, void *stream)
{
    row_stride = used(row_stride, tokens);
    dlogits_row_stride = used(dlogits_row_stride, tokens);
    if (!is_dtype(dtype))
        return RFQ_ERR_INVALID_ARG;
    if (!choices_fit(tokens, top_k) || experts < 1 || experts > kRouteExperts || top_k > experts || row_stride < 0 ||
        dlogits_row_stride < 0 || !apart(dlogits_row_stride, tokens, experts))
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!logits || !ids || !dweights || !dlogits))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(logits, 16) || !aligned(dlogits, 16) || !aligned(ids, 4) || !aligned(dweights, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    if (tokens == 0)
        return RFQ_OK;
    return from_cuda(launch_route_grad({logits, row_stride, dtype == RFQ_OUT_BF16, tokens, experts, top_k,
                                        normalize != 0, ids, dweights, dlogits, dlogits_row_stride},
                                       static_cast<cudaStream_t>(stream)));
}

int64_t rfq_moe_rows(int64_t tokens, int32_t top_k, int32_t experts, int32_t align)
{
    if (!groups_fit(tokens, top_k, experts, align))
        return -1;
    const int64_t pairs = tokens * top_k, groups = pairs < experts ? pairs : experts;
    return (pairs + groups * (align - 1)) / align * align;
}

rfq_status rfq_moe_sort(const int32_t *ids, int64_t tokens, int32_t top_k, int32_t experts, int32_t align,
                        int32_t *group_off, int32_t *row_of, int32_t *pair_of, int64_t rows, void *workspace,
                        void *stream)
{
    if (!groups_fit(tokens, top_k, experts, align) || rows < 0 || rows > INT32_MAX)
        return RFQ_ERR_SHAPE;
    if (!group_off || !workspace || (tokens > 0 && (!ids || !row_of)) || (rows > 0 && !pair_of))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(ids, 4) || !aligned(group_off, 4) || !aligned(row_of, 4) || !aligned(pair_of, 4) ||
        !aligned(workspace, 16))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    return from_cuda(launch_moe_sort({ids, tokens * top_k, experts, align, group_off, row_of, pair_of, rows,
                                      static_cast<int32_t *>(workspace)},
                                     static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_moe_gather(const void *x, int64_t x_row_stride, int32_t dtype, int64_t tokens, int32_t dim,
                          const int32_t *row_of, int32_t top_k, const int32_t *pair_of, void *out, int64_t rows,
                          void *stream)
{
    x_row_stride = used(x_row_stride, tokens);
    if (!is_dtype(dtype))
        return RFQ_ERR_INVALID_ARG;
    if (!rows_fit(tokens, top_k, rows, dim, x_row_stride))
        return RFQ_ERR_SHAPE;
    if ((tokens > 0 && (!x || !row_of)) || (rows > 0 && !out))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned(row_of, 4) || !aligned(pair_of, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    if (rows == 0)
        return RFQ_OK;
    return from_cuda(launch_moe_gather({x, x_row_stride, dtype == RFQ_OUT_BF16, tokens, dim, row_of, top_k, pair_of,
                                        out, rows},
                                       static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_moe_combine(const void *y, int32_t dtype, int64_t rows, int32_t dim, const int32_t *row_of,
                           const float *weights, int64_t tokens, int32_t top_k, void *out, int64_t out_row_stride,
                           void *stream)
{
    out_row_stride = used(out_row_stride, tokens);
    if (!is_dtype(dtype))
        return RFQ_ERR_INVALID_ARG;
    if (!rows_fit(tokens, top_k, rows, dim, out_row_stride) || !apart(out_row_stride, tokens, dim))
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!row_of || !out || (rows > 0 && !y)))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(y, 16) || !aligned(out, 16) || !aligned(row_of, 4) || !aligned(weights, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    if (tokens == 0)
        return RFQ_OK;
    return from_cuda(launch_moe_combine({y, dtype == RFQ_OUT_BF16, rows, dim, row_of, weights, tokens, top_k, out,
                                         out_row_stride},
                                        static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_moe_combine_grad(const void *dout, int64_t dout_row_stride, const void *y, int32_t dtype, int64_t rows,
                                int32_t dim, const int32_t *row_of, const int32_t *pair_of, const float *weights,
                                int64_t tokens, int32_t top_k, void *dy, float *dweights, void *stream)
{
    dout_row_stride = used(dout_row_stride, tokens);
    if (!is_dtype(dtype))
        return RFQ_ERR_INVALID_ARG;
    if (!rows_fit(tokens, top_k, rows, dim, dout_row_stride))
        return RFQ_ERR_SHAPE;
    if ((tokens > 0 && (!dout || !row_of || !weights || !dweights)) || (rows > 0 && (!y || !dy)))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(dout, 16) || !aligned(y, 16) || !aligned(dy, 16) || !aligned(row_of, 4) || !aligned(pair_of, 4) ||
        !aligned(weights, 4) || !aligned(dweights, 4))
        return RFQ_ERR_ALIGNMENT;
    if (rfq_status s = check_device())
        return s;
    return from_cuda(launch_moe_combine_grad({dout, dout_row_stride, y, dtype == RFQ_OUT_BF16, rows, dim, row_of,
                                              pair_of, weights, tokens, top_k, dy, dweights},
                                             static_cast<cudaStream_t>(stream)));
}

rfq_status rfq_moe_quantize(const void *x, int64_t x_row_stride, int64_t tokens, const int32_t *row_of, int32_t top_k,
                            const int32_t *pair_of, rfq_qtensor *xq, rfq_qtensor *xr, void *stream)
{
    x_row_stride = used(x_row_stride, tokens);
    if (!xq)
        return RFQ_ERR_INVALID_ARG;
    rfq_status s = check_qtensor(xq, xq->rows, xq->k);
    if (s != RFQ_OK || (xr && (s = check_qtensor(xr, xq->rows, xq->k)) != RFQ_OK))
        return s;
    if (xq->fmt != RFQ_FMT_MXFP4 || xq->scale_layout != RFQ_SCALE_MMA ||
        (xr && (xr->fmt != RFQ_FMT_MXFP4 || xr->scale_layout != RFQ_SCALE_MMA)))
        return RFQ_ERR_UNSUPPORTED;
    if (!rows_fit(tokens, top_k, xq->rows, xq->k, x_row_stride))
        return RFQ_ERR_SHAPE;
    if (tokens > 0 && (!x || !row_of))
        return RFQ_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(row_of, 4) || !aligned(pair_of, 4) || x_row_stride % 8 != 0)
        return RFQ_ERR_ALIGNMENT;
    if ((s = check_device()) != RFQ_OK)
        return s;
    if (xq->rows == 0)
        return RFQ_OK;
    return from_cuda(launch_moe_quantize({x, x_row_stride, tokens, (int32_t)xq->k, row_of, top_k, pair_of, xq->codes,
                                          xq->scales, xr ? xr->codes : nullptr, xr ? xr->scales : nullptr, xq->rows, 0},
                                         static_cast<cudaStream_t>(stream)));
}

} // extern "C"
