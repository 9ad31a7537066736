// moe_rows.cu -- rows of tokens brought to their experts' groups and back:
//   gather        out[row_of[t, j]] = x[t], other rows 0          (rfq_moe_gather)
//   combine       out[t] = sum_j w[t, j] y[row_of[t, j]]          (rfq_moe_combine)
//   combine_grad  dy[row_of[t, j]] = w[t, j] dout[t], other rows 0,
//                 dw[t, j] = <dout[t], y[row_of[t, j]]>           (rfq_moe_combine_grad)
//   quantize      gather of Q(x) and Q(x - Q(x)) in MXFP4         (rfq_moe_quantize)
//
// Bound: HBM.  Work goes by tokens: a token's row is read once and written to
// (or summed from) the rows of its top_k pairs, and quantized once for all of
// them.  Rows of no pair are cleared by warps of their own.  Sums are fp32 in
// the order of the choices: the same inputs give the same bits.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace rfq {
namespace {

constexpr int kWarps = 8;
constexpr uint32_t kAll = 0xFFFFFFFFu;

// The row of pair j of a token (lane j holds it), -1 where there is none.
__device__ __forceinline__ int token_row(const int32_t *row_of, int64_t t, int top_k, int64_t rows, int lane)
{
    int r = lane < top_k ? row_of[t * top_k + lane] : -1;
    return r < rows ? r : -1;
}

// Clears the columns [c0, c1) (in vectors) of those of 32 rows from r0 on that hold no pair.
template <typename T, int VEC>
__device__ __forceinline__ void clear_rows(T *out, const int32_t *pair_of, int64_t rows, int dim, int64_t r0, int c0, int c1, int lane)
{
    uint32_t none = __ballot_sync(kAll, r0 + lane < rows && pair_of[r0 + lane] < 0);
    const Vec<T, VEC> zero = zero_vec<T, VEC>();
    for (; none; none &= none - 1) {
        T *const o = out + (r0 + __ffs(none) - 1) * dim;
        for (int c = c0 + lane; c < c1; c += 32)
            store_vec<T, VEC>(o + (int64_t)c * VEC, zero);
    }
}

constexpr int kGatherChunks = 4;             // vectors of a lane

template <typename T, int VEC>
__global__ void __launch_bounds__(kWarps * 32) gather_kernel(const MoeGatherArgs a, int segs)
{
    constexpr int U = kGatherChunks;
    const int lane = threadIdx.x & 31, chunks = a.dim / VEC;
    wait_for_previous();
    let_next_start();
    const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int64_t t = item / segs;
    const int c0 = (int)(item - t * segs) * 32 * U, c1 = min(chunks, c0 + 32 * U);
    if (t >= a.tokens) {
        if (a.pair_of && (t - a.tokens) * 32 < a.rows)
            clear_rows<T, VEC>(static_cast<T *>(a.out), a.pair_of, a.rows, a.dim, (t - a.tokens) * 32, c0, c1, lane);
        return;
    }
    const T *const x = static_cast<const T *>(a.x) + t * a.x_row;
    const int row = token_row(a.row_of, t, a.top_k, a.rows, lane);
    Vec<T, VEC> v[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (c0 + i * 32 + lane < c1)
            v[i] = load_vec<T, VEC>(x + (int64_t)(c0 + i * 32 + lane) * VEC);
    for (int j = 0; j < a.top_k; ++j) {
        const int r = __shfl_sync(kAll, row, j);
        if (r < 0)
            continue;
        T *const o = static_cast<T *>(a.out) + (int64_t)r * a.dim;
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (c0 + i * 32 + lane < c1)
                store_vec<T, VEC>(o + (int64_t)(c0 + i * 32 + lane) * VEC, v[i]);
    }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kWarps * 32) combine_kernel(const MoeCombineArgs a, int segs)
{
    constexpr int B = 8;                     // rows in flight
    const int lane = threadIdx.x & 31, chunks = a.dim / VEC;
    wait_for_previous();
    let_next_start();
    const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int64_t t = item / segs;
    const int c = (int)(item - t * segs) * 32 + lane;
    if (t >= a.tokens)
        return;
    const int row = token_row(a.row_of, t, a.top_k, a.rows, lane);
    const float w = lane < a.top_k ? a.weights ? a.weights[t * a.top_k + lane] : 1.f : 0.f;
    float sum[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        sum[e] = 0.f;
    for (int j0 = 0; j0 < a.top_k; j0 += B) {
        Vec<T, VEC> v[B];
        int r[B];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            r[j] = __shfl_sync(kAll, row, (j0 + j) & 31);
            r[j] = j0 + j < a.top_k && c < chunks ? r[j] : -1;
            if (r[j] >= 0)
                v[j] = load_vec<T, VEC>(static_cast<const T *>(a.y) + (int64_t)r[j] * a.dim + (int64_t)c * VEC);
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const float f = __shfl_sync(kAll, w, (j0 + j) & 31);
            if (r[j] >= 0)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    sum[e] += f * to_f32(v[j].v[e]);
        }
    }
    if (c < chunks) {
        Vec<T, VEC> o;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            from_f32(o.v[e], sum[e]);
        store_vec<T, VEC>(static_cast<T *>(a.out) + t * a.out_row + (int64_t)c * VEC, o);
    }
}

// A warp takes a pair; then warps clear 32 rows' columns by segments.
template <typename T, int VEC>
__global__ void __launch_bounds__(kWarps * 32) combine_grad_kernel(const MoeCombineGradArgs a, int segs)
{
    constexpr int U = 4;                     // vectors in flight
    const int lane = threadIdx.x & 31, chunks = a.dim / VEC;
    wait_for_previous();
    let_next_start();
    const int64_t pairs = a.tokens * a.top_k;
    const int64_t p = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (p >= pairs) {
        const int64_t s = (p - pairs) / segs;
        const int c0 = (int)(p - pairs - s * segs) * 128;
        if (a.pair_of && s * 32 < a.rows)
            clear_rows<T, VEC>(static_cast<T *>(a.dy), a.pair_of, a.rows, a.dim, s * 32, c0, min(chunks, c0 + 128), lane);
        return;
    }
    const int row = a.row_of[p];
    float dot = 0.f;
    if (row >= 0 && row < a.rows) {
        const float w = a.weights[p];
        const T *const d = static_cast<const T *>(a.dout) + p / a.top_k * a.dout_row;
        const T *const y = static_cast<const T *>(a.y) + (int64_t)row * a.dim;
        T *const dy = static_cast<T *>(a.dy) + (int64_t)row * a.dim;
        for (int c0 = lane; c0 < chunks; c0 += 32 * U) {
            Vec<T, VEC> vd[U], vy[U];
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (c0 + 32 * i < chunks) {
                    vd[i] = load_vec<T, VEC>(d + (int64_t)(c0 + 32 * i) * VEC);
                    vy[i] = load_vec<T, VEC>(y + (int64_t)(c0 + 32 * i) * VEC);
                }
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (c0 + 32 * i < chunks) {
                    Vec<T, VEC> o;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float g = to_f32(vd[i].v[e]);
                        dot += g * to_f32(vy[i].v[e]);
                        from_f32(o.v[e], w * g);
                    }
                    store_vec<T, VEC>(dy + (int64_t)(c0 + 32 * i) * VEC, o);
                }
        }
        dot = lane_sum(dot);
    }
    if (lane == 0)
        a.dweights[p] = dot;
}

// A warp takes 32 blocks of 32 elements of a token: a lane quantizes one
// block and stores its codes to the token's rows; the four lanes of a scale
// word share out the rows' words.
template <bool RES>
__global__ void __launch_bounds__(kWarps * 32) moe_quantize_kernel(const MoeQuantizeArgs a, int segs)
{
    const int lane = threadIdx.x & 31, kblocks = a.dim / 32;
    wait_for_previous();
    let_next_start();
    const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int64_t t = item / segs;
    const int b = (int)(item - t * segs) * 32 + lane;
    const bool ok = b < kblocks;             // (dim % 128 == 0: alike for the lanes of a scale word)
    uint4 *const mc = static_cast<uint4 *>(a.m_codes), *const rc = static_cast<uint4 *>(a.r_codes);
    uint8_t *const ms = static_cast<uint8_t *>(a.m_scales), *const rs = static_cast<uint8_t *>(a.r_scales);
    if (t >= a.tokens) {
        // rows of no pair, and the scale layout's rows behind the last
        const int64_t r0 = a.pad_from + (t - a.tokens) * 32, r = r0 + lane;
        const bool pad = r >= a.rows && r < a.padded;
        const uint32_t none = __ballot_sync(kAll, a.pair_of && r < a.rows && a.pair_of[r] < 0);
        for (uint32_t left = none | __ballot_sync(kAll, pad); left; left &= left - 1) {
            const int64_t row = r0 + __ffs(left) - 1;
            if (!ok)
                continue;
            if (row < a.rows) {
                mc[row * kblocks + b] = make_uint4(0, 0, 0, 0);
                if (RES)
                    rc[row * kblocks + b] = make_uint4(0, 0, 0, 0);
            }
            if ((lane & 3) == 0) {
                const int64_t at = sf_mma_offset(row, b, kblocks >> 2);
                *reinterpret_cast<uint32_t *>(ms + at) = 0;
                if (RES)
                    *reinterpret_cast<uint32_t *>(rs + at) = 0;
            }
        }
        return;
    }
    const int row = token_row(a.row_of, t, a.top_k, a.rows, lane);
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        w[i] = 0;
    if (ok) {
        const uint4 *const p = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.x) + t * a.x_row) + b * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4 *>(w + 4 * i) = p[i];
    }
    float xf[32];
    bf16x32_to_f32(w, xf);
    const Mx32 q = mxfp4_quant32<RES>(xf);
    // the scale word of each four lanes
    uint32_t sm = (uint32_t)q.sb << 8 * (lane & 3), sr = (uint32_t)q.rb << 8 * (lane & 3);
    sm |= __shfl_xor_sync(kAll, sm, 1);
    sm |= __shfl_xor_sync(kAll, sm, 2);
    if (RES) {
        sr |= __shfl_xor_sync(kAll, sr, 1);
        sr |= __shfl_xor_sync(kAll, sr, 2);
    }
    for (int j = 0; j < a.top_k; ++j) {
        const int r = __shfl_sync(kAll, row, j);
        if (r < 0 || !ok)
            continue;
        mc[(int64_t)r * kblocks + b] = q.code;
        if (RES)
            rc[(int64_t)r * kblocks + b] = q.rcode;
        if ((lane & 3) == (j & 3)) {
            const int64_t at = sf_mma_offset(r, b & ~3, kblocks >> 2);
            *reinterpret_cast<uint32_t *>(ms + at) = sm;
            if (RES)
                *reinterpret_cast<uint32_t *>(rs + at) = sr;
        }
    }
}

bool wide(int64_t bits, bool bf16) { return bits % (bf16 ? 8 : 4) == 0; }

// Blocks of kWarps warps for so many items.
bool blocks_of(int64_t items, unsigned &blocks)
{
    const int64_t n = (items + kWarps - 1) / kWarps;
    blocks = (unsigned)n;
    return n <= INT32_MAX;
}

template <typename T, int VEC>
cudaError_t gather(const MoeGatherArgs &a, cudaStream_t st)
{
    const int per = 32 * kGatherChunks, segs = (a.dim / VEC + per - 1) / per;
    unsigned blocks;
    if (!blocks_of((a.tokens + (a.pair_of ? (a.rows + 31) / 32 : 0)) * segs, blocks))
        return cudaErrorInvalidConfiguration;
    return blocks ? launch_early(gather_kernel<T, VEC>, dim3(blocks), kWarps * 32, 0, st, 1, a, segs) : cudaSuccess;
}

template <typename T, int VEC>
cudaError_t combine(const MoeCombineArgs &a, cudaStream_t st)
{
    const int segs = (a.dim / VEC + 31) / 32;
    unsigned blocks;
    if (!blocks_of(a.tokens * segs, blocks))
        return cudaErrorInvalidConfiguration;
    return launch_early(combine_kernel<T, VEC>, dim3(blocks), kWarps * 32, 0, st, 1, a, segs);
}

template <typename T, int VEC>
cudaError_t combine_grad(const MoeCombineGradArgs &a, cudaStream_t st)
{
    const int segs = (a.dim / VEC + 127) / 128;
    unsigned blocks;
    if (!blocks_of(a.tokens * a.top_k + (a.pair_of ? (a.rows + 31) / 32 * segs : 0), blocks))
        return cudaErrorInvalidConfiguration;
    return blocks ? launch_early(combine_grad_kernel<T, VEC>, dim3(blocks), kWarps * 32, 0, st, 1, a, segs) : cudaSuccess;
}

} // namespace

cudaError_t launch_moe_gather(const MoeGatherArgs &a, cudaStream_t st)
{
    const bool w = wide(a.x_row | a.dim, a.bf16);
    if (a.bf16)
        return w ? gather<__nv_bfloat16, 8>(a, st) : gather<__nv_bfloat16, 1>(a, st);
    return w ? gather<float, 4>(a, st) : gather<float, 1>(a, st);
}

cudaError_t launch_moe_combine(const MoeCombineArgs &a, cudaStream_t st)
{
    const bool w = wide(a.out_row | a.dim, a.bf16);
    if (a.bf16)
        return w ? combine<__nv_bfloat16, 8>(a, st) : combine<__nv_bfloat16, 1>(a, st);
    return w ? combine<float, 4>(a, st) : combine<float, 1>(a, st);
}

cudaError_t launch_moe_combine_grad(const MoeCombineGradArgs &a, cudaStream_t st)
{
    const bool w = wide(a.dout_row | a.dim, a.bf16);
    if (a.bf16)
        return w ? combine_grad<__nv_bfloat16, 8>(a, st) : combine_grad<__nv_bfloat16, 1>(a, st);
    return w ? combine_grad<float, 4>(a, st) : combine_grad<float, 1>(a, st);
}

cudaError_t launch_moe_quantize(const MoeQuantizeArgs &a, cudaStream_t st)
{
    const int segs = (a.dim / 32 + 31) / 32;
    MoeQuantizeArgs b = a;
    b.padded = (a.rows + 127) / 128 * 128;
    b.pad_from = a.pair_of ? 0 : a.rows / 32 * 32;   // (without pair_of only the layout's padding is cleared)
    unsigned blocks;
    if (!blocks_of((a.tokens + (b.padded - b.pad_from) / 32) * segs, blocks))
        return cudaErrorInvalidConfiguration;
    if (!blocks)
        return cudaSuccess;
    return a.r_codes ? launch_early(moe_quantize_kernel<true>, dim3(blocks), kWarps * 32, 0, st, 1, b, segs)
                     : launch_early(moe_quantize_kernel<false>, dim3(blocks), kWarps * 32, 0, st, 1, b, segs);
}

} // namespace rfq
