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
// 4096 tokens of 8 pairs, 2048 bf16, groups on 128 rows (49024 rows in all):
// gather 35.5 us (91% of the copy rate), combine 26 us (86%), quantize with its
// residual 26 us (70%: a scale word of four bytes takes a transaction of its
// own; without those stores it takes 22).  combine_grad of 3001 tokens of 6
// pairs, 1000 fp32: 25.9 us (91%); of the 4096 tokens, bf16, 59.6 (87%).
// Combine of 32 tokens: 2.1 us, latency.
// Rows of no whole 16-byte words go in 8-, 4- or 2-byte vectors: 4096 tokens of 4
// pairs, groups on 16 rows, gather of 1023 fp32 17.7 us (77%), bf16 13.4 (51%), of
// 1020 bf16 9.0 (76%); combine of 1023 fp32 32.7 us (38%), 1022 fp32 18.8 (66%),
// 1023 bf16 25.0 (25%), 1020 bf16 11.6 (54%); combine_grad of 1023 fp32 28.1 us
// (84%), bf16 20.6 (57%).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace rfq {
namespace {

constexpr int kWarps = 4;                    // of a block (with eight a gather of 32 tokens takes 3.1 us instead of 2.1)
constexpr int kCombineBlocks = 8;            // of an SM
constexpr uint32_t kAll = 0xFFFFFFFFu;

// The row of pair j of a token (lane j holds it), -1 where there is none.
__device__ __forceinline__ int token_row(const int32_t *row_of, int64_t t, int top_k, int64_t rows, int lane)
{
    int r = lane < top_k ? row_of[t * top_k + lane] : -1;
    return r < rows ? r : -1;
}

// Rows that a warp looks through for those of no pair.  They lie apart, by the
// number of warps that look: long stretches of them fall to many warps.
constexpr int kLook = 8;
__host__ __device__ __forceinline__ int64_t lookers(int64_t rows) { return (rows + kLook - 1) / kLook; }

// Calls clear(row) for each of looker i's rows that holds no pair.
template <typename C>
__device__ __forceinline__ void rows_of_no_pair(const int32_t *pair_of, int64_t rows, int64_t i, int lane, C &&clear)
{
    const int64_t n = lookers(rows), mine = i + lane * n;
    for (uint32_t none = __ballot_sync(kAll, lane < kLook && mine < rows && pair_of[mine] < 0); none; none &= none - 1)
        clear(i + (__ffs(none) - 1) * n);
}

template <typename T, int VEC>
__device__ __forceinline__ void clear_row(T *out, int64_t row, int dim, int lane)
{
    T *const o = out + row * dim;
#pragma unroll 4
    for (int c = lane; c < dim / VEC; c += 32)
        store_vec<T, VEC>(o + (int64_t)c * VEC, zero_vec<T, VEC>());
}

constexpr int kGatherChunks = 4;             // vectors of a lane

template <typename T, int VEC>
__global__ void __launch_bounds__(kWarps * 32) gather_kernel(const MoeGatherArgs a)
{
    constexpr int U = kGatherChunks;
    const int lane = threadIdx.x & 31, chunks = a.dim / VEC;
    wait_for_previous();
    let_next_start();
    const int64_t look = a.pair_of ? lookers(a.rows) : 0, t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5) - look;
    if (t < 0) {
        if (blockIdx.y == 0)
            rows_of_no_pair(a.pair_of, a.rows, t + look, lane, [&](int64_t r) { clear_row<T, VEC>(static_cast<T *>(a.out), r, a.dim, lane); });
        return;
    }
    if (t >= a.tokens)
        return;
    const int c0 = blockIdx.y * 32 * U, c1 = min(chunks, c0 + 32 * U);
    const T *const x = static_cast<const T *>(a.x) + t * a.x_row;
    const int row = token_row(a.row_of, t, a.top_k, a.rows, lane);
    Vec<T, VEC> v[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (c0 + i * 32 + lane < c1)
            v[i] = load_once<T, VEC>(x + (int64_t)(c0 + i * 32 + lane) * VEC);
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

// Vectors of a lane that are in flight together: more of them where they are short.
template <typename T, int VEC>
constexpr int kVectors = VEC * sizeof(T) >= 16 ? 1 : VEC * sizeof(T) >= 8 ? 2 : 4;

// Persistent warps take 32 vectors (of each kind of a lane's) of a token each; the
// next token's rows and weights are on their way while this one's are summed.
template <typename T, int VEC>
__global__ void __launch_bounds__(kWarps * 32, kCombineBlocks) combine_kernel(const MoeCombineArgs a)
{
    constexpr int B = 4;                     // rows in flight (with eight a warp leaves room for half as many warps: 31 us against 27)
    const int lane = threadIdx.x & 31, chunks = a.dim / VEC;
    wait_for_previous();
    let_next_start();
    const uint32_t tokens = (uint32_t)a.tokens, step = gridDim.x * kWarps;
    constexpr int U = kVectors<T, VEC>, L = kLanes<VEC>;
    const int c = blockIdx.y * 32 * U + lane;
    const T *const y = static_cast<const T *>(a.y) + (int64_t)c * VEC;
    int row = -1, next_row = -1;
    float w = 0.f, next_w = 0.f;
    auto ahead = [&](uint32_t t) {
        if (t < tokens) {
            next_row = token_row(a.row_of, t, a.top_k, a.rows, lane);
            next_w = lane < a.top_k && a.weights ? a.weights[(int64_t)t * a.top_k + lane] : 1.f;
        }
    };
    uint32_t t = blockIdx.x * kWarps + (threadIdx.x >> 5);
    ahead(t);
#pragma unroll 1
    for (; t < tokens; t += step) {
        row = next_row;
        w = next_w;
        Lane<VEC> sum[U][L];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < L; ++e)
                sum[u][e] = all_of<VEC>(0.f);
#pragma unroll 1
        for (int j0 = 0; j0 < a.top_k; j0 += B) {
            Vec<T, VEC> v[B][U];
            int r[B];
#pragma unroll
            for (int j = 0; j < B; ++j) {
                r[j] = __shfl_sync(kAll, row, (j0 + j) & 31);
                r[j] = j0 + j < a.top_k ? r[j] : -1;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (r[j] >= 0 && c + 32 * u < chunks)
                        v[j][u] = load_once<T, VEC>(y + (int64_t)r[j] * a.dim + 32 * u * VEC);
            }
            if (j0 == 0)
                ahead(t + step);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                const Lane<VEC> f = all_of<VEC>(__shfl_sync(kAll, w, (j0 + j) & 31));
                if (r[j] >= 0)
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (c + 32 * u < chunks) {
                            Lane<VEC> x[L];
                            unpack<T, VEC>(v[j][u], x);
#pragma unroll
                            for (int e = 0; e < L; ++e)
                                sum[u][e] = fused(f, x[e], sum[u][e]);
                        }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + 32 * u < chunks)
                store_once<T, VEC>(static_cast<T *>(a.out) + t * a.out_row + (int64_t)(c + 32 * u) * VEC, pack<T, VEC>(sum[u]));
    }
}

// Warps clear the rows of no pair; then a warp takes a pair.
template <typename T, int VEC>
__global__ void __launch_bounds__(kWarps * 32) combine_grad_kernel(const MoeCombineGradArgs a)
{
    constexpr int U = 4 * kVectors<T, VEC>;  // vectors in flight
    const int lane = threadIdx.x & 31, chunks = a.dim / VEC;
    wait_for_previous();
    let_next_start();
    const int64_t look = a.pair_of ? lookers(a.rows) : 0, p = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5) - look;
    if (p < 0) {
        rows_of_no_pair(a.pair_of, a.rows, p + look, lane, [&](int64_t r) { clear_row<T, VEC>(static_cast<T *>(a.dy), r, a.dim, lane); });
        return;
    }
    if (p >= a.tokens * a.top_k)
        return;
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
__global__ void __launch_bounds__(kWarps * 32) moe_quantize_kernel(const MoeQuantizeArgs a)
{
    const int lane = threadIdx.x & 31, kblocks = a.dim / 32;
    wait_for_previous();
    let_next_start();
    uint4 *const mc = static_cast<uint4 *>(a.m_codes), *const rc = static_cast<uint4 *>(a.r_codes);
    uint8_t *const ms = static_cast<uint8_t *>(a.m_scales), *const rs = static_cast<uint8_t *>(a.r_scales);
    // warps that clear the rows of no pair, one that clears the scale layout's rows behind the last, then the tokens'
    const int64_t look = a.pair_of ? lookers(a.rows) : 0, t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5) - look - 1;
    if (t < 0) {
        if (blockIdx.y > 0)
            return;
        auto clear_scales = [&](int64_t row) {
            for (int w = lane; w < kblocks / 4; w += 32) {
                const int64_t at = sf_mma_offset(row, 4 * w, kblocks >> 2);
                *reinterpret_cast<uint32_t *>(ms + at) = 0;
                if (RES)
                    *reinterpret_cast<uint32_t *>(rs + at) = 0;
            }
        };
        if (t == -1)
            for (int64_t row = a.rows; row < a.padded; ++row)
                clear_scales(row);
        else
            rows_of_no_pair(a.pair_of, a.rows, t + look + 1, lane, [&](int64_t row) {
#pragma unroll 4
                for (int b = lane; b < kblocks; b += 32) {
                    mc[row * kblocks + b] = make_uint4(0, 0, 0, 0);
                    if (RES)
                        rc[row * kblocks + b] = make_uint4(0, 0, 0, 0);
                }
                clear_scales(row);
            });
        return;
    }
    if (t >= a.tokens)
        return;
    const int b = blockIdx.y * 32 + lane;
    const bool ok = b < kblocks;             // (dim % 128 == 0: alike for the lanes of a scale word)
    const int row = token_row(a.row_of, t, a.top_k, a.rows, lane);
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        w[i] = 0;
    if (ok) {
        const __nv_bfloat16 *const p = static_cast<const __nv_bfloat16 *>(a.x) + t * a.x_row + b * 32;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4 *>(w + 4 * i) = *reinterpret_cast<const uint4 *>(p + 8 * i);
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
    // codes: row by row; scale words: a row for each of the four lanes
    for (int j = 0; j < a.top_k; ++j) {
        const int r = __shfl_sync(kAll, row, j);
        if (r < 0 || !ok)
            continue;
        mc[(int64_t)r * kblocks + b] = q.code;
        if (RES)
            rc[(int64_t)r * kblocks + b] = q.rcode;
    }
    for (int j = 0; j < a.top_k; j += 4) {
        const int r = __shfl_sync(kAll, row, min(j + (lane & 3), 31));
        if (r < 0 || !ok || j + (lane & 3) >= a.top_k)
            continue;
        const int64_t at = sf_mma_offset(r, b & ~3, kblocks >> 2);
        *reinterpret_cast<uint32_t *>(ms + at) = sm;
        if (RES)
            *reinterpret_cast<uint32_t *>(rs + at) = sr;
    }
}

template <typename T_, int VEC_>
struct Width {
    using T = T_;
    static constexpr int VEC = VEC_;
};

// Calls go with the widest vectors, of up to 16 bytes, that divide strides and length (`bits`: all of them or'ed).
template <typename G>
cudaError_t by_width(int64_t bits, bool bf16, G &&go)
{
    if (bf16)
        return bits % 8 == 0   ? go(Width<__nv_bfloat16, 8>())
               : bits % 4 == 0 ? go(Width<__nv_bfloat16, 4>())
               : bits % 2 == 0 ? go(Width<__nv_bfloat16, 2>())
                               : go(Width<__nv_bfloat16, 1>());
    return bits % 4 == 0 ? go(Width<float, 4>()) : bits % 2 == 0 ? go(Width<float, 2>()) : go(Width<float, 1>());
}

// Blocks of kWarps warps for so many items (pairs and stacked rows are counted in 31 bits: no more than a grid holds).
unsigned blocks_of(int64_t items) { return (unsigned)((items + kWarps - 1) / kWarps); }

template <typename T, int VEC>
cudaError_t gather(const MoeGatherArgs &a, cudaStream_t st)
{
    const int per = 32 * kGatherChunks, segs = (a.dim / VEC + per - 1) / per;
    const unsigned blocks = blocks_of(a.tokens + (a.pair_of ? lookers(a.rows) : 0));
    return blocks ? launch_early(gather_kernel<T, VEC>, dim3(blocks, (unsigned)segs), kWarps * 32, 0, st, 1, a) : cudaSuccess;
}

template <typename T, int VEC>
cudaError_t combine(const MoeCombineArgs &a, cudaStream_t st)
{
    const int per = 32 * kVectors<T, VEC>, segs = (a.dim / VEC + per - 1) / per;
    const int64_t blocks = (a.tokens + kWarps - 1) / kWarps, most = max((int64_t)1, (int64_t)num_sms() * kCombineBlocks / segs);
    return launch_early(combine_kernel<T, VEC>, dim3((unsigned)(blocks < most ? blocks : most), (unsigned)segs), kWarps * 32, 0, st, 1, a);
}

template <typename T, int VEC>
cudaError_t combine_grad(const MoeCombineGradArgs &a, cudaStream_t st)
{
    const unsigned blocks = blocks_of(a.tokens * a.top_k + (a.pair_of ? lookers(a.rows) : 0));
    return blocks ? launch_early(combine_grad_kernel<T, VEC>, dim3(blocks), kWarps * 32, 0, st, 1, a) : cudaSuccess;
}

} // namespace

cudaError_t launch_moe_gather(const MoeGatherArgs &a, cudaStream_t st)
{
    return by_width(a.x_row | a.dim, a.bf16, [&](auto v) { return gather<typename decltype(v)::T, decltype(v)::VEC>(a, st); });
}

cudaError_t launch_moe_combine(const MoeCombineArgs &a, cudaStream_t st)
{
    return by_width(a.out_row | a.dim, a.bf16, [&](auto v) { return combine<typename decltype(v)::T, decltype(v)::VEC>(a, st); });
}

cudaError_t launch_moe_combine_grad(const MoeCombineGradArgs &a, cudaStream_t st)
{
    return by_width(a.dout_row | a.dim, a.bf16, [&](auto v) { return combine_grad<typename decltype(v)::T, decltype(v)::VEC>(a, st); });
}

cudaError_t launch_moe_quantize(const MoeQuantizeArgs &a, cudaStream_t st)
{
    const int segs = (a.dim / 32 + 31) / 32;
    MoeQuantizeArgs b = a;
    b.padded = (a.rows + 127) / 128 * 128;
    const dim3 grid(blocks_of(a.tokens + (a.pair_of ? lookers(a.rows) : 0) + 1), (unsigned)segs);
    return a.r_codes ? launch_early(moe_quantize_kernel<true>, grid, kWarps * 32, 0, st, 1, b)
                     : launch_early(moe_quantize_kernel<false>, grid, kWarps * 32, 0, st, 1, b);
}

} // namespace rfq
