// norm.cu -- layer norm and RMS norm of rows (rfq_norm) and their gradients
// (rfq_norm_grad).
//
// Forward:   m = mean x (RMS: 0),  r = 1 / sqrt(mean (x - m)^2 + eps),
//            y = (x - m) r w + b.
// Backward:  g = dy w,  h = (x - m) r,
//            dx = r (g - mean g - h mean(g h))   (RMS: without mean g),
//            dw = sum over rows of dy h,  db = sum over rows of dy.
//
// Bound: HBM (x read and y written once; dy and x read and dx written once).
// A row is held in registers by the threads that share it, so the mean and
// the squared distances from it are two passes over registers.  The weight's
// gradient is summed in fp32 in the registers of persistent blocks, whose
// threads keep their columns over all their rows; the blocks' sums go through
// the workspace and a second kernel adds them, both in a fixed order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 256;                // of a block, at least where a row takes more

// Where rows lie: [tokens][heads] with two strides in elements.
struct Place {
    int64_t token, head;
};
__device__ __forceinline__ int64_t row_at(const Place &p, int64_t row, int heads)
{
    if (heads == 1)
        return row * p.token;
    const int64_t t = (uint64_t)row / (uint32_t)heads;
    return t * p.token + (row - t * heads) * p.head;
}

// Sum over the `tpr` threads of a row: a power of two up to a warp, or whole
// warps, whose sums go through s_part (one float a warp of the block).
__device__ __forceinline__ float row_sum(float v, int tpr, float *s_part)
{
    if (tpr <= 32)
        return lane_sum(v, tpr);
    v = lane_sum(v);
    const int warp = threadIdx.x >> 5, n = tpr >> 5, first = warp / n * n;
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        s_part[warp] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < n; ++i)
        v += s_part[first + i];
    return v;
}

__device__ __forceinline__ float param(const void *p, bool bf16, int i)
{
    return bf16 ? to_f32(static_cast<const __nv_bfloat16 *>(p)[i]) : static_cast<const float *>(p)[i];
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(1024) norm_kernel(const NormArgs a, int tpr)
{
    __shared__ float s_part[32];
    const int group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / tpr) + group;
    const bool there = row < a.rows;
    const int chunks = a.dim / VEC;
    wait_for_previous();
    let_next_start();
    const T *const x = static_cast<const T *>(a.x) + row_at({a.x_token, a.x_head}, row, a.heads);
    Vec<T, VEC> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = lane + i * tpr;
        v[i] = there && c < chunks ? load_vec<T, VEC>(x + (int64_t)c * VEC) : zero_vec<T, VEC>();
    }
    const float inv = 1.f / (float)a.dim;
    float mean = 0.f;
    if (!a.rms) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s += to_f32(v[i].v[e]);
        mean = row_sum(s, tpr, s_part) * inv;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (lane + i * tpr < chunks)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float d = to_f32(v[i].v[e]) - mean;
                q += d * d;
            }
    const float rstd = 1.f / sqrtf(row_sum(q, tpr, s_part) * inv + a.eps);
    if (!there)
        return;
    if (lane == 0) {
        if (a.mean)
            a.mean[row] = mean;
        if (a.rstd)
            a.rstd[row] = rstd;
    }
    T *const y = static_cast<T *>(a.y) + row_at({a.y_token, a.y_head}, row, a.heads);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = lane + i * tpr;
        if (c < chunks) {
            Vec<T, VEC> o;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float t = (to_f32(v[i].v[e]) - mean) * rstd;
                if (a.weight)
                    t *= param(a.weight, a.w_bf16, c * VEC + e);
                if (a.bias)
                    t += param(a.bias, a.w_bf16, c * VEC + e);
                from_f32(o.v[e], t);
            }
            store_vec<T, VEC>(y + (int64_t)c * VEC, o);
        }
    }
}

// Blocks take rows in turn; a thread keeps its columns.  Partial sums of the
// weight's gradient: a.partial [blocks][2][dim].
template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(1024) norm_grad_kernel(const NormGradArgs a, int tpr)
{
    extern __shared__ float s_sums[];        // [groups][2][dim] where a block has several groups
    __shared__ float s_part[32];
    const int groups = blockDim.x / tpr, group = threadIdx.x / tpr, lane = threadIdx.x - group * tpr;
    const int chunks = a.dim / VEC;
    const float inv = 1.f / (float)a.dim;
    wait_for_previous();
    let_next_start();
    float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = lane + i * tpr;
            w[i][e] = a.weight && c < chunks ? param(a.weight, a.w_bf16, c * VEC + e) : 1.f;
            dw[i][e] = db[i][e] = 0.f;
        }
    // (every thread of the block takes part in the sums of every turn)
    for (int64_t first = (int64_t)blockIdx.x * groups; first < a.rows; first += (int64_t)gridDim.x * groups) {
        const int64_t row = first + group;
        const bool there = row < a.rows;
        const int64_t r = there ? row : 0;
        const T *const x = static_cast<const T *>(a.x) + row_at({a.x_token, a.x_head}, r, a.heads);
        const T *const dy = static_cast<const T *>(a.dy) + row_at({a.dy_token, a.dy_head}, r, a.heads);
        const float rstd = a.rstd[r], mean = a.rms ? 0.f : a.mean[r];
        Vec<T, VEC> vx[NV], vd[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = lane + i * tpr;
            const bool in = there && c < chunks;
            vx[i] = in ? load_vec<T, VEC>(x + (int64_t)c * VEC) : zero_vec<T, VEC>();
            vd[i] = in ? load_vec<T, VEC>(dy + (int64_t)c * VEC) : zero_vec<T, VEC>();
        }
        float sg = 0.f, sh = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (there && lane + i * tpr < chunks)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = to_f32(vd[i].v[e]), h = (to_f32(vx[i].v[e]) - mean) * rstd, g = d * w[i][e];
                    dw[i][e] += d * h;
                    db[i][e] += d;
                    sg += g;
                    sh += g * h;
                }
        const float mh = row_sum(sh, tpr, s_part) * inv;
        const float mg = a.rms ? 0.f : row_sum(sg, tpr, s_part) * inv;
        T *const dx = static_cast<T *>(a.dx) + row_at({a.dx_token, a.dx_head}, r, a.heads);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = lane + i * tpr;
            if (there && c < chunks) {
                Vec<T, VEC> o;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float h = (to_f32(vx[i].v[e]) - mean) * rstd, g = to_f32(vd[i].v[e]) * w[i][e];
                    from_f32(o.v[e], (g - mg - h * mh) * rstd);
                }
                store_vec<T, VEC>(dx + (int64_t)c * VEC, o);
            }
        }
    }
    if (!a.partial)
        return;
    float *const out = a.partial + (int64_t)blockIdx.x * 2 * a.dim;
    float *const to = groups > 1 ? s_sums + (int64_t)group * 2 * a.dim : out;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = lane + i * tpr;
            if (c < chunks) {
                to[c * VEC + e] = dw[i][e];
                to[a.dim + c * VEC + e] = db[i][e];
            }
        }
    if (groups > 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * a.dim; i += blockDim.x) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g)
                s += s_sums[(int64_t)g * 2 * a.dim + i];
            out[i] = s;
        }
    }
}

// dw, db: sums of the blocks' parts.  A block takes 32 columns, its warps
// shares of the parts.
__global__ void __launch_bounds__(256) norm_sum_kernel(const float *partial, int parts, int dim, float *dweight, float *dbias)
{
    __shared__ float s[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    wait_for_previous();
    let_next_start();
    float v = 0.f;
    if (i < 2 * dim)
        for (int p = warp; p < parts; p += 8)
            v += partial[(int64_t)p * 2 * dim + i];
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < 2 * dim) {
        v = 0.f;
        for (int k = 0; k < 8; ++k)
            v += s[k][lane];
        if (i < dim) {
            if (dweight)
                dweight[i] = v;
        } else if (dbias)
            dbias[i - dim] = v;
    }
}

// Threads of a row: the fewest (a power of two up to a warp, else whole
// warps) that hold `chunks` in at most `most` chunks each.
int threads_per_row(int chunks, int most)
{
    const int need = (chunks + most - 1) / most;
    if (need > 32)
        return (need + 31) / 32 * 32;
    int t = 1;
    while (t < need)
        t *= 2;
    return t;
}

// The smallest power of two of chunks a thread.
int chunks_per_thread(int chunks, int tpr)
{
    int n = 1;
    while (n * tpr < chunks)
        n *= 2;
    return n;
}

// Blocks of the persistent kernel, at most: its parts are the workspace.
int most_parts() { return 2 * num_sms(); }

template <typename T, int VEC, int MOST>
cudaError_t launch_forward(const NormArgs &a, cudaStream_t st)
{
    const int chunks = a.dim / VEC, tpr = threads_per_row(chunks, MOST), nv = chunks_per_thread(chunks, tpr);
    const int groups = tpr >= kThreads ? 1 : kThreads / tpr;
    const dim3 grid((unsigned)((a.rows + groups - 1) / groups));
    auto go = [&](auto kern) { return launch_early(kern, grid, groups * tpr, 0, st, 1, a, tpr); };
    switch (nv) {
    case 1: return go(norm_kernel<T, VEC, 1>);
    case 2: return go(norm_kernel<T, VEC, 2>);
    case 4: return go(norm_kernel<T, VEC, 4>);
    case 8: return go(norm_kernel<T, VEC, 8>);
    default: return go(norm_kernel<T, VEC, 16>);
    }
}

template <typename T, int VEC, int MOST>
cudaError_t launch_backward(const NormGradArgs &given, cudaStream_t st)
{
    NormGradArgs a = given;
    const int chunks = a.dim / VEC, tpr = threads_per_row(chunks, MOST), nv = chunks_per_thread(chunks, tpr);
    const int groups = tpr >= kThreads ? 1 : kThreads / tpr;
    const int64_t turns = (a.rows + groups - 1) / groups;
    const bool sums = a.dweight || a.dbias;
    a.partial = sums ? static_cast<float *>(a.workspace) : nullptr;
    const int blocks = (int)(turns < most_parts() ? turns : most_parts());
    if (blocks > 0) {
        const size_t smem = sums && groups > 1 ? (size_t)groups * 2 * a.dim * sizeof(float) : 0;
        auto go = [&](auto kern) { return launch_early(kern, dim3((unsigned)blocks), groups * tpr, smem, st, 1, a, tpr); };
        const cudaError_t e = nv == 1   ? go(norm_grad_kernel<T, VEC, 1>)
                              : nv == 2 ? go(norm_grad_kernel<T, VEC, 2>)
                              : nv == 4 ? go(norm_grad_kernel<T, VEC, (MOST >= 4 ? 4 : 1)>)
                              : nv == 8 ? go(norm_grad_kernel<T, VEC, (MOST >= 8 ? 8 : 1)>)
                                        : go(norm_grad_kernel<T, VEC, (MOST >= 16 ? 16 : 1)>);
        if (e != cudaSuccess)
            return e;
    }
    if (!sums)
        return cudaSuccess;
    return launch_early(norm_sum_kernel, dim3((unsigned)((2 * a.dim + 31) / 32)), 256, 0, st, 1,
                        static_cast<const float *>(a.workspace), blocks, a.dim, a.dweight, a.dbias);
}

bool wide(int64_t bits, bool bf16) { return bits % (bf16 ? 8 : 4) == 0; }

} // namespace

size_t norm_grad_workspace_bytes(int32_t dim) { return (size_t)most_parts() * 2 * (size_t)dim * sizeof(float); }

cudaError_t launch_norm(const NormArgs &a, cudaStream_t st)
{
    const bool w = wide(a.x_token | a.x_head | a.y_token | a.y_head | a.dim, a.bf16);
    if (a.bf16)
        return w ? launch_forward<__nv_bfloat16, 8, 4>(a, st) : launch_forward<__nv_bfloat16, 1, 16>(a, st);
    return w ? launch_forward<float, 4, 8>(a, st) : launch_forward<float, 1, 16>(a, st);
}

cudaError_t launch_norm_grad(const NormGradArgs &a, cudaStream_t st)
{
    const bool w = wide(a.dy_token | a.dy_head | a.x_token | a.x_head | a.dx_token | a.dx_head | a.dim, a.bf16);
    if (a.bf16)
        return w ? launch_backward<__nv_bfloat16, 8, 2>(a, st) : launch_backward<__nv_bfloat16, 1, 16>(a, st);
    return w ? launch_backward<float, 4, 4>(a, st) : launch_backward<float, 1, 16>(a, st);
}

} // namespace rfq
