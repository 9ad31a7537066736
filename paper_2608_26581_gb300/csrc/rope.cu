// rope.cu -- rotary positions with several axes (rfq_rope): every pair i of a
// head's elements is turned by angle = position[axis_i][token] * inv_freq_i,
//     (a, b) -> (a cos - b sin, b cos + a sin),
// or by -angle (`inverse`), which is the gradient: the rotation is orthogonal.
//
// Bound: HBM (each element read and written once).  The sine and cosine of a
// (token, pair) are computed once for all heads of the block's tokens and kept
// in shared memory.  The angle is formed in turns in fp64 and reduced there
// (three operations), so that a position of 10^6 keeps the full fp32 accuracy
// of its sine; everything else is fp32, rounded once to the output's type.
// Loads and stores are 16 bytes wide where strides and sizes allow (VEC
// elements), else single elements (VEC = 1).  32760 tokens of 40 heads of 128,
// bf16, three axes: 111 us, 6.05 TB/s, 90% of the copy rate; 4096 tokens
// in fp32, backwards, 32 us at 76% (short: its first loads and last wave show).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"

namespace rfq {
namespace {

constexpr int kThreads = 256;                // of a block, at most (more where a head has more chunks)
constexpr int kMostHeads = 65536;            // of a block: its rows, of four tokens, are told apart in fp32
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Vec {
    T v[VEC];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16 &d, float x) { d = __float2bfloat16_rn(x); }

// Block: tokens [blockIdx.x tb, + tb), heads in blockIdx.y's share; a row is
// one (token, head).  A thread takes the same chunk of every row it visits:
// VEC consecutive elements (a whole pair at least with INTER), or with !INTER
// for rotated elements the chunk and its partner `pairs` elements further on.
template <typename T, int VEC, bool INTER>
__global__ void rope_kernel(const RopeArgs a, int tb, int heads_per, int chunks, int rot)
{
    extern __shared__ float2 s_cs[];         // [tb][pairs]
    const int64_t t0 = (int64_t)blockIdx.x * tb;
    const int nt = (int)min((int64_t)tb, a.tokens - t0);
    const int h0 = blockIdx.y * heads_per, nh = min(heads_per, a.heads - h0);
    const int P = a.pairs;
    const T *const x = static_cast<const T *>(a.x) + t0 * a.x_token + h0 * a.x_head;
    T *const out = static_cast<T *>(a.out) + t0 * a.out_token + h0 * a.out_head;
    using V = Vec<T, VEC>;
    constexpr int PV = INTER && VEC < 2 ? 2 : VEC;      // elements of a chunk
    constexpr int NV = INTER ? PV / VEC : 2;            // vectors of a chunk: of a pair, or a chunk and its partner
    const int c = threadIdx.x % chunks, step = blockDim.x / chunks, rows = nt * nh;
    const bool turn = c < rot;
    // first element; distance of the second vector (a chunk that passes through has one)
    const int d = turn ? c * PV : 2 * P + (c - rot) * VEC;
    const int dist = INTER ? VEC : P, nv = turn ? NV : 1;
    const float inv_nh = 1.f / (float)nh;
    auto token_of = [&](int r) { return (int)(((float)r + 0.5f) * inv_nh); };   // r / nh (nh <= kMostHeads, r < 4 nh)
    auto load = [&](int r, V (&v)[NV]) {
        const int t = token_of(r), h = r - t * nh;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < nv)
                v[i] = *reinterpret_cast<const V *>(x + t * a.x_token + h * a.x_head + d + i * dist);
    };
    // the first row is on its way while the angles are formed, every other
    // while the one before it is turned
    int r = threadIdx.x / chunks;
    V v[NV];
    wait_for_previous();
    let_next_start();
    if (r < rows)
        load(r, v);
    for (int i = threadIdx.x; i < nt * P; i += blockDim.x) {
        const int t = i / P, p = i - t * P;
        const int axis = a.axis_of[p];
        float2 cs = make_float2(1.f, 0.f);
        if (axis >= 0 && axis < a.axes) {
            const double turns = (double)a.positions[(int64_t)axis * a.tokens + t0 + t] *
                                 ((double)a.inv_freq[p] * 0.15915494309189533577); // 1 / (2 pi)
            const float half = (float)(2.0 * (turns - rint(turns)));                  // angle / pi in [-1, 1]
            sincospif(a.inverse ? -half : half, &cs.y, &cs.x);
        }
        s_cs[i] = cs;
    }
    __syncthreads();

#pragma unroll 1
    for (; r < rows; r += step) {
        V next[NV];
        if (r + step < rows)
            load(r + step, next);
        const int t = token_of(r), h = r - t * nh;
        if (turn) {
            const float2 *const cs = s_cs + t * P + (INTER ? d / 2 : d);
#pragma unroll
            for (int j = 0; j < (INTER ? PV / 2 : VEC); ++j) {
                T &e0 = INTER ? v[2 * j / VEC].v[2 * j % VEC] : v[0].v[j];
                T &e1 = INTER ? v[(2 * j + 1) / VEC].v[(2 * j + 1) % VEC] : v[NV - 1].v[j];
                const float2 w = cs[j];
                const float p = to_f32(e0), q = to_f32(e1);
                from_f32(e0, p * w.x - q * w.y);
                from_f32(e1, q * w.x + p * w.y);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i < nv)
                *reinterpret_cast<V *>(out + t * a.out_token + h * a.out_head + d + i * dist) = v[i];
            v[i] = next[i];
        }
    }
}

template <typename T, int VEC>
cudaError_t launch(const RopeArgs &a, cudaStream_t st)
{
    // four tokens a block fill its threads with angles at 64 pairs; fewer
    // where that leaves SMs without a block, and then the heads are split
    const int64_t target = 2ll * num_sms();
    int tb = (int)min((int64_t)4, max((int64_t)1, a.tokens / target));
    const int64_t bx = (a.tokens + tb - 1) / tb;
    const int by = (int)min((int64_t)a.heads, max(((int64_t)a.heads + kMostHeads - 1) / kMostHeads, target / bx));
    const int hp = (int)(((int64_t)a.heads + by - 1) / by);
    const dim3 grid((unsigned)bx, (unsigned)(((int64_t)a.heads + hp - 1) / hp));
    const size_t smem = (size_t)tb * a.pairs * sizeof(float2);
    // chunks of a head: rotated ones first, then the elements that pass through
    const int pv = a.interleaved && VEC < 2 ? 2 : VEC;
    const int rot = a.interleaved ? 2 * a.pairs / pv : a.pairs / VEC;
    const int chunks = rot + (a.head_dim - 2 * a.pairs) / VEC;
    const int threads = chunks >= kThreads ? chunks : kThreads / chunks * chunks;
    if (a.interleaved)
        return launch_early(rope_kernel<T, VEC, true>, grid, threads, smem, st, 1, a, tb, hp, chunks, rot);
    return launch_early(rope_kernel<T, VEC, false>, grid, threads, smem, st, 1, a, tb, hp, chunks, rot);
}

} // namespace

cudaError_t launch_rope(const RopeArgs &a, cudaStream_t st)
{
    const int vec = a.bf16 ? 8 : 4;
    const bool wide = (a.x_token | a.x_head | a.out_token | a.out_head | a.head_dim) % vec == 0 &&
                      (a.interleaved ? 2 * a.pairs : a.pairs) % vec == 0;
    if (a.bf16)
        return wide ? launch<__nv_bfloat16, 8>(a, st) : launch<__nv_bfloat16, 1>(a, st);
    return wide ? launch<float, 4>(a, st) : launch<float, 1>(a, st);
}

} // namespace rfq
