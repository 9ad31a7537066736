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
// elements), else single elements (VEC = 1).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "internal.h"

namespace rfq {
namespace {

constexpr int kThreads = 256;

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Vec {
    T v[VEC];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16 &d, float x) { d = __float2bfloat16_rn(x); }

// Block: tokens [blockIdx.x tb, + tb), heads in blockIdx.y's share.  An item is
// one chunk of VEC consecutive elements of the output, or with !INTER for
// rotated elements the chunk and its partner `pairs` elements further on.
template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeArgs a, int tb, int heads_per)
{
    extern __shared__ float2 s_cs[];         // [tb][pairs]
    const int64_t t0 = (int64_t)blockIdx.x * tb;
    const int nt = (int)min((int64_t)tb, a.tokens - t0);
    const int h0 = blockIdx.y * heads_per, nh = min(heads_per, a.heads - h0);
    const int P = a.pairs;
    for (int i = threadIdx.x; i < nt * P; i += kThreads) {
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

    const T *const x = static_cast<const T *>(a.x);
    T *const out = static_cast<T *>(a.out);
    using V = Vec<T, VEC>;
    const int D = a.head_dim;
    // chunks of a head: rotated ones first, then the elements that pass through
    constexpr int PV = VEC < 2 ? 2 : VEC;    // elements of an INTER chunk: whole pairs
    const int rot = INTER ? 2 * P / PV : P / VEC, chunks = rot + (D - 2 * P) / VEC;
    const int per_token = nh * chunks, items = nt * per_token;
    for (int i = threadIdx.x; i < items; i += kThreads) {
        const int t = i / per_token, r = i - t * per_token, h = r / chunks, c = r - h * chunks;
        const int64_t xo = (t0 + t) * a.x_token + (int64_t)(h0 + h) * a.x_head;
        const int64_t oo = (t0 + t) * a.out_token + (int64_t)(h0 + h) * a.out_head;
        if (c >= rot) {
            const int d = 2 * P + (c - rot) * VEC;
            *reinterpret_cast<V *>(out + oo + d) = *reinterpret_cast<const V *>(x + xo + d);
        } else if (INTER) {
            const int d = c * PV;
            alignas(sizeof(T) * PV) T v[PV];
#pragma unroll
            for (int j = 0; j < PV; j += VEC)
                *reinterpret_cast<V *>(v + j) = *reinterpret_cast<const V *>(x + xo + d + j);
#pragma unroll
            for (int j = 0; j < PV; j += 2) {
                const float2 cs = s_cs[t * P + (d + j) / 2];
                const float p = to_f32(v[j]), q = to_f32(v[j + 1]);
                from_f32(v[j], p * cs.x - q * cs.y);
                from_f32(v[j + 1], q * cs.x + p * cs.y);
            }
#pragma unroll
            for (int j = 0; j < PV; j += VEC)
                *reinterpret_cast<V *>(out + oo + d + j) = *reinterpret_cast<const V *>(v + j);
        } else {
            const int d = c * VEC;
            V v = *reinterpret_cast<const V *>(x + xo + d), w = *reinterpret_cast<const V *>(x + xo + d + P);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float2 cs = s_cs[t * P + d + j];
                const float p = to_f32(v.v[j]), q = to_f32(w.v[j]);
                from_f32(v.v[j], p * cs.x - q * cs.y);
                from_f32(w.v[j], q * cs.x + p * cs.y);
            }
            *reinterpret_cast<V *>(out + oo + d) = v;
            *reinterpret_cast<V *>(out + oo + d + P) = w;
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
    const int by = (int)min((int64_t)a.heads, max((int64_t)1, target / bx));
    const int hp = (a.heads + by - 1) / by;
    const dim3 grid((unsigned)bx, (unsigned)((a.heads + hp - 1) / hp));
    const size_t smem = (size_t)tb * a.pairs * sizeof(float2);
    if (a.interleaved)
        rope_kernel<T, VEC, true><<<grid, kThreads, smem, st>>>(a, tb, hp);
    else
        rope_kernel<T, VEC, false><<<grid, kThreads, smem, st>>>(a, tb, hp);
    return cudaGetLastError();
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
