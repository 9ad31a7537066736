// route.cu -- the router of a mixture of experts: each token's top_k experts
// and their weights from the experts' logits (rfq_route), and the logits'
// gradient (rfq_route_grad).
//
// With p = softmax(l) over a token's logits and e_j its j-th largest,
//     w_j = p[e_j],  or with normalize  w_j = p[e_j] / sum_m p[e_m],
// which is the softmax over the chosen logits alone.  Gradient, with d_i the
// sum of dw_j over the j that chose expert i and p restricted to the chosen
// experts with normalize:
//     dl_i = p_i (d_i - sum_m p_m d_m).
//
// A warp takes a token; lane i holds the logits of experts i, i + 32, ...  A
// choice is the maximum over the warp of the logits as ordered integers, then
// the lowest expert that has it.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cmath>
#include <type_traits>
#include <cstdint>

#include "internal.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace rfq {
namespace {

constexpr int kWarps = 8;                    // tokens of a block
constexpr uint32_t kAll = 0xFFFFFFFFu;

// Logits as integers of the same order: 0 for -inf (never chosen), NaN above
// everything, -0 like 0.
__device__ __forceinline__ uint32_t ordered(float x)
{
    if (x != x)
        return 0xFFFFFFFFu;
    if (x == -INFINITY)
        return 0u;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// (NaN where a lane has one)
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float u = __shfl_xor_sync(kAll, v, d);
        v = v != v || v > u ? v : u;
    }
    return v;
}

template <typename T, int PER>
__device__ __forceinline__ void load_logits(const void *logits, int64_t at, int experts, int lane, float (&l)[PER])
{
    const T *const p = static_cast<const T *>(logits) + at;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        l[i] = lane + 32 * i < experts ? to_f32(p[lane + 32 * i]) : -INFINITY;
}

template <typename T, int PER>
__global__ void __launch_bounds__(kWarps * 32) route_kernel(const RouteArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    wait_for_previous();
    let_next_start();
    if (t >= a.tokens)
        return;
    float l[PER];
    load_logits<T, PER>(a.logits, t * a.row, a.experts, lane, l);
    uint32_t key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i)
        key[i] = ordered(l[i]);
    float m = l[0];
#pragma unroll
    for (int i = 1; i < PER; ++i)
        m = m != m || m > l[i] ? m : l[i];
    m = warp_max(m);
    const bool none = m == -INFINITY;
    float z = 0.f;
    if (!a.normalize) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            z += l[i] == -INFINITY ? 0.f : expf(l[i] - m);
        z = lane_sum(z);
    }
    int id = -1;
    float w = 0.f;                           // lane j: the j-th choice
    for (int j = 0; j < a.top_k; ++j) {
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            best = max(best, key[i]);
        best = __reduce_max_sync(kAll, best);
        if (best == 0)
            break;
        int at = INT32_MAX;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
            if (key[i] == best)
                at = lane + 32 * i;
        at = __reduce_min_sync(kAll, at);
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (at == lane + 32 * i) {
                v = l[i];
                key[i] = 0;
            }
        v = __shfl_sync(kAll, v, at & 31);
        if (lane == j) {
            id = at;
            w = expf(v - m);
        }
    }
    if (a.normalize)
        z = lane_sum(w);
    if (lane < a.top_k) {
        a.ids[t * a.top_k + lane] = id;
        a.weights[t * a.top_k + lane] = none || id < 0 ? 0.f : w / z;
    }
}

template <typename T, int PER>
__global__ void __launch_bounds__(kWarps * 32) route_grad_kernel(const RouteGradArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    wait_for_previous();
    let_next_start();
    if (t >= a.tokens)
        return;
    float l[PER], d[PER];
    bool taken[PER];
    load_logits<T, PER>(a.logits, t * a.row, a.experts, lane, l);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        d[i] = 0.f;
        taken[i] = false;
    }
    const bool mine = lane < a.top_k;
    const int id = mine ? a.ids[t * a.top_k + lane] : -1;
    const float dw = mine ? a.dweights[t * a.top_k + lane] : 0.f;
    for (int j = 0; j < a.top_k; ++j) {
        const int e = __shfl_sync(kAll, id, j);
        const float v = __shfl_sync(kAll, dw, j);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (e == lane + 32 * i && e < a.experts) {
                d[i] += v;
                taken[i] = true;
            }
    }
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (a.normalize && !taken[i])
            l[i] = -INFINITY;
        m = m != m || m > l[i] ? m : l[i];
    }
    m = warp_max(m);
    float z = 0.f, s = 0.f, p[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        p[i] = l[i] == -INFINITY ? 0.f : expf(l[i] - m);
        z += p[i];
    }
    z = lane_sum(z);
    const float inv = z == 0.f ? 0.f : 1.f / z;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        p[i] *= inv;
        s += p[i] * d[i];
    }
    s = lane_sum(s);
    T *const out = static_cast<T *>(a.dlogits) + t * a.out_row;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (lane + 32 * i < a.experts)
            from_f32(out[lane + 32 * i], p[i] * (d[i] - s));
}

template <typename T, typename A>
cudaError_t launch(const A &a, cudaStream_t st)
{
    const dim3 grid((unsigned)((a.tokens + kWarps - 1) / kWarps));
    auto go = [&](auto fwd, auto bwd) {
        if constexpr (std::is_same_v<A, RouteArgs>)
            return launch_early(fwd, grid, kWarps * 32, 0, st, 1, a);
        else
            return launch_early(bwd, grid, kWarps * 32, 0, st, 1, a);
    };
    static_assert(kRouteExperts == 256, "eight logits a lane");
    if (a.experts <= 32)
        return go(route_kernel<T, 1>, route_grad_kernel<T, 1>);
    if (a.experts <= 64)
        return go(route_kernel<T, 2>, route_grad_kernel<T, 2>);
    if (a.experts <= 128)
        return go(route_kernel<T, 4>, route_grad_kernel<T, 4>);
    return go(route_kernel<T, 8>, route_grad_kernel<T, 8>);
}

} // namespace

cudaError_t launch_route(const RouteArgs &a, cudaStream_t st)
{
    return a.bf16 ? launch<__nv_bfloat16>(a, st) : launch<float>(a, st);
}

cudaError_t launch_route_grad(const RouteGradArgs &a, cudaStream_t st)
{
    return a.bf16 ? launch<__nv_bfloat16>(a, st) : launch<float>(a, st);
}

} // namespace rfq
