// route.cu -- the router of a mixture of experts: each token's top_k experts
// and their weights from the experts' logits (rfq_route), and the logits'
// gradient (rfq_route_grad).
//
// With p = softmax(l) over a token's logits and e_j its j-th largest,
//     w_j = p[e_j],  or with normalize  w_j = p[e_j] / sum_m p[e_m],
// which is the softmax over the chosen logits alone.  Gradient, with d_i = dw_j
// where e_j = i (0 elsewhere) and p restricted to the chosen experts with
// normalize:
//     dl_i = p_i (d_i - sum_m p_m d_m).
//
// A warp takes a token; a lane holds consecutive experts' logits.  A choice is
// the maximum over the warp of the logits as ordered integers; of equal ones
// the lowest lane's lowest is taken.  Bound: instructions of some 200 a token
// (32768 tokens of 128 experts in fp32, gradient: 9.6 us, 55% of the copy rate,
// issue slots 68% busy), latency where tokens are few (61 tokens, top 8: 2.4 us).
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

// The logit of an ordered integer (some NaN for NaN).
__device__ __forceinline__ float logit_of(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Maximum over the warp; NaN counts as nothing (its exponential is NaN all the same).
__device__ __forceinline__ float warp_max(float v)
{
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}

// Lane's logits: experts PER lane .. PER lane + PER - 1, as one vector where VEC.
template <typename T, int PER, bool VEC>
__device__ __forceinline__ void load_logits(const void *logits, int64_t at, int experts, int lane, float (&l)[PER])
{
    const T *const p = static_cast<const T *>(logits) + at + lane * PER;
    if (VEC) {
        if (lane * PER < experts) {
            const Vec<T, PER> v = load_vec<T, PER>(p);
#pragma unroll
            for (int i = 0; i < PER; ++i)
                l[i] = to_f32(v.v[i]);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
        l[i] = !VEC && lane * PER + i < experts ? to_f32(p[i]) : -INFINITY;
}

template <typename T, int PER, bool VEC>
__global__ void __launch_bounds__(kWarps * 32) route_kernel(const RouteArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    wait_for_previous();
    let_next_start();
    if (t >= a.tokens)
        return;
    float l[PER];
    load_logits<T, PER, VEC>(a.logits, t * a.row, a.experts, lane, l);
    uint32_t key[PER], best = 0;
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        key[i] = ordered(l[i]);
        best = max(best, key[i]);
    }
    best = __reduce_max_sync(kAll, best);
    const float m = logit_of(best);
    if (!a.normalize && best != 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            z += l[i] == -INFINITY ? 0.f : expf(l[i] - m);
        z = lane_sum(z);
    }
    int id = -1;
    float w = 0.f;                           // lane j: the j-th choice
    for (int j = 0; j < a.top_k && best != 0; ++j) {
        int at = PER;                        // this lane's lowest expert with that logit
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
            at = key[i] == best ? i : at;
        const int from = __ffs(__ballot_sync(kAll, at < PER)) - 1;
        const int chosen = __shfl_sync(kAll, lane * PER + at, from);
        if (lane == j) {
            id = chosen;
            w = expf(logit_of(best) - m);
        }
        best = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            key[i] = chosen == lane * PER + i ? 0u : key[i];
            best = max(best, key[i]);
        }
        best = __reduce_max_sync(kAll, best);
    }
    if (a.normalize)
        z = lane_sum(w);
    if (lane < a.top_k) {
        a.ids[t * a.top_k + lane] = id;
        a.weights[t * a.top_k + lane] = id < 0 ? 0.f : w / z;
    }
}

template <typename T, int PER, bool VEC>
__global__ void __launch_bounds__(kWarps * 32) route_grad_kernel(const RouteGradArgs a)
{
    __shared__ __align__(16) int8_t s_choice[kWarps][32 * PER];      // which choice took an expert, -1 where none
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    int8_t *const choice = s_choice[threadIdx.x >> 5];
    wait_for_previous();
    let_next_start();
    if (t >= a.tokens)
        return;
    const bool mine = lane < a.top_k;
    const int id = mine ? a.ids[t * a.top_k + lane] : -1;
    const float dw = mine ? a.dweights[t * a.top_k + lane] : 0.f;
    float l[PER], d[PER];
    load_logits<T, PER, VEC>(a.logits, t * a.row, a.experts, lane, l);
    using Choices = Vec<int8_t, PER>;
    Choices none;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        none.v[i] = -1;
    store_vec<int8_t, PER>(choice + lane * PER, none);
    __syncwarp();
    if (id >= 0 && id < a.experts)
        choice[id] = (int8_t)lane;
    __syncwarp();
    const Choices taken = load_vec<int8_t, PER>(choice + lane * PER);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float v = __shfl_sync(kAll, dw, taken.v[i] & 31);
        d[i] = taken.v[i] >= 0 ? v : 0.f;
        l[i] = a.normalize && taken.v[i] < 0 ? -INFINITY : l[i];
        m = fmaxf(m, l[i]);
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
    T *const out = static_cast<T *>(a.dlogits) + t * a.out_row + lane * PER;
    Vec<T, PER> o;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        from_f32(o.v[i], p[i] * (d[i] - s));
    if (VEC) {
        if (lane * PER < a.experts)
            store_vec<T, PER>(out, o);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane * PER + i < a.experts)
                out[i] = o.v[i];
    }
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
    // vectors of a lane's logits where the rows' strides and length allow
    int64_t strides = a.row | a.experts;
    if constexpr (std::is_same_v<A, RouteGradArgs>)
        strides |= a.out_row;
    static_assert(kRouteExperts == 256, "eight logits a lane");
    if (a.experts <= 32)
        return go(route_kernel<T, 1, false>, route_grad_kernel<T, 1, false>);
    if (a.experts <= 64)
        return strides % 2 == 0 ? go(route_kernel<T, 2, true>, route_grad_kernel<T, 2, true>)
                                : go(route_kernel<T, 2, false>, route_grad_kernel<T, 2, false>);
    if (a.experts <= 128)
        return strides % 4 == 0 ? go(route_kernel<T, 4, true>, route_grad_kernel<T, 4, true>)
                                : go(route_kernel<T, 4, false>, route_grad_kernel<T, 4, false>);
    return strides % 8 == 0 ? go(route_kernel<T, 8, true>, route_grad_kernel<T, 8, true>)
                            : go(route_kernel<T, 8, false>, route_grad_kernel<T, 8, false>);
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
