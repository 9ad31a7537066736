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
// the lowest expert is taken.  Bound: latency where tokens are few (61 tokens of
// 128 experts, top 8: 1.8 us), else instructions: some 350 a token forward (32768
// tokens 12.6 us; without the experts in the keys, or a lane's logits in order,
// 19.6), backwards less (32768 tokens in fp32 8.4 us, 63% of the copy rate; with
// a persistent grid 8.6, with 4 warps a block 9.0).
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

// The logit of a key (some NaN for NaN): an ordered integer, of bf16 logits the
// upper half alone.
template <typename T>
__device__ __forceinline__ float logit_of(uint32_t k)
{
    const uint32_t b = k & 0x80000000u ? k ^ 0x80000000u : ~k;
    return __uint_as_float(std::is_same_v<T, float> ? b : b & 0xFFFF0000u);
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

// The warp's choices: best() is the key of the largest logit left (0 where none
// is), take(best) its expert, which is left out from then on.  A key of a bf16
// logit holds the expert as well, so one maximum over the warp finds both, and
// equal logits follow by their experts.
template <typename T, int PER>
struct Choices {
    uint32_t key[PER];
    __device__ __forceinline__ Choices(const float (&l)[PER], int lane)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t k = ordered(l[i]);
            key[i] = k ? (k & 0xFFFF0000u) | (0xFFFFu - (lane * PER + i)) : 0u;
        }
    }
    __device__ __forceinline__ uint32_t best() const
    {
        uint32_t k = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i)
            k = max(k, key[i]);
        return __reduce_max_sync(kAll, k);
    }
    __device__ __forceinline__ int take(uint32_t best)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            key[i] = key[i] == best ? 0u : key[i];
        return 0xFFFF - (best & 0xFFFFu);
    }
};

// fp32: a lane's keys in order (equal ones by expert), the first of them left is
// compared with the others'.
template <int PER>
struct Choices<float, PER> {
    uint32_t key[PER], order = 0;            // order: the experts' places in the lane, 4 bits each
    int from;
    __device__ __forceinline__ Choices(const float (&l)[PER], int lane) : from(lane * PER)
    {
        uint32_t at[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            key[i] = ordered(l[i]);
            at[i] = i;
        }
        // (neighbours alone change places: equal ones never pass each other)
#pragma unroll
        for (int pass = 0; pass < PER; ++pass)
#pragma unroll
            for (int i = pass & 1; i + 1 < PER; i += 2) {
                const bool swap = key[i + 1] > key[i];
                const uint32_t k = key[i], n = at[i];
                key[i] = max(k, key[i + 1]);
                key[i + 1] = min(k, key[i + 1]);
                at[i] = swap ? at[i + 1] : n;
                at[i + 1] = swap ? n : at[i + 1];
            }
#pragma unroll
        for (int i = 0; i < PER; ++i)
            order |= at[i] << 4 * i;
    }
    __device__ __forceinline__ uint32_t best() const { return __reduce_max_sync(kAll, key[0]); }
    __device__ __forceinline__ int take(uint32_t best)
    {
        const uint32_t first = from + (order & 15);
        const uint32_t chosen = __reduce_min_sync(kAll, key[0] == best ? first : 0xFFFFu);
        if (first == chosen) {
#pragma unroll
            for (int i = 0; i + 1 < PER; ++i)
                key[i] = key[i + 1];
            key[PER - 1] = 0;
            order >>= 4;
        }
        return (int)chosen;
    }
};

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
    Choices<T, PER> choices(l, lane);
    uint32_t best = choices.best();
    const float m = logit_of<T>(best);
    float z = 0.f;
    if (!a.normalize && best != 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            z += l[i] == -INFINITY ? 0.f : expf(l[i] - m);
        z = lane_sum(z);
    }
    int id = -1;
    uint32_t key = 0;                        // lane j: the j-th choice
    for (int j = 0; best != 0; best = choices.best()) {
        const int chosen = choices.take(best);
        id = lane == j ? chosen : id;
        key = lane == j ? best : key;
        if (++j == a.top_k)
            break;
    }
    const float w = id < 0 ? 0.f : expf(logit_of<T>(key) - m);
    if (a.normalize)
        z = lane_sum(w);
    if (lane < a.top_k) {
        a.ids[t * a.top_k + lane] = id;
        a.weights[t * a.top_k + lane] = id < 0 ? 0.f : w / z;
    }
}

// What an expert that was not chosen has in the place of its dweight (a NaN
// that no dweight is scattered as).
constexpr uint32_t kNone = 0xFFFFFFFFu;

template <typename T, int PER, bool VEC>
__global__ void __launch_bounds__(kWarps * 32) route_grad_kernel(const RouteGradArgs a)
{
    __shared__ __align__(16) uint32_t s_dw[kWarps][32 * PER];        // each expert's dweight
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    uint32_t *const of = s_dw[threadIdx.x >> 5];
    wait_for_previous();
    let_next_start();
    if (t >= a.tokens)
        return;
    const bool mine = lane < a.top_k;
    const int id = mine ? a.ids[t * a.top_k + lane] : -1;
    const uint32_t dw = mine ? __float_as_uint(a.dweights[t * a.top_k + lane]) : 0;
    float l[PER], d[PER];
    load_logits<T, PER, VEC>(a.logits, t * a.row, a.experts, lane, l);
    using All = Vec<uint32_t, PER>;
    All all;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        all.v[i] = kNone;
    store_vec<uint32_t, PER>(of + lane * PER, all);
    __syncwarp();
    if (id >= 0 && id < a.experts)
        of[id] = dw == kNone ? 0x7FFFFFFFu : dw;
    __syncwarp();
    all = load_vec<uint32_t, PER>(of + lane * PER);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool taken = all.v[i] != kNone;
        d[i] = taken ? __uint_as_float(all.v[i]) : 0.f;
        l[i] = a.normalize && !taken ? -INFINITY : l[i];
        m = fmaxf(m, l[i]);
    }
    m = warp_max(m);
    m = m == -INFINITY ? 0.f : m;            // (no logit at all: every exponential is 0)
    float z = 0.f, s = 0.f, p[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        p[i] = expf(l[i] - m);
        z += p[i];
        s += p[i] * d[i];
    }
    // both sums over the warp: half of it takes z, the other s
    float half = (lane < 16 ? z : s) + __shfl_xor_sync(kAll, lane < 16 ? s : z, 16);
    half = lane_sum(half, 16);
    z = __shfl_sync(kAll, half, 0);
    s = __shfl_sync(kAll, half, 16);
    const float inv = z == 0.f ? 0.f : 1.f / z;
    s *= inv;
    T *const out = static_cast<T *>(a.dlogits) + t * a.out_row + lane * PER;
    Vec<T, PER> o;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        from_f32(o.v[i], p[i] * inv * (d[i] - s));
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
