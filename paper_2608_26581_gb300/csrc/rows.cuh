// rows.cuh -- what the kernels over rows of fp32 or bf16 elements share
// (norms, router, rows brought to experts and back): vectors of elements,
// conversions, sums over lanes.
#pragma once

#include <cuda_bf16.h>
#include <cstdint>

namespace rfq {

// VEC elements loaded or stored at once (16 bytes, or one element where
// strides, sizes or addresses allow no more).
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Vec {
    T v[VEC];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16 &d, float x) { d = __float2bfloat16_rn(x); }

template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load_vec(const T *p)
{
    return *reinterpret_cast<const Vec<T, VEC> *>(p);
}

template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T *p, const Vec<T, VEC> &v)
{
    *reinterpret_cast<Vec<T, VEC> *>(p) = v;
}

template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> zero_vec()
{
    Vec<T, VEC> v;
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        from_f32(v.v[e], 0.f);
    return v;
}

// Sum over each `n` lanes that lie together (n a power of two up to 32).
__device__ __forceinline__ float lane_sum(float v, int n = 32)
{
    for (int d = n >> 1; d > 0; d >>= 1)
        v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

} // namespace rfq
