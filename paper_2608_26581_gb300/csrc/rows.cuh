// rows.cuh -- what the kernels over rows of fp32 or bf16 elements share
// (norms, router, rows brought to experts and back): vectors of elements,
// conversions, sums over lanes.
#pragma once

#include <cuda_bf16.h>
#include <cstdint>
#include <type_traits>

#include "mxfp4_math.cuh"

namespace rfq {

// VEC elements loaded or stored at once (16 bytes, or one element where
// strides, sizes or addresses allow no more).
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC < 16 ? sizeof(T) * VEC : 16) Vec {
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

// Loads and stores that leave L1 to what is read again.
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load_once(const T *p)
{
    if constexpr (sizeof(T) * VEC == 16) {
        uint4 u;
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
        return *reinterpret_cast<Vec<T, VEC> *>(&u);
    } else
        return load_vec<T, VEC>(p);
}

template <typename T, int VEC>
__device__ __forceinline__ void store_once(T *p, const Vec<T, VEC> &v)
{
    if constexpr (sizeof(v) == 16) {
        const uint4 u = *reinterpret_cast<const uint4 *>(&v);
        asm volatile("st.global.L1::no_allocate.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
    } else
        store_vec<T, VEC>(p, v);
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

// Two fp32 values in one register pair, each operation one instruction.
struct F2 {
    uint64_t v;
};
__device__ __forceinline__ F2 operator+(F2 a, F2 b)
{
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) { return {fmul2(a.v, b.v)}; }
__device__ __forceinline__ F2 fused(F2 a, F2 b, F2 c) { return {ffma2(a.v, b.v, c.v)}; }
__device__ __forceinline__ float fused(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float both(float a) { return a; }
__device__ __forceinline__ float both(F2 a)
{
    float x, y;
    f2unpack(a.v, x, y);
    return x + y;
}

// The values of a vector of VEC elements in fp32: pairs where VEC is even,
// single ones for VEC = 1.
template <int VEC>
using Lane = std::conditional_t<VEC == 1, float, F2>;
template <int VEC>
constexpr int kLanes = VEC == 1 ? 1 : VEC / 2;

template <int VEC>
__device__ __forceinline__ Lane<VEC> all_of(float v)
{
    if constexpr (VEC == 1)
        return v;
    else
        return {f2pack(v, v)};
}

template <typename T, int VEC>
__device__ __forceinline__ void unpack(const Vec<T, VEC> &v, Lane<VEC> *x)
{
    if constexpr (VEC == 1)
        x[0] = to_f32(v.v[0]);
    else if constexpr (std::is_same_v<T, float>) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i)
            x[i] = {f2pack(v.v[2 * i], v.v[2 * i + 1])};
    } else {
        const uint32_t *const w = reinterpret_cast<const uint32_t *>(&v);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i)
            x[i] = {f2pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u))};
    }
}

template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> pack(const Lane<VEC> *x)
{
    Vec<T, VEC> v;
    if constexpr (VEC == 1)
        from_f32(v.v[0], x[0]);
    else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            float a, b;
            f2unpack(x[i].v, a, b);
            if constexpr (std::is_same_v<T, float>) {
                v.v[2 * i] = a;
                v.v[2 * i + 1] = b;
            } else
                reinterpret_cast<__nv_bfloat162 *>(&v)[i] = __floats2bfloat162_rn(a, b);
        }
    }
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
