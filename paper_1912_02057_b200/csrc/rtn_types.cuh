// Element types of the layer operators (rtn_dtype) on the device: conversion to and from fp32, 16-byte vectors.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include "rtn.h"

namespace rtn {

inline int dtype_bytes(int dtype) { return dtype == RTN_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == RTN_F32 || dtype == RTN_BF16 || dtype == RTN_F16; }

#ifdef __CUDACC__

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Two values rounded to T, in one 32-bit word (x in the low half).
template <typename T> __device__ __forceinline__ uint32_t pack2(float x, float y);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float x, float y)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float x, float y)
{
    const __half2 v = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// The elements of T in 16 bytes, as fp32 and back.
template <typename T> struct Vec16 {
    static constexpr int N = 16 / (int)sizeof(T);
    static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[N])
    {
        const T* e = reinterpret_cast<const T*>(&u);
        #pragma unroll
        for (int i = 0; i < N; ++i) f[i] = to_f32(e[i]);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[N])
    {
        uint4 u;
        T* e = reinterpret_cast<T*>(&u);
        #pragma unroll
        for (int i = 0; i < N; ++i) e[i] = from_f32<T>(f[i]);
        return u;
    }
};

// Pairs of fp32 values in one 64-bit register: one instruction for both.
typedef unsigned long long pair_t;
__device__ __forceinline__ pair_t make_pair(float a, float b)
{
    pair_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void take_pair(pair_t p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ pair_t mul_pair(pair_t a, pair_t b)
{
    pair_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pair_t fma_pair(pair_t a, pair_t b, pair_t c)
{
    pair_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// The elements of T in 16 bytes as fp32 pairs and back.
template <typename T> struct Pairs16 {
    static constexpr int N = Vec16<T>::N / 2;
    static __device__ __forceinline__ void unpack(const uint4& u, pair_t (&f)[N])
    {
        float v[2 * N];
        Vec16<T>::unpack(u, v);
        #pragma unroll
        for (int i = 0; i < N; ++i) f[i] = make_pair(v[2 * i], v[2 * i + 1]);
    }
    static __device__ __forceinline__ uint4 pack(const pair_t (&f)[N])
    {
        float v[2 * N];
        #pragma unroll
        for (int i = 0; i < N; ++i) take_pair(f[i], v[2 * i], v[2 * i + 1]);
        if constexpr (sizeof(T) == 4)
            return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        else
            return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[2 * N - 4], v[2 * N - 3]), pack2<T>(v[2 * N - 2], v[2 * N - 1]));
    }
};

// Calls f(T{}) with the C++ type of `dtype`.
template <typename F>
inline cudaError_t with_dtype(int dtype, F&& f)
{
    if (dtype == RTN_BF16) return f(__nv_bfloat16{});
    if (dtype == RTN_F16) return f(__half{});
    return f(float{});
}

#endif  // __CUDACC__

}  // namespace rtn
