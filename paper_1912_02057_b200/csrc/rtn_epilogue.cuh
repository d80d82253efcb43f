// What rtn_ternary_linear does to a value after the affine form.
#pragma once
#include "rtn_internal.cuh"
#include "rtn_types.cuh"

namespace rtn {

#ifdef __CUDACC__

// The activations, other than none.  Called rather than inlined: at every unrolled output they were most of a kernel's instructions, and a
// short kernel's time is made of fetching them.  The four-value form keeps four chains in flight.
__device__ __forceinline__ float activation_of(float y, int act)
{
    if (act == RTN_ACT_RELU) return y < 0.f ? 0.f : y;                                     // a NaN stays one
    if (act == RTN_ACT_GELU) return 0.5f * y * (1.f + erff(y * 0.70710678118654752f));
    if (act == RTN_ACT_GELU_TANH) return 0.5f * y * (1.f + tanhf(0.79788456080286536f * fmaf(0.044715f * y * y, y, y)));
    return y / (1.f + expf(-y));
}
static __device__ __noinline__ float activation(float y, int act) { return activation_of(y, act); }
static __device__ __noinline__ float4 activation4(float4 y, int act)
{
    switch (act) {
        case RTN_ACT_RELU: return make_float4(activation_of(y.x, RTN_ACT_RELU), activation_of(y.y, RTN_ACT_RELU), activation_of(y.z, RTN_ACT_RELU), activation_of(y.w, RTN_ACT_RELU));
        case RTN_ACT_GELU: return make_float4(activation_of(y.x, RTN_ACT_GELU), activation_of(y.y, RTN_ACT_GELU), activation_of(y.z, RTN_ACT_GELU), activation_of(y.w, RTN_ACT_GELU));
        case RTN_ACT_GELU_TANH: return make_float4(activation_of(y.x, RTN_ACT_GELU_TANH), activation_of(y.y, RTN_ACT_GELU_TANH), activation_of(y.z, RTN_ACT_GELU_TANH), activation_of(y.w, RTN_ACT_GELU_TANH));
        default: return make_float4(activation_of(y.x, RTN_ACT_SILU), activation_of(y.y, RTN_ACT_SILU), activation_of(y.z, RTN_ACT_SILU), activation_of(y.w, RTN_ACT_SILU));
    }
}
__device__ __forceinline__ float activate(float y, int act) { return act == RTN_ACT_NONE ? y : activation(y, act); }

__device__ __forceinline__ float load_as_f32(const void* p, int64_t i, int dtype)
{
    if (dtype == RTN_F32) return static_cast<const float*>(p)[i];
    if (dtype == RTN_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(static_cast<const __half*>(p)[i]);
}

__device__ __forceinline__ void store_from_f32(void* p, int64_t i, int dtype, float y)
{
    if (dtype == RTN_F32) static_cast<float*>(p)[i] = y;
    else if (dtype == RTN_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(y);
    else static_cast<__half*>(p)[i] = from_f32<__half>(y);
}

#endif

}  // namespace rtn
