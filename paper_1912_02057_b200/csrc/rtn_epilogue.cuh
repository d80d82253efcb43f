// What rtn_ternary_linear does to a value after the affine form.
#pragma once
#include "rtn_internal.cuh"
#include "rtn_types.cuh"

namespace rtn {

#ifdef __CUDACC__

// One copy of the code, called: inlined at every unrolled output it was most of a kernel's instructions, and a short kernel's time is
// made of fetching them.
static __device__ __noinline__ float activation(float y, int act)
{
    switch (act) {
        case RTN_ACT_RELU: return y < 0.f ? 0.f : y;                                     // a NaN stays one
        case RTN_ACT_GELU: return 0.5f * y * (1.f + erff(y * 0.70710678118654752f));
        case RTN_ACT_GELU_TANH: return 0.5f * y * (1.f + tanhf(0.79788456080286536f * fmaf(0.044715f * y * y, y, y)));
        default: return y / (1.f + expf(-y));
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
