// Element types of the feature-map operators and the device helpers that the
// kernels on them share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.hpp"

namespace msvm {

template <int DT>
struct ElemOf {
    using type = float;
};
template <>
struct ElemOf<SVM_BF16> {
    using type = __bf16;
};
template <>
struct ElemOf<SVM_F16> {
    using type = _Float16;
};
template <int DT>
using Elem = typename ElemOf<DT>::type;

// Calls f.template operator()<DT>() for the type of a call.
template <class F>
void for_dtype(int32_t t, F&& f)
{
    if (t == SVM_F32)
        f.template operator()<SVM_F32>();
    else if (t == SVM_BF16)
        f.template operator()<SVM_BF16>();
    else
        f.template operator()<SVM_F16>();
}

// Sum over the 64 lanes; every lane ends with it.
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

// act(z)
__device__ __forceinline__ float act_value(int act, float z)
{
    switch (act) {
    case SVM_ACT_RELU: return z > 0.0f ? z : (z != z ? z : 0.0f);
    case SVM_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    case SVM_ACT_SILU: return z / (1.0f + __expf(-z));
    case SVM_ACT_TANH: return tanhf(z);
    case SVM_ACT_COS: return cosf(z);
    default: return z;
    }
}

// act'(z)
__device__ __forceinline__ float act_slope(int act, float z)
{
    switch (act) {
    case SVM_ACT_RELU: return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    case SVM_ACT_GELU:
        return fmaf(z * 0.39894228f, __expf(-0.5f * z * z),
                    0.5f * (1.0f + erff(z * 0.70710678f)));
    case SVM_ACT_SILU: {
        const float s = 1.0f / (1.0f + __expf(-z));
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    case SVM_ACT_TANH: {
        const float y = tanhf(z);
        return fmaf(-y, y, 1.0f);
    }
    case SVM_ACT_COS: return -sinf(z);
    default: return 1.0f;
    }
}

}  // namespace msvm
