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

// t / n for 0 <= t < all, in 32 bits where they hold all (64-bit division is
// long).
__device__ __forceinline__ int64_t quotient(int64_t t, int64_t n, int64_t all)
{
    return all >> 31 ? t / n : (int64_t)((uint32_t)t / (uint32_t)n);
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

// cos(z) and sin(z): z less the nearest multiple of pi (in 64 bits: the
// angle of a 32-bit z is then good to 1e-8 up to |z| = 1e8), by the series
// to r^14 and r^13 (below 1e-9 at r = pi/2), with the sign of the multiple.
__device__ __forceinline__ float turn(float z, bool& odd)
{
    const double k = rint((double)z * 0.31830988618379067154);
    odd = k != 2.0 * rint(0.5 * k);
    return (float)fma(-k, 3.14159265358979323846, (double)z);
}

__device__ __forceinline__ float cos_of(float z)
{
    bool odd;
    const float r = turn(z, odd), q = r * r;
    float c = fmaf(q, -1.1470746e-11f, 2.0876757e-9f);
    c = fmaf(q, c, -2.7557319e-7f);
    c = fmaf(q, c, 2.4801587e-5f);
    c = fmaf(q, c, -1.3888889e-3f);
    c = fmaf(q, c, 4.1666667e-2f);
    c = fmaf(q, c, -0.5f);
    c = fmaf(q, c, 1.0f);
    return odd ? -c : c;
}

__device__ __forceinline__ float sin_of(float z)
{
    bool odd;
    const float r = turn(z, odd), q = r * r;
    float c = fmaf(q, 1.6059044e-10f, -2.5052108e-8f);
    c = fmaf(q, c, 2.7557319e-6f);
    c = fmaf(q, c, -1.9841270e-4f);
    c = fmaf(q, c, 8.3333333e-3f);
    c = fmaf(q, c, -1.6666667e-1f);
    c = fmaf(r * q, c, r);
    return odd ? -c : c;
}

// Eight consecutive values of a row: 16 or 32 bytes at once where all are
// there, else the first `count` one by one.  Rows may begin at any multiple
// of their type's size (loads and stores of 16 bytes need no alignment here).
template <int DT>
struct Eight {
    using T = Elem<DT>;
    typedef T Wide __attribute__((ext_vector_type(DT == SVM_F32 ? 4 : 8)));
    typedef Wide Loose __attribute__((aligned(sizeof(T))));
    float v[8];

    __device__ __forceinline__ void load(const void* p, int64_t at, int count)
    {
        const T* q = (const T*)p + at;
        if (count == 8) {
            if constexpr (DT == SVM_F32) {
                const Wide a = *(const Loose*)q, b = *(const Loose*)(q + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
            } else {
                const Wide a = *(const Loose*)q;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = e < count ? (float)q[e] : 0.0f;
        }
    }

    __device__ __forceinline__ void store(void* p, int64_t at, int count) const
    {
        T* q = (T*)p + at;
        if (count == 8) {
            if constexpr (DT == SVM_F32) {
                Wide a, b;
#pragma unroll
                for (int e = 0; e < 4; ++e) a[e] = v[e], b[e] = v[4 + e];
                *(Loose*)q = a;
                *(Loose*)(q + 4) = b;
            } else {
                Wide a;
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] = (T)v[e];
                *(Loose*)q = a;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) q[e] = (T)v[e];
        }
    }
};

// The same as they lie in memory: loaded ahead of their use in a fraction of
// the registers.
template <int DT>
struct RawEight {
    using T = Elem<DT>;
    using E = Eight<DT>;
    static constexpr int kN = DT == SVM_F32 ? 2 : 1;
    typename E::Wide v[kN];

    __device__ __forceinline__ void load(const void* p, int64_t at, int count)
    {
        constexpr int kEach = 8 / kN;
        const T* q = (const T*)p + at;
        if (count == 8) {
#pragma unroll
            for (int k = 0; k < kN; ++k)
                v[k] = *(const typename E::Loose*)(q + k * kEach);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e / kEach][e % kEach] = e < count ? q[e] : (T)0.0f;
        }
    }

    __device__ __forceinline__ void ones()
    {
#pragma unroll
        for (int k = 0; k < kN; ++k) v[k] = (T)1.0f;
    }

    __device__ __forceinline__ float at(int e) const
    {
        constexpr int kEach = 8 / kN;
        return (float)v[e / kEach][e % kEach];
    }
};

// Of n values, how many of the eight from j on there are.
__device__ __forceinline__ int eight_of(int64_t n, int64_t j)
{
    return n - j >= 8 ? 8 : n - j > 0 ? (int)(n - j) : 0;
}

// The three bf16 parts of eight 32-bit values: x = h + m + l, each part what
// is left rounded to nearest.  Where x is not finite, or rounds to a bf16
// that is not, h is that and the others are 0.  From |x| = 2^-109 on they hold
// all 24 bits; below, l falls under bf16's smallest step, and the sum is off
// by up to half of it, 2^-134.
typedef __bf16 Bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void three_parts(const float (&v)[8],
                                            Bf16x8 (&part)[3])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        part[0][e] = (__bf16)v[e];
        const float h = (float)part[0][e];
        const float r = fabsf(h) <= 3.402823466e38f ? v[e] - h : 0.0f;
        part[1][e] = (__bf16)r;
        part[2][e] = (__bf16)(r - (float)part[1][e]);
    }
}

// The normal distribution's upper tail at |z| and exp(-z^2 / 2): the rational
// approximation 7.1.26 of Abramowitz and Stegun's handbook (to 7.5e-8).
__device__ __forceinline__ float upper_tail(float z, float& e)
{
    const float a = fabsf(z);
    e = __expf(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.23164189f, a, 1.0f));
    float q = fmaf(t, 0.530702714f, -0.726576014f);
    q = fmaf(t, q, 0.710706870f);
    q = fmaf(t, q, -0.142248368f);
    q = fmaf(t, q, 0.127414796f);
    return t * q * e;
}

// tanh by exp, and by its series near 0 (to 1e-8 below 0.2)
__device__ __forceinline__ float tanh_of(float z)
{
    const float e = __expf(-2.0f * fabsf(z));
    const float y = copysignf(
        (1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e), z);
    const float q = z * z;
    float c = fmaf(q, 2.1869489e-2f, -5.3968254e-2f);
    c = fmaf(q, c, 1.3333333e-1f);
    c = fmaf(q, c, -3.3333333e-1f);
    return fabsf(z) < 0.2f ? fmaf(z * q, c, z) : y;
}

__device__ __forceinline__ float sigmoid_of(float z)
{
    return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
}

// act(z)
__device__ __forceinline__ float act_value(int act, float z)
{
    switch (act) {
    case SVM_ACT_RELU: return z > 0.0f ? z : (z != z ? z : 0.0f);
    case SVM_ACT_GELU: {
        float e;
        const float q = upper_tail(z, e);
        return z * (z > 0.0f ? 1.0f - q : q);
    }
    case SVM_ACT_SILU: return z * sigmoid_of(z);
    case SVM_ACT_TANH: return tanh_of(z);
    case SVM_ACT_COS: return cos_of(z);
    default: return z;
    }
}

// act'(z)
__device__ __forceinline__ float act_slope(int act, float z)
{
    switch (act) {
    case SVM_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case SVM_ACT_GELU: {
        float e;
        const float q = upper_tail(z, e);
        return fmaf(z * 0.39894228f, e, z > 0.0f ? 1.0f - q : q);
    }
    case SVM_ACT_SILU: {
        const float s = sigmoid_of(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    case SVM_ACT_TANH: {
        const float y = tanh_of(z);
        return fmaf(-y, y, 1.0f);
    }
    case SVM_ACT_COS: return -sin_of(z);
    default: return 1.0f;
    }
}

// act and act' of eight values, the choice made once
#define MSVM_EACH(F, A)                                                      \
    case A:                                                                  \
        _Pragma("unroll") for (int e = 0; e < 8; ++e) v[e] = F(A, v[e]);     \
        break
#define MSVM_EIGHT(NAME, F)                                                  \
    __device__ __forceinline__ void NAME(int act, float (&v)[8])             \
    {                                                                        \
        switch (act) {                                                       \
            MSVM_EACH(F, SVM_ACT_RELU);                                      \
            MSVM_EACH(F, SVM_ACT_GELU);                                      \
            MSVM_EACH(F, SVM_ACT_SILU);                                      \
            MSVM_EACH(F, SVM_ACT_TANH);                                      \
            MSVM_EACH(F, SVM_ACT_COS);                                       \
        default: break;                                                      \
        }                                                                    \
    }
MSVM_EIGHT(act_values, act_value)
MSVM_EIGHT(act_slopes, act_slope)
#undef MSVM_EIGHT
#undef MSVM_EACH

}  // namespace msvm
