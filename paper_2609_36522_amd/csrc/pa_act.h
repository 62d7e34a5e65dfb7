// Activations on the device: value, and value with derivative.
#pragma once

#include <hip/hip_runtime.h>

#include "paraanya_ops.h"

namespace pa {

__device__ __forceinline__ float exp_f32(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// 2 Q(a), Q the normal upper tail, a >= 0, as 2^-P(a) with the polynomials that gelu_fit.py derives. For results of 16 bits
// (EXACT false) within 1e-5 of 1 near 0, so that gelu is off by 1.3e-7 max(1, |z|) and its derivative by 3.8e-6. For fp32
// P(0) = 0 and four terms more: both are off by a few units of rounding (3e-6 of the value itself at z = -5), where the shorter
// one's results were 8.8e-7 off in the mean.
template <bool EXACT>
__device__ __forceinline__ float upper_tail2(float a) {
    if constexpr (EXACT) {
        float p = fmaf(a, 1.4279759319446583e-10f, -7.2095813763439764e-09f);
        p = fmaf(p, a, 1.6186365314752038e-07f);
        p = fmaf(p, a, -2.128163259840221e-06f);
        p = fmaf(p, a, 1.8058883142657578e-05f);
        p = fmaf(p, a, -0.00010078817285830155f);
        p = fmaf(p, a, 0.00033124530455097556f);
        p = fmaf(p, a, -6.576548184966668e-05f);
        p = fmaf(p, a, -0.006899686064571142f);
        p = fmaf(p, a, 0.052424635738134384f);
        p = fmaf(p, a, 0.45922285318374634f);
        p = fmaf(p, a, 1.151104211807251f);
        return __builtin_amdgcn_exp2f(-p * a);
    }
    float p = fmaf(a, 1.1180667343069217e-06f, -4.9184127419721335e-05f);
    p = fmaf(p, a, 0.0008520559640601277f);
    p = fmaf(p, a, -0.008282574824988842f);
    p = fmaf(p, a, 0.05366271361708641f);
    p = fmaf(p, a, 0.45861566066741943f);
    p = fmaf(p, a, 1.1512444019317627f);
    p = fmaf(p, a, -1.0669231414794922e-05f);
    return __builtin_amdgcn_exp2f(-p);
}

// silu(z) = z / (1 + e^-z); gelu(z) = z Phi(z) = max(z, 0) - |z| Q(|z|).
template <int ACT, bool EXACT = false>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == PA_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + exp_f32(-z));
    if constexpr (ACT == PA_ACT_GELU) {
        const float a = fabsf(z);
        return 0.5f * fmaf(-fminf(a, 1e4f), upper_tail2<EXACT>(a), z + a);      // an infinite a times a tail of 0 is no number
    }
    return z;
}

// {value, derivative}: silu' = p + z p (1 - p), p = 1 / (1 + e^-z); gelu' = Phi(z) + z phi(z).
template <int ACT, bool EXACT = false>
__device__ __forceinline__ float2 activate_grad(float z) {
    if constexpr (ACT == PA_ACT_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.0f + exp_f32(-z)), v = z * p;
        return make_float2(v, fmaf(v, 1.0f - p, p));
    }
    if constexpr (ACT == PA_ACT_GELU) {
        const float a = fabsf(z), q2 = upper_tail2<EXACT>(a);
        const float phi = 0.3989422804014327f * __builtin_amdgcn_exp2f(-0.7213475204444817f * z * z);
        return make_float2(0.5f * fmaf(-fminf(a, 1e4f), q2, z + a), fmaf(z, phi, z < 0.0f ? 0.5f * q2 : 1.0f - 0.5f * q2));
    }
    return make_float2(z, 1.0f);
}

}  // namespace pa
