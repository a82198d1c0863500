// Activation functions of the training operators (group_norm.hip, linear.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "dolphin_hip.h"

namespace dol {

// act(z), and act'(z) as *slope.
template <int ACT, bool SLOPE>
__device__ __forceinline__ float act_of(float z, float *slope)
{
    if constexpr (ACT == DOL_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896340736f));
        if (SLOPE) *slope = s * __builtin_fmaf(z, 1.0f - s, 1.0f);
        return z * s;
    } else if constexpr (ACT == DOL_ACT_GELU) {
        // Phi(-|z|) = exp(-z^2 / 2) t q(t), t = 1 / (1 + 0.3 |z| / sqrt 2): a polynomial fitted to erfcx(x) / t, off by 4e-8 of it at most
        // up to |z| = 19, where the exponential has vanished; the slope has the same exponential.  (The library's erff takes twice as long.)
        const float bell = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170368f);
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), 0.21213203435596425732f, 1.0f));
        float q = -0.063308546f;
        q = __builtin_fmaf(q, t, 0.23591424f);
        q = __builtin_fmaf(q, t, -0.242347969f);
        q = __builtin_fmaf(q, t, 0.258526498f);
        q = __builtin_fmaf(q, t, -0.0370258253f);
        q = __builtin_fmaf(q, t, 0.103193045f);
        q = __builtin_fmaf(q, t, 0.0752343293f);
        q = __builtin_fmaf(q, t, 0.0852118725f);
        q = __builtin_fmaf(q, t, 0.084602376f);
        const float tail = q * t * bell, cdf = z < 0.0f ? tail : 1.0f - tail;
        if (SLOPE) *slope = __builtin_fmaf(z * 0.39894228040143267794f, bell, cdf);
        return z * cdf;
    } else if constexpr (ACT == DOL_ACT_RELU) {
        if (SLOPE) *slope = z > 0.0f ? 1.0f : z == z ? 0.0f : z;
        return z > 0.0f ? z : z == z ? 0.0f : z;
    } else {
        if (SLOPE) *slope = 1.0f;
        return z;
    }
}

template <int A>
struct Act {
    static constexpr int value = A;
};

// f for the activation function that the call names, chosen once and not at every element.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f)
{
    if (act == DOL_ACT_SILU) f(Act<DOL_ACT_SILU>());
    else if (act == DOL_ACT_GELU) f(Act<DOL_ACT_GELU>());
    else if (act == DOL_ACT_RELU) f(Act<DOL_ACT_RELU>());
    else f(Act<DOL_ACT_NONE>());
}

}  // namespace dol
