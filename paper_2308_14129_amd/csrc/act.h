// Activations of the dense layer and their slopes, in fp32.
#pragma once

#include <type_traits>

#include "kernels_common.h"

namespace tig {

// The normal distribution's upper tail at |z|, times two, over exp(-z^2 / 2): erfc(x) exp(x^2) at x = |z| / sqrt 2 by formula 7.1.26
// of Abramowitz and Stegun's handbook (a polynomial of degree five in 1 / (1 + 0.3275911 x), 1.5e-7 off at most; the library's
// erff takes about three times as many instructions, both of its branches for nearly every wavefront).
__device__ inline float tail_over_density(float z)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
    return t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
}

template <int ACT>
__device__ inline float activate(float z)
{
    if constexpr (ACT == TIG_ACT_RELU) {
        return z < 0.0f ? 0.0f : z;  // (a NaN stays one)
    } else if constexpr (ACT == TIG_ACT_GELU) {
        const float q = 0.5f * tail_over_density(z) * __builtin_amdgcn_exp2f(z * z * -0.72134752f);  // the tail beyond |z|
        const float zq = q > 0.0f ? z * q : q;  // (a tail of zero: also at infinity; a NaN stays one)
        return z > 0.0f ? z - zq : zq;
    } else if constexpr (ACT == TIG_ACT_SILU) {
        return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
    } else {
        return z;
    }
}

template <int ACT>
__device__ inline float slope(float z)
{
    if constexpr (ACT == TIG_ACT_RELU) {
        return z > 0.0f ? 1.0f : 0.0f;
    } else if constexpr (ACT == TIG_ACT_GELU) {
        const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752f), q = 0.5f * tail_over_density(z) * e;
        return fmaf(e > 0.0f ? z * e : e, 0.39894228f, z > 0.0f ? 1.0f - q : q);
    } else if constexpr (ACT == TIG_ACT_SILU) {
        const float g = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        return g * (1.0f + z * (1.0f - g));
    } else {
        return 1.0f;
    }
}

// f(std::integral_constant) for the selector's value; selectors are checked on the host before
template <class F>
inline auto with_activation(int act, F &&f)
{
    switch (act) {
    case TIG_ACT_RELU: return f(std::integral_constant<int, TIG_ACT_RELU>());
    case TIG_ACT_GELU: return f(std::integral_constant<int, TIG_ACT_GELU>());
    case TIG_ACT_SILU: return f(std::integral_constant<int, TIG_ACT_SILU>());
    default: return f(std::integral_constant<int, TIG_ACT_NONE>());
    }
}
template <class F>
inline auto with_dtype(int dtype, F &&f)
{
    switch (dtype) {
    case TIG_BF16: return f(__bf16());
    case TIG_F16: return f(_Float16());
    default: return f(float());
    }
}
inline int dtype_bytes(int dtype) { return dtype == TIG_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == TIG_F32 || dtype == TIG_BF16 || dtype == TIG_F16; }

}  // namespace tig
