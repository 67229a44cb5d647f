// Activations of the dense layer and their slopes, in fp32.
#pragma once

#include <type_traits>

#include "kernels_common.h"

namespace tig {

template <int ACT>
__device__ inline float activate(float z)
{
    if constexpr (ACT == TIG_ACT_RELU)
        return z < 0.0f ? 0.0f : z;  // (a NaN stays one)
    else if constexpr (ACT == TIG_ACT_GELU)
        return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    else if constexpr (ACT == TIG_ACT_SILU)
        return z / (1.0f + expf(-z));
    else
        return z;
}

template <int ACT>
__device__ inline float slope(float z)
{
    if constexpr (ACT == TIG_ACT_RELU) {
        return z > 0.0f ? 1.0f : 0.0f;
    } else if constexpr (ACT == TIG_ACT_GELU) {
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    } else if constexpr (ACT == TIG_ACT_SILU) {
        const float g = 1.0f / (1.0f + expf(-z));
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
