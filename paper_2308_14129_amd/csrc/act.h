// Activations of the dense layer and their slopes, in fp32.
#pragma once

#include <numeric>
#include <type_traits>

#include "kernels_common.h"

namespace tig {

// The normal distribution's upper tail at |z| over exp(-z^2 / 2), that is erfc(x) exp(x^2) / 2 at x = |z| / sqrt 2: t Q(t) with
// t = 1 / (1 + 0.35 |z|) and Q of degree eight, fitted to the least relative error over 0 <= |z| <= 15 (6e-8 with these coefficients; with the operations'
// own roundings 5 units of 2^-24 by an emulation).  Relative, so that gelu's lower tail is right too, where it is this times z
// exp(-z^2 / 2).  (The library's erff takes about twice as many instructions, both of its branches for nearly every wavefront, and
// 1 + erf has no lower tail.)
__device__ inline float tail_over_density(float z)
{
    constexpr float c[9] = {0.13962126f, 0.13986433f, 0.11981556f, 0.10557454f, -0.023263184f, 0.15939192f, -0.25590098f, 0.14406036f, -0.029163832f};
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, fabsf(z), 1.0f));
    float q = c[8];
#pragma unroll
    for (int i = 7; i >= 0; --i)
        q = fmaf(t, q, c[i]);
    return t * q;
}

template <int ACT>
__device__ inline float activate(float z)
{
    if constexpr (ACT == TIG_ACT_RELU) {
        return z < 0.0f ? 0.0f : z;  // (a NaN stays one)
    } else if constexpr (ACT == TIG_ACT_GELU) {
        const float q = tail_over_density(z) * __builtin_amdgcn_exp2f(z * z * -0.72134752f);  // the tail beyond |z|
        const float zq = q > 0.0f ? z * q : q;  // (a tail of zero: also at infinity; a NaN stays one)
        return z > 0.0f ? z - zq : zq;
    } else if constexpr (ACT == TIG_ACT_SILU) {
        const float g = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        return g > 0.0f ? z * g : g;  // (zero at -infinity too; a NaN stays one)
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
        const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752f), q = tail_over_density(z) * e;
        return fmaf(e > 0.0f ? z * e : e, 0.39894228f, z > 0.0f ? 1.0f - q : q);
    } else if constexpr (ACT == TIG_ACT_SILU) {
        const float g = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        const float h = 1.0f - g, zh = h > 0.0f ? z * h : h;  // (one at infinity, zero at -infinity; a NaN stays one)
        return g > 0.0f ? g * (1.0f + zh) : g;
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
// A matrix of a call (p NULL: none), strides in elements.
struct Placed {
    const void *p;
    int64_t rows, cols, ld;
    int elem;
};
// No element of one is an element of the other: their ranges do not meet, or their columns do not (two column ranges, or every other
// row, of one buffer): then their rows keep apart within what both strides are multiples of.
inline bool apart(const Placed &a, const Placed &b)
{
    if (!a.p || !b.p || a.rows == 0 || b.rows == 0)
        return true;
    const int64_t wa = a.cols * a.elem, wb = b.cols * b.elem, sa = a.rows > 1 ? a.ld * a.elem : 0, sb = b.rows > 1 ? b.ld * b.elem : 0;
    const uintptr_t la = (uintptr_t)a.p, lb = (uintptr_t)b.p;
    if (la + (uintptr_t)((a.rows - 1) * sa + wa) <= lb || lb + (uintptr_t)((b.rows - 1) * sb + wb) <= la)
        return true;
    const int64_t g = std::gcd(sa, sb);
    if (g == 0)
        return false;
    const int64_t d = (((int64_t)(lb - la)) % g + g) % g;
    return d >= wa && d + wb <= g;
}
// ... of each of `out` and everything in `in` and the rest of `out`
template <int I, int O>
inline bool all_apart(const Placed (&in)[I], const Placed (&out)[O])
{
    for (int o = 0; o < O; ++o) {
        for (int i = 0; i < I; ++i)
            if (!apart(out[o], in[i]))
                return false;
        for (int k = 0; k < o; ++k)
            if (!apart(out[o], out[k]))
                return false;
    }
    return true;
}
inline bool dtype_ok(int dtype) { return dtype == TIG_F32 || dtype == TIG_BF16 || dtype == TIG_F16; }

}  // namespace tig
