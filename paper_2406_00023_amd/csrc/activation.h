// The activations of the experts' products and what their derivatives are made of.
#pragma once

#include "etr_internal.h"

namespace etr {
namespace {

// Activations by the hardware's exponential of 2 and reciprocal, an ulp each.  What costs more is the exponent, whose rounding the exponential
// magnifies (at |a| = 80 to 63 half steps of fp32, 208 in the distribution function at 12).  Results that are rounded to bf16 do not
// show it; for fp32 the exponent keeps its lower part l, as 2^(t + l) = 2^t (1 + l ln 2): 4 and 9 half steps.  (The bounds keep an infinite
// exponent's lower part from being no number; exponentials are 0 or infinite there already.)
__device__ __forceinline__ float exp_f32(float v) {                   // e^v
    v = fminf(fmaxf(v, -150.f), 150.f);
    const float t = v * 1.44269504f, l = fmaf(v, 1.44269504f, -t) + v * 1.92596303e-8f;
    return __builtin_amdgcn_exp2f(t) * fmaf(l, 0.693147181f, 1.0f);
}
__device__ __forceinline__ float gaussian_f32(float a) {              // e^(-a^2 / 2)
    a = fminf(fabsf(a), 20.f);
    const float q = a * a, t = q * 0.721347520f, l = fmaf(q, 0.721347520f, -t) + fmaf(fmaf(a, a, -q), 0.721347520f, q * 9.62981517e-9f);
    return __builtin_amdgcn_exp2f(-t) * fmaf(l, -0.693147181f, 1.0f);
}
template <bool BF16>
__device__ __forceinline__ float sigmoid(float a) { return __builtin_amdgcn_rcpf(1.0f + (BF16 ? __expf(-a) : exp_f32(-a))); }
// The normal distribution function: Phi(-|a|) = u Q(u) exp(-a^2 / 2), u = 1 / (1 + 0.297 |a|) (1 + 0.42 x for x = |a| / sqrt 2), Q of degree 7
// fitted to the least relative error over |a| <= 13.4 (1.7e-7; with fp32's roundings 5.4e-7).  12825 rows, 192 x 7744 in bf16: 108 us; with a
// fit of erfc's logarithm of degree 9 (1.2e-7) 120.  No branch, where erff has two and keeps every value of a tile alive across them (789
// spilled registers).
template <bool BF16>
__device__ __forceinline__ float normal_cdf(float a) {
    const float u = __builtin_amdgcn_rcpf(fmaf(0.29698485f, fabsf(a), 1.0f)), x = a * 0.84932180f;         // x^2 = a^2 / 2 log2 e
    float s = fmaf(0.0351077948f, u, -0.160095614f);
    s = fmaf(s, u, 0.220279561f); s = fmaf(s, u, -0.0652102044f); s = fmaf(s, u, 0.134342835f);
    s = fmaf(s, u, 0.0973718593f); s = fmaf(s, u, 0.119791471f); s = fmaf(s, u, 0.118412214f);
    const float tail = s * (u * (BF16 ? __builtin_amdgcn_exp2f(-x * x) : gaussian_f32(a)));
    return a < 0.f ? tail : 1.0f - tail;
}

}  // namespace
}  // namespace etr
