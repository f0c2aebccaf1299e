// The normal distribution of the gated-GELU experts and of switch_linear's activations.
#pragma once
#include "common.h"

namespace sw {

// The experts' (normal_of): Phi(u) and the density phi(u) of the standard normal distribution, sharing one exponential.
// erfc(z), z = |u| / sqrt 2 >= 0, comes from the rational approximation 7.1.26 of Abramowitz &
// Stegun, erfc(z) = (a1 t + ... + a5 t^5) exp(-z^2), t = 1 / (1 + p z), |error| <= 1.5e-7: a
// dozen instructions instead of the library erfc's sixty (the kernels that use it would be
// bound by their arithmetic otherwise, not by HBM).  The error of GELU(u) = u Phi(u) is
// |u| * 7.5e-8, two orders below the fp32 tolerance of the layer.
struct NormalOf {
    float cdf, pdf;
};
__device__ __forceinline__ NormalOf normal_of(float u) {
    const float z = fabsf(u) * 0.70710678f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.0f));   // 1 ulp: far inside the error of the fit
    const float e = __expf(-z * z);
    float poly = fmaf(1.061405429f, t, -1.453152027f);
    poly = fmaf(poly, t, 1.421413741f);
    poly = fmaf(poly, t, -0.284496736f);
    poly = fmaf(poly, t, 0.254829592f);
    const float half_erfc = 0.5f * poly * t * e;
    NormalOf r;
    r.cdf = u >= 0.f ? 1.0f - half_erfc : half_erfc;
    r.pdf = 0.3989422804f * e;
    return r;
}

// switch_linear's (normal_at<T>, T the storage type): the same with small relative errors, so that the tail of GELU, times
// a linear part of any size, is as good as the rest (the fit above is off by 5e-5 of Phi at u = -3 and 4e-3 at -6).
// Phi(-|u|) = t poly(t) exp(-u^2 / 2), t = 1 / (1 + q |u|): t poly(t) was fitted to erfcx(|u| / sqrt 2) / 2 on 0 .. 13.4, where
// Phi leaves the normal numbers, by least squares with weights raised where the relative error was largest; with its
// rounded coefficients it is off by 5.4e-8.  fp32: a refined quotient and u^2 in two terms, u Phi(u) measured to
// be off by up to 6.1 half steps; bf16: the quotient within 1 ulp and the exponent's rounding, 8e-6 at u = -12, far inside the
// store's.
template <typename T> __device__ __forceinline__ NormalOf normal_at(float u) {
    constexpr float q = 0.339411259f, half_log2e = -0.72134752f;
    const float v = sizeof(T) == 4 ? fminf(fabsf(u), 16.f) : fabsf(u);   // (from 13.4 on all is 0 or 1)
    const float d = fmaf(q, v, 1.0f), x = v * v * half_log2e;
    float t = __builtin_amdgcn_rcpf(d), e = __builtin_amdgcn_exp2f(x);
    if (sizeof(T) == 4) {
        t = fmaf(t, fmaf(-d, t, 1.0f), t);
        const float square = v * v, square_rest = fmaf(v, v, -square);
        float rest = fmaf(square, half_log2e, -x);
        rest = fmaf(square, -9.6298e-9f, rest);   // (-1 / (2 ln 2) less half_log2e)
        rest = fmaf(square_rest, half_log2e, rest);
        e = fmaf(e * rest, 0.693147181f, e);
    }
    float poly = fmaf(-0.0261368435f, t, 0.140120924f);
    poly = fmaf(poly, t, -0.275948048f);
    poly = fmaf(poly, t, 0.206848294f);
    poly = fmaf(poly, t, -0.0475171581f);
    poly = fmaf(poly, t, 0.116574563f);
    poly = fmaf(poly, t, 0.114761427f);
    poly = fmaf(poly, t, 0.135913119f);
    poly = fmaf(poly, t, 0.13538374f);
    const float tail = poly * t * e;
    NormalOf r;
    r.cdf = u >= 0.f ? 1.0f - tail : tail;
    r.pdf = 0.3989422804f * e;
    return r;
}

}  // namespace sw
