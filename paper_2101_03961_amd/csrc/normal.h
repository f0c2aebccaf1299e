// The normal distribution of the gated-GELU experts and of switch_linear's activations.
#pragma once
#include "common.h"

namespace sw {

// Phi(u) and the density phi(u) of the standard normal distribution, sharing one exponential.
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

}  // namespace sw
