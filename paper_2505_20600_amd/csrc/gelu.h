// GELU as the row products' epilogues compute it (gemm.hip, mx4_linear.hip).
#pragma once

#include "common.h"

namespace ms {

// GELU(x) = x (1 + erf(x / sqrt 2)) / 2 = max(x, 0) - |x| erfc(|x| / sqrt 2) / 2, with
// erfc(y) by Abramowitz & Stegun, Handbook of Mathematical Functions, formula
// 7.1.26: t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) exp(-y^2), t = 1 / (1 + p y),
// |error| <= 1.5e-7. An absolute bound: the result is within 3.3e-7 of GELU over
// [-12, 12], far below the bf16 rounding of most outputs, but the tail of negative x
// is relatively off by 0.2% at -5 and 3% at -12 (as 0.5 x (1 + erf) loses it to the
// subtraction). One reciprocal, one exponential and twelve other instructions (the
// epilogue of a 256 x 256 tile evaluates 128 per lane, ~60 cycles each as
// 0.5 x (1 + erf)).
// |x| is taken of min(x, FLT_MAX), so that +inf gives +inf and not inf - inf * 0;
// -inf gives NaN, as x (1 + erf) does.
__device__ __forceinline__ float gelu(float x) {
    const float ax = fabsf(fminf(x, 3.402823466e+38f));
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, ax, 1.0f));
    float q = fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);
    q = fmaf(q, t, 0.5f * 1.421413741f);
    q = fmaf(q, t, 0.5f * -0.284496736f);
    q = fmaf(q, t, 0.5f * 0.254829592f);
    q *= t * __builtin_amdgcn_exp2f(x * (x * (-0.5f * 1.4426950408889634f)));
    return fmaf(-ax, q, fmaxf(x, 0.f));
}

}  // namespace ms
