// Scalar functions of the operators around the attention, and a loop over constants.
#pragma once

#include <type_traits>

#include "la_common.h"

namespace la {

constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.693147181f;  // log2(e) in two parts

// exp(-|x|).  The exponential's argument in base 2 is rounded, an error of up to |x| U relative to it: FINE adds what the
// rounding lost; bfloat16 rounds to 2^-8 what that is far below.
template <bool FINE>
__device__ __forceinline__ float exp_down(float x)
{
    const float y = -fabsf(x), t = y * kLog2e;
    float E = __builtin_amdgcn_exp2f(t);
    if (FINE) {
        const float lost = fmaf(y, kLog2eRest, fmaf(y, kLog2e, -t));
        E = fmaf(E, (y > -128.f ? lost : 0.f) * kLn2, E);
    }
    return E;
}
// f = 1 / (1 + exp(-x)) and 1 - f, both from the smaller one's exponential E = exp(-|x|): neither loses digits to a
// difference, and infinite arguments give 0 and 1.
__device__ __forceinline__ void sigmoid_of(float x, float E, float &f, float &rest)
{
    const float large = __builtin_amdgcn_rcpf(1.f + E), small = E * large;
    f = x >= 0.f ? large : small;
    rest = x >= 0.f ? small : large;
}
template <bool FINE>
__device__ __forceinline__ void sigmoid(float x, float &f, float &rest)
{
    sigmoid_of(x, exp_down<FINE>(x), f, rest);
}
// log(1 + exp(x)) = max(x, 0) + log(1 + E).  log(1 + E) = 2 atanh(s), s = E / (2 + E) <= 1/3, by its series up to s^13 (the
// next term is 1.4e-8 of the first): relative to itself it is exact to a few U however small E is.
__device__ __forceinline__ float softplus_of(float x, float E)
{
    const float s = E * __builtin_amdgcn_rcpf(2.f + E), z = s * s;
    float p = fmaf(z, 2.f / 13.f, 2.f / 11.f);
    p = fmaf(z, p, 2.f / 9.f);
    p = fmaf(z, p, 2.f / 7.f);
    p = fmaf(z, p, 2.f / 5.f);
    p = fmaf(z, p, 2.f / 3.f);
    p = fmaf(z, p, 2.f);
    return fmaf(s, p, fmaxf(x, 0.f));
}

// f(0), f(1), .. as constants.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        each<N, I + 1>(f);
    }
}

}  // namespace la
