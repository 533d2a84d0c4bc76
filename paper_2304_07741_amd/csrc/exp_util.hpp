// Exponentials by the unit for powers of two.  x log2(e) is rounded, by up to 2^-24 of itself, which moves the power by as many units as |x| has:
// c = x - t ln 2, exact but for the last bits with ln 2 in two parts, makes it good as e^x = 2^t (1 + c).
#pragma once
#include <hip/hip_runtime.h>

namespace canvas {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kLn2Rest = (float)(0.6931471805599453094 - (double)kLn2);

__device__ __forceinline__ float exp_rest(float x, float t) { return fmaf(-t, kLn2Rest, fmaf(-t, kLn2, x)); }
// e^x to about a unit of the last place; x in [-300, 88].
__device__ __forceinline__ float exp_finite(float x) {
    const float t = x * kLog2e, y = __builtin_amdgcn_exp2f(t);
    return fmaf(y, exp_rest(x, t), y);
}

}  // namespace canvas
