// Sums and maxima over the lanes of a wavefront, by moves between registers (no LDS traffic).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace canvas {
namespace wave {

struct Sum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};

// v joined with the value of the lane `O` places away in a pattern that all lanes of a group of 2 O lanes see alike.  For O = 8 and
// less the groups of 2 O lanes must hold the same values already (a row of 16 lanes is rotated), so use them in the order
// 32, 16, 8, 4, 2, 1.
template <int O, class J>
__device__ __forceinline__ float step(float v) {
    const uint32_t u = __float_as_uint(v);
    if (O == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return J::of(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if (O == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return J::of(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return J::of(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, u, 0x120 + (O & 15), 0xf, 0xf, true)));
}

// Over the lanes whose numbers differ in the bits from LOW on: LOW = 1 is the whole wavefront.
template <int LOW, class J>
__device__ __forceinline__ float over(float v) {
    if (LOW <= 32) v = step<32, J>(v);
    if (LOW <= 16) v = step<16, J>(v);
    if (LOW <= 8) v = step<8, J>(v);
    if (LOW <= 4) v = step<4, J>(v);
    if (LOW <= 2) v = step<2, J>(v);
    if (LOW <= 1) v = step<1, J>(v);
    return v;
}

}  // namespace wave
}  // namespace canvas
