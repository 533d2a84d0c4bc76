// Orthogonalised updates of matrices that one workgroup holds in LDS.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "ortho_kernels.hpp"

namespace canvas {
namespace ortho {

constexpr int kMostSmallLds = 128 * 1024;

struct SmallPlan {
    bool fits = false;
    int mp = 0, np = 0, ld = 0;  // sides in 16s, floats from one row of X to the next
    int lds = 0;                 // bytes
};
__host__ __device__ inline SmallPlan small_plan(const Shape& s) {
    SmallPlan p;
    if (s.m > 64 || s.n > 4096) return p;
    p.mp = (int)(s.m + 15) / 16 * 16;
    p.np = (int)(s.n + 15) / 16 * 16;
    p.ld = p.np + 4;
    const int tiles = (p.mp / 16) * (p.mp / 16), units = tiles > 8 ? tiles : 8;
    p.lds = 4 * (p.mp * p.ld + 2 * p.mp * (p.mp + 4) + units * 256);
    // (one compute unit against a chain of launches over all: 89 us against 90 at 64 x 256, 112 against 102 at 48 x 500)
    p.fits = p.lds <= kMostSmallLds && p.mp * p.np <= 24000;
    return p;
}

void step_small(const Shape& s, const Args& a, hipStream_t stream);

}  // namespace ortho
}  // namespace canvas
