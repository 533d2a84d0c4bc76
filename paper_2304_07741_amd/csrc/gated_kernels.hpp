// Launches of the gated pair of FCs (include/canvas_gated.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "product_kernels.hpp"

namespace canvas {
namespace gated {

struct Shape {
    int64_t rows = 0, features = 0, width = 0;
    bool f32 = false, inference = false;
    int act = 0;
};

struct Plan {
    bool few = false;      // few rows (few::fits): operands are read as they are
    bool copies = false;   // products read copies of x and the weights: three planes of fp32 ones, rows of a multiple of 8 of bf16 ones
    product::Cut forward, dx, dw;
    int launches_fwd = 0, launches_bwd = 0;
    // where the workspace holds what, and its end
    uint64_t kept_at = 0, copy_at[3] = {}, grad_at = 0, parts_at = 0, parts_dw_at = 0, workspace_bytes = 0;
    int64_t most_tiles = 0;
};
Plan plan_of(const Shape& s);

struct Fwd {
    const void *x, *w_gate, *w_up;
    void* y;
    char* ws;
};
struct Bwd {
    const void *x, *w_gate, *w_up, *dy;
    void *dx, *dw_gate, *dw_up;
    char* ws;
};
void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream);
void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream);

}  // namespace gated
}  // namespace canvas
