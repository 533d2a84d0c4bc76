// Launches of the residual norm (include/canvas_norm.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace canvas {
namespace norm {

struct Shape {
    int64_t N = 0, P = 0;  // images, pixels of one
    int C = 0;
    bool bf16 = false, post = false, pre = false;
    int gate = 0;  // canvas_gate
    float eps = 0.f;
    float down = 1.f;  // the power of two at C^-1/2 or below: squares are summed of values times it, so that the sum has the range of the mean
};

// How maps are cut: pieces side by side in a workgroup, its threads, channels that a thread holds.
struct Tiling {
    int log_gx = 0, threads = 0, kc = 0;
};
// Which kernels a shape takes.
struct Plan {
    int tpr = 0, kv = 0;      // rows: threads per row, 16-byte accesses of a thread (0: maps)
    int vec = 0, pieces = 0;  // maps: pixels of a thread, pieces of a plane
    int64_t total = 0;        // of all planes
    Tiling fwd, bwd;
    int partials = 0;         // workgroups of the backward kernel
};
Plan plan_of(const Shape& s);

struct Fwd {
    const void *x, *z, *g;
    const float *w_post, *scale, *w_pre;
    void *x_out, *u;
    float *r2, *r1;  // one per pixel, null for an inference plan
};
struct Bwd {
    const void *x, *z, *g;
    const float *w_post, *scale, *w_pre;
    const void *dx_out, *du;
    void *dx, *dz, *dg;
    float *dw_post, *dscale, *dw_pre;
    const float *r2, *r1;
    float* partial;  // [partials][2][C]: sums of D act zh, of du xh
};

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream);
void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream);
// Everything but the sums over the partials.
void maps_backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream);
void rows_backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream);

}  // namespace norm
}  // namespace canvas
