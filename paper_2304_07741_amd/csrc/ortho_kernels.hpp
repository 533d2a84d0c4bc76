// Launches of the orthogonalised update (include/canvas_ortho.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace canvas {
namespace ortho {

struct Shape {
    int64_t G = 0, R = 0, K = 0;
    int64_t m = 0, n = 0;  // the shorter and the longer side
    bool tall = false;     // R > K: the products work on the transposed matrices
    bool bf16 = false, nesterov = false;
    int steps = 0;
};

struct Plan {
    uint64_t workspace_bytes = 0;
    int launches = 0;
    bool small = false;       // one launch of ortho_small_kernels.hip, without a workspace
    int parts = 0;            // workgroups per matrix that square and sum
    uint64_t part_bytes = 0;  // of sums that are cut into parts
    int64_t workgroups = 0;   // of the longest launch, of 256 threads each
};
Plan plan_of(const Shape& s);

struct Args {
    const float *grad, *momentum;
    float* momentum_out;
    double mu;
    const float* master;
    float* master_out;
    double lr, decay;
    void *weights, *update;
    char* ws;
};

void step(const Shape& s, const Plan& p, const Args& a, hipStream_t stream);

}  // namespace ortho
}  // namespace canvas
