// Launches of the clipping of gradients (include/canvas_clip.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <vector>

namespace canvas {
namespace clip {

struct Tensor {
    int64_t count = 0;
    bool bf16 = false, out_bf16 = false;
};

// Tensors are handed to a launch as its arguments, up to kBatch of those that have elements at a time.
constexpr int kBatch = 96;
constexpr int kChunk = 16384;  // elements that a workgroup takes at a time
struct Batch {
    std::vector<int> tensors;
    int64_t chunks = 0;
    int parts = 0;  // workgroups of the launch that adds squares
    int first_part = 0;
};
struct Plan {
    std::vector<Tensor> tensors;
    std::vector<Batch> batches;
    int parts = 0;
    bool one = false;        // few elements: one workgroup, one launch
    bool alone = false;      // the parts are added by a launch of their own, not by every workgroup that scales
    bool past = false;       // what is written goes past the last-level cache
    uint64_t workspace_bytes = 0;
    int launches = 0, launches_norm = 0;
};
void make_plan(Plan& p);

struct Args {
    const void* const* grads;
    void* const* outs;
    double most;
    float *norm, *scale;
    char* ws;
};
void step(const Plan& p, const Args& a, hipStream_t stream);

}  // namespace clip
}  // namespace canvas
