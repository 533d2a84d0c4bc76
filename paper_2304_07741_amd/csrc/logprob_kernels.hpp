// Launches of the token log probabilities (include/canvas_logprob.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace canvas {
namespace logprob {

struct Shape {
    int64_t rows = 0, classes = 0;
    bool bf16 = false;
    int top = 0;
};

// What backward needs of a row: its largest logit (the lowest finite value if there is none), log sum_i exp(z_i - z_max) (-inf for a row
// with nothing left), the entropy and 1 / sum_i exp(z_i - z_max).
struct alignas(16) Row {
    float most, log_sum, entropy, inverse;
};

// Rows are read in `segments` pieces of `length` classes by `threads` threads.
struct Plan {
    uint64_t workspace_bytes = 0;  // the rows' results first, then those of segments
    uint64_t parts_at = 0, keys_at = 0;
    int64_t length = 0;
    int segments = 1, threads = 0;
    int launches_fwd = 1;
};
Plan plan_of(const Shape& s);

struct Fwd {
    const void* logits;
    int64_t pitch;
    float it;  // inverse temperature
    const uint8_t* mask;
    int64_t mask_pitch;
    const int64_t* tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t* top_index;
    char* ws;
};
struct Bwd {
    const void* logits;
    int64_t pitch;
    float it;
    const uint8_t* mask;
    int64_t mask_pitch;
    const int64_t* tokens;
    const float *dlogprob, *dentropy;
    void* dlogits;
    int64_t dpitch;
    const char* ws;
};

void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream);
void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream);

}  // namespace logprob
}  // namespace canvas
