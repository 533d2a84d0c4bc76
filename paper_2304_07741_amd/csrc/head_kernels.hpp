// Launches of the head's log probabilities (include/canvas_head.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "product_kernels.hpp"

namespace canvas {
namespace head {

struct Shape {
    int64_t rows = 0, features = 0, classes = 0;
    bool f32 = false, inference = false;
};

// What backward needs of a row: its largest logit before the temperature (the lowest finite value if there is none), log sum_i exp(z_i - z_max)
// (-inf for a row with nothing left), the entropy and 1 / sum_i exp(z_i - z_max).
struct alignas(16) Row {
    float most, log_sum, entropy, inverse;
};
// The gradient of a row's logits: e^x (first + second x) with x = z_i - z_max (in fp32 plans; in powers of two in bf16 ones), and `token` more at the token.
struct alignas(16) Slope {
    float most, first, second, token;
    int32_t at;        // the token, -1 if there is none
    uint32_t keep;     // 0 for a row whose gradient is zero whatever its logits are
    int32_t unused[2];
};

struct Plan {
    bool few = false, copies = false;
    int kept = 0;                        // pieces whose logits forward leaves for backward
    product::Cut logits, piece, dx, dw;  // `piece`: of the logits of one piece
    int segments = 0;                    // of the classes: what forward leaves sums of
    int pieces = 1;
    int64_t length = 0;                  // of a piece
    int launches_fwd = 0, launches_bwd = 0;
    int launches_mask = 0;               // more of backward with a mask
    int64_t again = 0;                   // classes whose logits backward computes
    uint64_t rows_at = 0, sums_at = 0, token_at = 0, copy_at[2] = {}, slope_at = 0, grad_at = 0, logits_at = 0, parts_dx_at = 0, parts_dw_at = 0, workspace_bytes = 0;
    int64_t most_tiles = 0;
};
Plan plan_of(const Shape& s);

struct Fwd {
    const void *x, *weight;
    float it;  // inverse temperature
    const uint8_t* mask;
    const int64_t* tokens;
    float *logprob, *entropy;
    char* ws;
};
struct Bwd {
    const void *x, *weight;
    float it;
    const uint8_t* mask;
    const int64_t* tokens;
    const float *dlogprob, *dentropy;
    void *dx, *dweight;
    char* ws;
};
void forward(const Shape& s, const Plan& p, const Fwd& a, hipStream_t stream);
void backward(const Shape& s, const Plan& p, const Bwd& a, hipStream_t stream);

}  // namespace head
}  // namespace canvas
