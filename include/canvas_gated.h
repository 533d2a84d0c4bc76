/* C ABI: a gated pair of FCs on rows of features, the widening half of a gated feed-forward block, in one kernel:
 *
 *   g = x Wg^T,  u = x Wu^T,  y = act(g) u                 x [rows, features], Wg and Wu [width, features], y [rows, width]
 *
 * act is the sigmoid, g * sigmoid(g) or the GELU in its erf form.  Gradients:
 *
 *   du = dy act(g),  dg = dy u act'(g)
 *   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x
 *
 * Rows are maps of one pixel; the weights are laid out as those of an FC with one group (weight_shape [1, width, features]).
 *
 * All sums are fp32.  bf16 plans: g and u stay in fp32 up to y, and up to backward, whose dg and du are computed in fp32 and rounded to bf16 once,
 * as operands of the products behind them; dx, dWg and dWu are fp32 sums rounded once.  fp32 plans: products are those of fp32, or, of larger
 * operands, each is taken as three bf16 numbers that together hold its 24 bits (smaller ones than 2^-100 lose their last) and a product adds the six largest of their nine; what
 * is left out is half a step of fp32 at most, of either sign.  An infinity among the operands may act as NaN.  Deterministic: no atomics, sums in a fixed order.
 *
 * Pointers: device pointers, owned by the caller, 16-byte aligned, contiguous, in the plan's element type.  What a call writes must not share
 * bytes with anything else that it reads or writes (BAD_ARG).  All functions return a canvas_status (0 = OK); canvas_last_error() has the
 * message; nothing is launched after an error was found.  A handle keeps no state of its calls: it may be used on several streams with a
 * workspace each.
 */
#ifndef CANVAS_GATED_H
#define CANVAS_GATED_H

#include "canvas_dag.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CANVAS_GATED_MAX_SIDE (1 << 18) /* of features and of width */

typedef enum { CANVAS_GATED_SIGMOID = 0, CANVAS_GATED_SILU = 1, CANVAS_GATED_GELU = 2 } canvas_gated_act;

typedef struct canvas_gated canvas_gated;

typedef struct canvas_gated_info {
    int32_t n_launches_fwd, n_launches_bwd; /* kernels enqueued per call */
    uint64_t workspace_bytes;               /* g and u for backward, dg and du, copies of operands, parts of sums */
    double flops_fwd, flops_bwd;            /* of the products above */
    double min_bytes_fwd, min_bytes_bwd;    /* every tensor of a call read or written once */
} canvas_gated_info;

/* Host only.  1 <= rows < 2^31, 1 <= features, width <= CANVAS_GATED_MAX_SIDE; at most 2^23 - 1 tiles of 128 x 128 results
 * (times the parts of their sums) per product.
 * opt: flags 0 or CANVAS_OPT_INFERENCE (forward only).  Errors: BAD_ARG, UNSUPPORTED. */
int canvas_gated_compile(int64_t rows, int64_t features, int64_t width, canvas_dtype dt, canvas_gated_act act, const canvas_options* opt,
                         canvas_gated** out);

int canvas_gated_query(const canvas_gated* gated, canvas_gated_info* info);

/* Reads x, w_gate, w_up; writes y.  The workspace carries g and u, and copies of x and of the weights, to canvas_gated_backward. */
int canvas_gated_forward(canvas_gated* gated, const void* x, const void* w_gate, const void* w_up, void* y, void* workspace,
                         size_t workspace_bytes, void* stream);

/* After canvas_gated_forward with the same x, weights and workspace; may be called again.  Writes dx, dw_gate, dw_up.
 * Errors: UNSUPPORTED for an inference plan. */
int canvas_gated_backward(canvas_gated* gated, const void* x, const void* w_gate, const void* w_up, const void* dy, void* dx, void* dw_gate,
                          void* dw_up, void* workspace, size_t workspace_bytes, void* stream);

void canvas_gated_destroy(canvas_gated* gated);

#ifdef __cplusplus
}
#endif
#endif
