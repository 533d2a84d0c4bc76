/* C ABI: the norms behind and in front of a block, fused with the block's gate and residual scale.
 *
 * A network of micro-DAG blocks (canvas_dag.h) keeps a residual stream x [N, C, H, W].  Between two blocks it computes,
 * per pixel, over the channels c (means over all C of them):
 *
 *   POST   r2 = (mean_c z^2 + eps)^(-1/2)                      z: the block's output
 *          x' = x + scale[c] * act(gate) * (z * r2 * w_post[c])
 *   PRE    r1 = (mean_c x'^2 + eps)^(-1/2)
 *          u  = x' * r1 * w_pre[c]                             u: the next block's input
 *
 * act is 1 (CANVAS_GATE_NONE), the sigmoid of the gate or gate * sigmoid(gate).  A plan has one of the parts or both; with
 * PRE alone x' is x.  Rows of tokens are maps of one pixel: N rows of C.
 *
 * Gradients, with D the whole gradient of x' (what arrives on the stream, dx_out, and what comes back through u):
 *
 *   xh = x' r1, t1 = mean_c(du w_pre xh):  D = dx_out + r1 (du w_pre - xh t1),  dw_pre[c] = sum du xh,  dx = D
 *   zh = z r2, q = D act scale w_post, t2 = mean_c(q zh):  dz = r2 (q - zh t2),  dgate = D act'(gate) scale w_post zh
 *   dw_post[c] = scale[c] K,  dscale[c] = w_post[c] K,  K = sum D act zh           (sums over n, h, w)
 *
 * Everything is computed in fp32 (the means of squares too: |z| and |x'| up to 1e19) and rounded once where it is stored; u is computed from x' before its rounding, and backward
 * computes that x' again from x, z and the gate (the rounded one would put 2^-9 of every term into the sums of dw_pre, and D
 * is a difference of nearly equal terms where the channels are few).
 * Deterministic: no atomics, sums in a fixed order.
 *
 * Pointers: device pointers, owned by the caller, 16-byte aligned, contiguous NCHW in the plan's element type; w_post,
 * scale, w_pre and their gradients are fp32 tensors of C elements.  What a call writes must not share bytes with anything
 * else that it reads or writes (BAD_ARG).  Tensors that the plan's parts do not have are ignored and may be NULL.  All functions
 * return a canvas_status (0 = OK), canvas_last_error() has the message; nothing is launched after an error was found.
 * A handle keeps no state of its calls: it may be used on several streams with a workspace each.
 */
#ifndef CANVAS_NORM_H
#define CANVAS_NORM_H

#include "canvas_dag.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CANVAS_NORM_POST 1u
#define CANVAS_NORM_PRE 2u
#define CANVAS_NORM_MAX_CHANNELS 16384

typedef enum { CANVAS_GATE_NONE = 0, CANVAS_GATE_SIGMOID = 1, CANVAS_GATE_SILU = 2 } canvas_gate;

typedef struct canvas_norm canvas_norm;

typedef struct canvas_norm_info {
    int32_t n_launches_fwd, n_launches_bwd; /* kernels enqueued per call */
    uint64_t workspace_bytes;               /* r2 and r1 of every pixel, and partial sums of the weights' gradients */
    double min_bytes_fwd, min_bytes_bwd;    /* every tensor of a call read or written once */
} canvas_norm_info;

/* Host only.  shape: N, C, H, W, all >= 1, C <= CANVAS_NORM_MAX_CHANNELS, N * H * W < 2^31.  parts: CANVAS_NORM_POST,
 * CANVAS_NORM_PRE or both.  gate: CANVAS_GATE_NONE without POST.  eps > 0.  opt: flags 0 or CANVAS_OPT_INFERENCE (forward
 * only, no workspace).  Errors: BAD_ARG, UNSUPPORTED (too many channels or pixels). */
int canvas_norm_compile(const int64_t shape[4], canvas_dtype dt, uint32_t parts, canvas_gate gate, float eps,
                        const canvas_options* opt, canvas_norm** out);

int canvas_norm_query(const canvas_norm* norm, canvas_norm_info* info);

/* Reads x, z, gate (unless NONE), w_post, scale, w_pre; writes x_out (x', plans with POST) and u (plans with PRE).  The
 * workspace carries r2 and r1 to canvas_norm_backward. */
int canvas_norm_forward(canvas_norm* norm, const void* x, const void* z, const void* gate, const float* w_post,
                        const float* scale, const float* w_pre, void* x_out, void* u, void* workspace,
                        size_t workspace_bytes, void* stream);

/* After canvas_norm_forward with the same x, z, gate, weights and workspace (x: plans with PRE).  dx_out: the
 * gradient that arrives on the stream; NULL is zero for a plan with PRE.  du: plans with PRE.  Writes dx (plans with PRE;
 * without it the gradient of x is dx_out itself), dz, dgate, dw_post, dscale, dw_pre.
 * Errors: UNSUPPORTED for an inference plan. */
int canvas_norm_backward(canvas_norm* norm, const void* x, const void* z, const void* gate, const float* w_post,
                         const float* scale, const float* w_pre, const void* dx_out, const void* du, void* dx, void* dz,
                         void* dgate, float* dw_post, float* dscale, float* dw_pre, void* workspace,
                         size_t workspace_bytes, void* stream);

void canvas_norm_destroy(canvas_norm* norm);

#ifdef __cplusplus
}
#endif
#endif
