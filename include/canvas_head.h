/* C ABI: log probabilities of given tokens with the entropy of their distributions, straight from features and the head's weight, and the
 * gradients of both: the loss of a head with many classes whose logits (rows x classes) are no tensor of the step.
 *
 * x [rows, features], W [classes, features].  With z_i = inv_temperature * (x . W_i) over the classes that the mask allows:
 *
 *   logprob = z_token - log sum_i exp z_i          entropy = - sum_i p_i log p_i,  p_i = exp(z_i) / sum_j exp z_j
 *   dlogit_i = inv_temperature * ( dlogprob (1[i = token] - p_i) - dentropy p_i (log p_i + entropy) ),  0 where masked
 *   dx = sum_i dlogit_i W_i,  dW_i = sum over the rows of dlogit_i x
 *
 * as canvas_logprob.h has them for logits that are at hand.  Forward keeps the largest logit and the sums of each row; backward takes the
 * classes a piece at a time, computes a piece's logits again, the same ones, and leaves its gradients (up to 288 MB of pieces of 256 classes and more) in the
 * workspace only.  Some logits are not computed again but left there by forward, in fp32: those of few rows (up to 32; in fp32 plans of any number that takes the same
 * way, 512 MB at most), all where they are 16 MB or less, and of plans with 2048 features or more (fp32: 512) those of the first pieces, up to a GiB.
 *
 * A masked class is not looked at (its row of W may be NaN) and has a gradient of zeros.  A row of x that has nothing left (all classes masked
 * or -inf) has the log probability -inf, the entropy 0 and a gradient of zeros.  A token that is no class (negative, say, for positions
 * without a target) has the log probability 0 and adds nothing to the gradient: without dentropy such a row of x may be NaN, and its gradient
 * is zero.  So it is of any row whose dlogprob and dentropy are zero or not given.  A masked token has the log probability -inf.  NaN or +inf among the allowed logits makes
 * log probability, entropy and gradients of its row NaN, and dW with them.  dx is a sum over all allowed classes: NaN or an infinity in one's row of W makes the same element
 * of dx NaN in every row, those without a gradient among them (zero times it is NaN).
 *
 * All sums are fp32.  bf16 plans: dlogit is rounded to bf16 once, as the operand of the products behind it; dx and dW are fp32 sums rounded
 * once.  fp32 plans: products are those of fp32, or, of larger operands, each is taken as three bf16 numbers that together hold its 24 bits (smaller ones than 2^-100
 * lose their last) and a product adds the six largest of their nine; what is left out is half a step of fp32 at most, of either sign.  An infinity among the operands may act
 * as NaN.  Deterministic: no atomics, sums in a fixed order.
 *
 * Pointers: device pointers, owned by the caller, 16-byte aligned, contiguous; x, W and their gradients in the plan's element type.  What a
 * call writes must not share bytes with anything else that it reads or writes (BAD_ARG).  All functions return a canvas_status (0 = OK);
 * canvas_last_error() has the message; nothing is launched after an error was found.  A handle keeps no state of its calls: it may be used on
 * several streams with a workspace each.
 */
#ifndef CANVAS_HEAD_H
#define CANVAS_HEAD_H

#include "canvas_dag.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CANVAS_HEAD_MAX_FEATURES (1 << 18)
#define CANVAS_HEAD_MAX_CLASSES (1 << 20)

typedef struct canvas_head canvas_head;

typedef struct canvas_head_info {
    int32_t n_launches_fwd, n_launches_bwd; /* kernels enqueued per call, without a mask */
    int32_t pieces;                         /* how many pieces backward takes the classes in */
    int32_t n_launches_bwd_mask;            /* as many more with one: copies of a weight that is otherwise read as it is */
    uint64_t workspace_bytes;               /* the rows' sums, a piece's dlogit, copies of operands, parts of sums, some logits */
    double flops_fwd, flops_bwd;            /* of the products above; backward's with those of the logits that it computes again */
    double min_bytes_fwd, min_bytes_bwd;    /* every tensor of a call read or written once; without a mask */
} canvas_head_info;

/* Host only.  1 <= rows < 2^31, 1 <= features <= CANVAS_HEAD_MAX_FEATURES, 1 <= classes <= CANVAS_HEAD_MAX_CLASSES; at most 2^23 - 1
 * tiles of 128 x 128 results (times the parts of their sums) per product.  opt: flags 0 or CANVAS_OPT_INFERENCE (no backward).  Errors: BAD_ARG, UNSUPPORTED. */
int canvas_head_compile(int64_t rows, int64_t features, int64_t classes, canvas_dtype dt, const canvas_options* opt, canvas_head** out);

int canvas_head_query(const canvas_head* head, canvas_head_info* info);

/* inv_temperature: finite, > 0.  mask: one byte per class, 0 = not allowed, the same for all rows; NULL allows everything.  tokens [rows]
 * int64.  Writes logprob [rows] and entropy [rows], fp32.  tokens and logprob may both be NULL, entropy may be NULL. */
int canvas_head_forward(canvas_head* head, const void* x, const void* weight, float inv_temperature, const uint8_t* mask, const int64_t* tokens,
                        float* logprob, float* entropy, void* workspace, size_t workspace_bytes, void* stream);

/* After canvas_head_forward with the same x, weight, mask, temperature and workspace; may be called again.  dlogprob [rows] and dentropy [rows],
 * fp32: the gradients that arrive; either may be NULL (zeros).  tokens may be NULL with dlogprob NULL.  Writes dx and dweight.
 * Errors: UNSUPPORTED for an inference plan. */
int canvas_head_backward(canvas_head* head, const void* x, const void* weight, float inv_temperature, const uint8_t* mask, const int64_t* tokens,
                         const float* dlogprob, const float* dentropy, void* dx, void* dweight, void* workspace, size_t workspace_bytes,
                         void* stream);

void canvas_head_destroy(canvas_head* head);

#ifdef __cplusplus
}
#endif
#endif
