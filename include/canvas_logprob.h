/* C ABI: log probabilities of given tokens with the entropy and the top alternatives of their distributions, and the
 * gradient of both: the loss of a head whose logits are rows of classes, and what a sampler reports of its choice.
 *
 * logits: `rows` rows of `classes` elements, `pitch` elements from one row to the next (an FC over maps of one pixel writes
 * them so, with pitch = classes).  With z_i = inv_temperature * logit_i over the classes that the mask allows:
 *
 *   logprob = z_token - log sum_i exp z_i          entropy = - sum_i p_i log p_i,  p_i = exp(z_i) / sum_j exp z_j
 *   dlogit_i = inv_temperature * ( dlogprob (1[i = token] - p_i) - dentropy p_i (log p_i + entropy) ),  0 where masked
 *
 * Top alternatives: the top_k allowed classes with the largest logits, largest first, the lower index first among equals,
 * with their log probabilities.  A class that is masked or has the logit -inf is no alternative; places without one have the
 * index -1 and the log probability -inf.
 *
 * What a mask hides is not looked at (it may be NaN).  A row that has nothing left (all masked or -inf) has the log
 * probability -inf, the entropy 0, no alternatives and a gradient of zeros.  A token that is no class (negative, say, for
 * positions without a target) has the log probability 0 and adds nothing to the gradient.  A masked token has the log
 * probability -inf.  NaN or +inf among the allowed logits makes log probabilities, entropy and gradient of its row NaN; NaN
 * is then the first alternative.
 *
 * Sums are kept in fp32 relative to the row's largest logit.  Deterministic: no floating-point atomics.
 *
 * Pointers: device pointers, owned by the caller; logits and dlogits are aligned to their element, the others to 16 bytes.
 * What a call writes must not share bytes with anything else that it reads or writes (BAD_ARG), dlogits in the place of logits
 * aside; rows of the one between the rows of the other do not.
 * All functions return a canvas_status (0 = OK); canvas_last_error() has the message; nothing is launched after an error was
 * found.  A handle keeps no state of its calls: it may be used on several streams with a workspace each.
 */
#ifndef CANVAS_LOGPROB_H
#define CANVAS_LOGPROB_H

#include "canvas_dag.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CANVAS_LOGPROB_MAX_TOP 64
#define CANVAS_LOGPROB_MAX_CLASSES (1 << 20)

typedef struct canvas_logprob canvas_logprob;

typedef struct canvas_logprob_info {
    int32_t n_launches_fwd, n_launches_bwd; /* kernels enqueued per call */
    uint64_t workspace_bytes;               /* what backward needs of every row, and the parts of rows that are split */
    double min_bytes_fwd, min_bytes_bwd;    /* logits read once, or read and written once; without a mask */
} canvas_logprob_info;

/* Host only.  1 <= rows < 2^31, 1 <= classes <= CANVAS_LOGPROB_MAX_CLASSES, dt: type of logits and dlogits,
 * 0 <= top_k <= CANVAS_LOGPROB_MAX_TOP.  opt: flags 0 or CANVAS_OPT_INFERENCE (no backward).  Errors: BAD_ARG, UNSUPPORTED (too many rows or classes). */
int canvas_logprob_compile(int64_t rows, int64_t classes, canvas_dtype dt, int32_t top_k, const canvas_options* opt,
                           canvas_logprob** out);

int canvas_logprob_query(const canvas_logprob* lp, canvas_logprob_info* info);

/* inv_temperature: finite, > 0.  mask: one byte per class, 0 = not allowed, mask_pitch bytes from one row's to the next's (0:
 * one mask for all rows); NULL allows everything.  tokens [rows] int64.  Writes logprob [rows] and entropy [rows], fp32, and
 * with top_k > 0 top_logprob [rows, top_k], fp32, and top_index [rows, top_k], int32.  tokens and logprob may both be NULL
 * (entropy and alternatives alone), entropy may be NULL. */
int canvas_logprob_forward(canvas_logprob* lp, const void* logits, int64_t pitch, float inv_temperature, const uint8_t* mask,
                           int64_t mask_pitch, const int64_t* tokens, float* logprob, float* entropy, float* top_logprob,
                           int32_t* top_index, void* workspace, size_t workspace_bytes, void* stream);

/* After canvas_logprob_forward with the same logits, mask, tokens, temperature and workspace.  dlogprob [rows] and
 * dentropy [rows], fp32: the gradients that arrive; either may be NULL (zeros).  tokens may be NULL with dlogprob NULL.
 * Writes dlogits, `dpitch` elements from one row to the next; what lies between the rows is not written.  dlogits may be
 * logits itself with dpitch = pitch. */
int canvas_logprob_backward(canvas_logprob* lp, const void* logits, int64_t pitch, float inv_temperature,
                            const uint8_t* mask, int64_t mask_pitch, const int64_t* tokens, const float* dlogprob,
                            const float* dentropy, void* dlogits, int64_t dpitch, void* workspace, size_t workspace_bytes,
                            void* stream);

void canvas_logprob_destroy(canvas_logprob* lp);

#ifdef __cplusplus
}
#endif
#endif
