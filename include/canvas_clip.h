/* C ABI: the norm over all gradients of a network, and the gradients scaled down to a largest norm: what a training step does between
 * backward and the updates of its weights.
 *
 *   norm = (sum of the squares of all elements of all tensors)^(1/2)
 *   scale = min(1, max_norm / norm)                 (1 for a norm of zero)
 *   out_i = scale * grad_i                          element by element
 *
 * Squares are added in 64 bits: gradients of any size that their types hold are in range (a norm that fp32 does not hold is written as
 * infinity, the scale is right all the same).  The scale is rounded to fp32 and so is its product with an element, which is rounded again where out_i is bf16; scales
 * below fp32's normal numbers are taken in 64 bits.  NaN among the elements makes norm, scale and all of out NaN.  An infinity makes the norm infinite and the scale 0: finite
 * elements become 0, infinite ones NaN.  max_norm = infinity asks for the norm and, where a tensor's types differ, for its conversion: the scale is 1 whatever the norm, and
 * every element stays what it is, NaN and infinities too; the norm tells of them.  Deterministic: no atomics, sums in a fixed order.
 *
 * Pointers: device pointers, owned by the caller, aligned to their element (16-byte aligned ones are read in whole vectors).  out_i may be
 * grad_i itself where both have one type; apart from that, what a call writes must not share bytes with anything else that it reads or writes
 * (BAD_ARG).  A tensor without elements may be NULL.  All functions return a canvas_status (0 = OK); canvas_last_error() has the message;
 * nothing is launched after an error was found.  A handle keeps no state of its calls: it may be used on several streams with a workspace each.
 */
#ifndef CANVAS_CLIP_H
#define CANVAS_CLIP_H

#include "canvas_dag.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CANVAS_CLIP_MAX_TENSORS 65536

typedef struct canvas_clip canvas_clip;

typedef struct canvas_clip_info {
    int32_t n_launches, n_launches_norm; /* kernels enqueued by a call that writes out, and by one that asks for the norm alone */
    uint64_t workspace_bytes;            /* partial sums */
    double min_bytes;                    /* every gradient read once and written once */
} canvas_clip_info;

/* Host only.  tensors: 1 .. CANVAS_CLIP_MAX_TENSORS; counts [tensors]: their elements, each 0 .. 2^40, fewer than 2^44 in all; types [tensors]
 * and out_types [tensors] (NULL: the same).  Errors: BAD_ARG, UNSUPPORTED. */
int canvas_clip_compile(int32_t tensors, const int64_t* counts, const canvas_dtype* types, const canvas_dtype* out_types, canvas_clip** out);

int canvas_clip_query(const canvas_clip* clip, canvas_clip_info* info);

/* grads [tensors] and outs [tensors]: host arrays of device pointers, read before the call returns.  outs may be NULL (the norm alone).
 * max_norm > 0.  Writes norm and scale, fp32, one element each, on the device; scale may be NULL. */
int canvas_clip_step(canvas_clip* clip, const void* const* grads, void* const* outs, double max_norm, float* norm, float* scale, void* workspace,
                     size_t workspace_bytes, void* stream);

void canvas_clip_destroy(canvas_clip* clip);

#ifdef __cplusplus
}
#endif
#endif
