/* C ABI: the update of an FC weight, orthogonalised by Newton-Schulz products.
 *
 * canvas_dag_backward gives the gradient of an FC weight as G matrices [R, K] in fp32 (weight_shape of canvas_dag_info).  An
 * orthogonalised update replaces each by a matrix with nearly the same singular vectors and all singular values near one:
 *
 *   m' = mu m + g              momentum, fp32            v = g + mu m' (CANVAS_ORTHO_NESTEROV) or m'
 *   X  = v / (|v|_F + 1e-7)    transposed where R > K
 *   `steps` times:  A = X X^T,  X = a X + (b A + c A A) X      (a, b, c) = (3.4445, -4.7750, 2.0315), the coefficients of
 *                   K. Jordan et al., "Muon: an optimizer for hidden layers in neural networks" (2024)
 *   update = X (transposed back),  master' = (1 - lr decay) master - lr update,  weights = master' in the plan's type
 *
 * The products run on the matrix units with fp32 sums.  Each operand is a pair of fp16 numbers that together hold 22 bits of
 * it, and a product adds the three pairings that matter, which is as exact as products in fp32 (measured against
 * 64 bits: 0.4 to 1.2 times their error, on noise and on singular values that spread over six decades; |X| <= 1.3 throughout; a
 * power of two per matrix keeps both numbers in range where X is small).  Where the longer side is several times the shorter one, two steps are joined, which
 * changes the order of the products and not what they are: both polynomials of A are multiplied before X is.  The sum of squares is kept in 64 bits: gradients of any size that fp32 holds are
 * in range.  A matrix of zeros gives zeros; infinities and NaN make their own matrix NaN and no other.
 *
 * Pointers: device pointers, owned by the caller, 16-byte aligned, contiguous [G, R, K].  All functions return a
 * canvas_status (0 = OK); canvas_last_error() has the message; nothing is launched after an error was found.  A handle keeps
 * no state of its calls: it may be used on several streams with a workspace each.
 */
#ifndef CANVAS_ORTHO_H
#define CANVAS_ORTHO_H

#include "canvas_dag.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CANVAS_ORTHO_NESTEROV 1u
#define CANVAS_ORTHO_MAX_SIDE 16384 /* of the shorter side of a matrix */
#define CANVAS_ORTHO_MAX_STEPS 16

typedef struct canvas_ortho canvas_ortho;

typedef struct canvas_ortho_info {
    int32_t n_launches;       /* kernels enqueued per call */
    int32_t reserved0;
    uint64_t workspace_bytes;
    double flops;             /* of the products as they are written above, each symmetric one on one side of its diagonal only */
    double min_bytes;         /* gradient read, update written; momentum read and written; without master weights */
} canvas_ortho_info;

/* Host only.  shape: G, R, K, all >= 1, G <= 65535, min(R, K) <= CANVAS_ORTHO_MAX_SIDE, R * K < 2^30, G * R * K < 2^31, and fewer
 * than 2^24 blocks of 64 x 64 in all.  dt: type of update and weights.
 * steps: 0 .. CANVAS_ORTHO_MAX_STEPS (0: the normalised matrix itself).  flags: 0 or CANVAS_ORTHO_NESTEROV.
 * Errors: BAD_ARG, UNSUPPORTED. */
int canvas_ortho_compile(const int64_t shape[3], canvas_dtype dt, int32_t steps, uint32_t flags, canvas_ortho** out);

int canvas_ortho_query(const canvas_ortho* ortho, canvas_ortho_info* info);

/* grad fp32.  momentum and momentum_out: fp32, read and written, both or neither (then v = g); they may be the same tensor.
 * master and master_out: fp32, both or neither; they may be the same tensor.  weights: needs master; may be NULL.
 * update: may be NULL when master is given.  mu in [0, 1); lr and decay finite.  Nothing else that is written
 * may share bytes with anything (BAD_ARG). */
int canvas_ortho_step(canvas_ortho* ortho, const float* grad, const float* momentum, float* momentum_out, double mu,
                      const float* master, float* master_out, double lr, double decay, void* weights, void* update,
                      void* workspace, size_t workspace_bytes, void* stream);

void canvas_ortho_destroy(canvas_ortho* ortho);

#ifdef __cplusplus
}
#endif
#endif
