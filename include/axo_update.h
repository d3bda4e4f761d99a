/*
 * axo_update.h -- C ABI of what becomes of a weight's gradient on its way into the weight, on MI355X (gfx950): the orthogonalised update.
 *
 * axo_fc_wgrad, axo_fc_wgrad_acc and the gated block's forms of them leave the gradient of a weight [K x N], axo_ortho takes it (or a momentum that the program keeps of
 * it) to an update whose singular values are all about 1, and the program adds that, times its learning rate, to the weight.
 *
 * Problems, data, ownership, checks and statuses are those of axo.h: the caller owns every buffer, the library only enqueues on the caller's stream, allocates no device memory and
 * keeps no pointer.
 */
#ifndef AXO_UPDATE_H
#define AXO_UPDATE_H

#include "axo_block.h" /* axo_type_t */

#ifdef __cplusplus
extern "C" {
#endif

#define AXO_ORTHO_MOST_STEPS 64

/* O[K x N] = X after `steps` (1 to AXO_ORTHO_MOST_STEPS) of the Newton-Schulz iteration
 *   X <- G / (|G| + eps), |G| the root of the sum of squares;   X <- a X + b (X X^T) X + c (X X^T)^2 X
 * which maps every singular value v of X to a v + b v^3 + c v^5 and leaves the singular vectors as they are.  p is the problem of the layer whose weight it is: K in-features,
 * N out-features; T is not used.  The iteration needs the whole matrix: grids whose X and Y axes have size 1 (BAD_GRID otherwise; on others the caller gathers the gradient, and
 * each GPU of the group can take weights of its own).
 * G: of `type` (axo_type_t).  abc: 3 * steps floats in HOST memory, read before the call returns, (a, b, c) of each step; NULL: (3.4445, -4.7750, 2.0315) in all, of which five
 * steps bring singular values from 0.01 on to between 0.6 and 1.3.  The coefficients have to keep singular values below 2: X is held in fp16 between steps.  eps >= 0 and
 * finite.  A G of zeros gives zeros.  A G with an infinity or a NaN gives NaN.
 * O: bf16, rounded once.  Between steps X, X X^T and its polynomial are rounded to fp16, X times a power of two; sums are fp32, |G| is formed in fp64.  Before its rounding to bf16
 * (0.2 %) O is off by 0.1 to 0.2 % for random G, and, what rounding adds being taken up along with G's small singular values, for G whose singular values lie evenly in their logarithm
 * over a factor of 10 by 0.1 %, 30 0.2, 100 0.2 to 0.4, 1000 0.3 to 1.1 (five steps; with X, X X^T and its polynomial in bf16 eight times as much).  Results are a fixed function of the inputs.
 * ws: axo_ortho_workspace_bytes(p) bytes or more of device memory, 16-byte aligned.  It begins with arrival counters: zero-fill it once after allocating it and leave it to
 * calls of axo_ortho, of any sizes that it is large enough for, which must not overlap in time on one workspace.
 * Errors: those of axo_shard_dims; BAD_GRID; BAD_ARG (type, steps, coefficients or eps, shared bytes); NULL_PTR, BAD_LD, MISALIGNED; BAD_SIZE (a weight
 * is taken with s (l + 256) below 2^31 - 2^15, s the smaller and l the larger of K and N, each rounded up to 64); WORKSPACE; HIP. */
int axo_ortho(const axo_problem_t *p, const void *G, int64_t ldg, int type, int steps, const float *abc, float eps, void *O, int64_t ldo, void *ws,
              size_t ws_bytes, void *hip_stream);

/* Host only.  Bytes of device workspace that axo_ortho needs for this problem; 0 for an invalid one. */
size_t axo_ortho_workspace_bytes(const axo_problem_t *p);

#ifdef __cplusplus
}
#endif
#endif /* AXO_UPDATE_H */
