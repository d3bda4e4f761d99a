/*
 * axo_block.h -- C ABI of what surrounds the fully-connected layers of axo.h in a transformer's MLP sublayer on MI355X
 * (gfx950): layer norm and the gated feed-forward block, forward and backward.
 *
 *   n = norm(x + r)                        axo_norm_fwd
 *   h = act(n Wg + bg) * (n Wu + bu)       axo_gated_fwd        (a layer of two weight matrices, K -> N each)
 *   y = h Wd                               axo_fc_fwd           (the layer behind it, N -> K; with its residual: axo_fc_add, and the norms around the addition:
 *                                                               axo_resnorm_fwd, both of axo_residual.h)
 *
 * and back: axo_gated_dgrad_act takes dY through Wd and the product to (dG, dU), axo_gated_dgrad and axo_gated_wgrad give the
 * gradients of n, Wg and Wu, axo_norm_bwd those of x, gamma and beta; axo_fc_wgrad gives dWd, axo_bias_grad the biases'.
 *
 * Problems, shards, data and ownership are those of axo.h: every call works on this GPU's shard (M x Kl activations, Kl x Nl weights)
 * of an axo_problem_t, matrices are row-major with leading dimensions in elements (multiples of 8; pointers 16-byte aligned), the caller
 * owns every buffer, the library only enqueues on the caller's stream, allocates nothing and keeps no pointer.  No output may share a byte with
 * an input or with another output of the same call (AXO_ERR_BAD_ARG).  Matrices without elements are never dereferenced.
 * All checks run on the host ahead of the first HIP call; statuses are those of axo.h.
 *
 * Arithmetic: sums, statistics and activations in fp32; every bf16 result is rounded once, to nearest even.  No floating-point atomics: results are
 * a fixed function of the inputs.
 *
 * Where an axis of the grid splits the width of a row or a reduction, a GPU's result is a part of the layer's:
 *   - a norm needs whole rows.  axo_norm_fwd and axo_norm_bwd take grids whose K axis has size 1 (AXO_ERR_BAD_GRID otherwise); on
 *     others axo_norm_part gives each shard's statistics, which the caller gathers over the K axis, and axo_norm_apply finishes; back
 *     axo_norm_bwd_part gives two sums per row, which the caller adds up over the K axis, and axo_norm_bwd_apply finishes.
 *   - the activation of the gated block belongs behind the sum over the K axis.  Where that has size 1, axo_gated_fwd and (for the layer
 *     behind the block, whose data gradient is summed over its N axis) axo_gated_dgrad_act are whole; elsewhere two axo_fc_fwd, the
 *     all-reduce and axo_gated_act give H, and axo_fc_dgrad, the all-reduce and axo_gated_dact give (dG, dU).  Neither call refuses
 *     the other grids: axo_gated_fwd then gives this shard's parts of G and U, and an H of those parts, which is no part of the layer's.
 */
#ifndef AXO_BLOCK_H
#define AXO_BLOCK_H

#include "axo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of the residual stream: what a norm reads and the gradient that it hands back.  Everything else is bf16. */
typedef enum axo_type { AXO_TYPE_BF16 = 0, AXO_TYPE_F32 = 1 } axo_type_t;

/* Activation of the gate. */
typedef enum axo_gate {
    AXO_GATE_SILU = 0,      /* v / (1 + exp(-v))                                        */
    AXO_GATE_GELU_TANH = 1, /* 0.5 v (1 + tanh( sqrt(2/pi) (v + 0.044715 v^3) ))        */
    AXO_GATE_GELU_ERF = 2   /* 0.5 v (1 + erf( v / sqrt(2) ))                           */
} axo_gate_t;

/* ---- layer norm ------------------------------------------------------------------------------
 * p is the problem of the layer that reads the norm's output: rows of K values, T tokens; N is not used. */

/* S = X + R and Y[M x K] = (S - mean) * rstd * gamma + beta over each row of S, rstd = 1 / sqrt(variance + eps), the variance
 * that of the row (divided by K), formed from the row's deviations from its mean.
 * X, R, S: of `type` (axo_type_t).  R == NULL: S = X, and S is not written (pass NULL).  With R, S is required, is rounded to `type`
 * once, and the norm is that of the rounded values, which are what the backward pass sees.
 * gamma, beta: K bf16 values, or NULL for ones and zeros.  Y: bf16.  stats: M pairs of fp32 (mean, rstd) for the backward
 * pass, 8-byte aligned, or NULL.  eps >= 0 and finite.  K == 0: nothing is written.
 * Errors: those of axo_shard_dims; BAD_GRID (also for a K axis larger than 1); BAD_ARG (type, eps, shared bytes); NULL_PTR, BAD_LD, MISALIGNED; HIP.
 * Speed: one pass over the data for rows of up to 32768 bf16 or 24576 fp32 values. */
int axo_norm_fwd(const axo_problem_t *p, const void *X, int64_t ldx, const void *R, int64_t ldr, int type, const void *gamma,
                 const void *beta, float eps, void *S, int64_t lds, void *Y, int64_t ldy, float *stats, void *hip_stream);

/* The same for a K axis of any size, first half: S as above and, for each row, part[2 i] = the mean of this shard's Kl values and
 * part[2 i + 1] = the sum of their squared deviations from it.  Errors as axo_norm_fwd, without those of what it has not. */
int axo_norm_part(const axo_problem_t *p, const void *X, int64_t ldx, const void *R, int64_t ldr, int type, void *S, int64_t lds,
                  float *part, void *hip_stream);

/* Second half: parts holds the `part` arrays of the n_parts shards of the K axis one behind the other ([n_parts x M x 2], the same
 * on every shard; n_parts must be the axis's size, BAD_ARG otherwise).  S as axo_norm_part left it (or its X, where there was no R), gamma,
 * beta, Y: this shard's Kl columns.  The statistics written are those of the whole row. */
int axo_norm_apply(const axo_problem_t *p, const void *S, int64_t lds, int type, const float *parts, int n_parts, const void *gamma,
                   const void *beta, float eps, void *Y, int64_t ldy, float *stats, void *hip_stream);

/* Backward, with h = (S - mean) * rstd and g = dY * gamma:
 *   dX = R + rstd * (g - mean(g) - h * mean(g h))     means over the row;  R: a gradient to be added (the residual's), or NULL
 *   dgamma = sum over rows of dY * h,   dbeta = sum over rows of dY       (accumulate == 1: added to what is there)
 * S, R, dX: of `type`; dY bf16; stats as axo_norm_fwd wrote them.  dgamma, dbeta: K fp32 values, 4-byte aligned; either may be NULL and
 * is then not formed.  ws: axo_norm_workspace_bytes(p) bytes of device memory, 16-byte aligned, need not be initialised (may be NULL when that is
 * 0, and when dgamma and dbeta are NULL).  With M == 0 the sums are zero.
 * Errors: as axo_norm_fwd; BAD_ARG (accumulate not 0 or 1); WORKSPACE. */
int axo_norm_bwd(const axo_problem_t *p, const void *dY, int64_t lddy, const void *S, int64_t lds, const void *R, int64_t ldr, int type,
                 const void *gamma, const float *stats, void *dX, int64_t lddx, float *dgamma, float *dbeta, int accumulate,
                 void *ws, size_t ws_bytes, void *hip_stream);

/* The same for a K axis of any size, first half: sums[2 i] = sum of g, sums[2 i + 1] = sum of g h over this shard's columns of row i, and
 * dgamma, dbeta of its columns. */
int axo_norm_bwd_part(const axo_problem_t *p, const void *dY, int64_t lddy, const void *S, int64_t lds, int type, const void *gamma,
                      const float *stats, float *sums, float *dgamma, float *dbeta, int accumulate, void *ws, size_t ws_bytes,
                      void *hip_stream);

/* Second half: sums added up over the shards of the K axis; dX of this shard's columns. */
int axo_norm_bwd_apply(const axo_problem_t *p, const void *dY, int64_t lddy, const void *S, int64_t lds, const void *R, int64_t ldr, int type,
                       const void *gamma, const float *stats, const float *sums, void *dX, int64_t lddx, void *hip_stream);

/* Host only.  Bytes of device workspace that axo_norm_bwd and axo_norm_bwd_part need for this problem; 0 for an invalid one. */
size_t axo_norm_workspace_bytes(const axo_problem_t *p);

/* ---- gated feed-forward block ----------------------------------------------------------------
 * p is the problem of the block's two projections, K -> N each, in axo_gated_fwd, axo_gated_dgrad, axo_gated_wgrad and
 * axo_gated_wgrad_acc; in axo_gated_act, axo_gated_dact and axo_gated_dgrad_act it is that of the layer behind the block, whose K is
 * the projections' N.  Wg and Wu, G and U, dG and dU, dWg and dWu are matrices of their own with one leading dimension for each
 * pair; column blocks of one buffer do as well. */

/* G = X . Wg + bg, U = X . Wu + bu, H[M x Nl] = act(G) * U, `gate` an axo_gate_t.  H is formed from the unrounded sums.  G and U
 * (both or neither, ldz) are stored rounded to bf16 for the backward pass.  bg, bu: Nl bf16 values or NULL, each; added on shards whose coordinate on
 * the K axis is 0, as in axo_fc_fwd.  Kl == 0 gives act(bg) * bu.
 * ws: axo_gated_workspace_bytes(p) bytes of device memory, 16-byte aligned (may be NULL when that is 0).  It begins with arrival counters that must be
 * ZERO when the call starts executing and are zero again when it has finished: zero-fill the workspace once after allocating it and leave it to calls of the
 * gated entry points, which must not overlap in time on one workspace.
 * Errors: those of axo_shard_dims; BAD_EPILOGUE (gate); NULL_PTR (also G without U), BAD_LD, MISALIGNED; BAD_ARG (shared bytes); WORKSPACE; BAD_SIZE (over 8388480
 * rows in the general kernel, which takes empty reductions, operands whose spans pass 4 GiB and outputs of more 256 x 128 tiles than a launch takes, 8388607,
 * the columns of both projections counted); HIP; NO_MEMORY. */
int axo_gated_fwd(const axo_problem_t *p, const void *X, int64_t ldx, const void *Wg, const void *Wu, int64_t ldw, const void *bg,
                  const void *bu, int gate, void *G, void *U, int64_t ldz, void *H, int64_t ldh, void *ws, size_t ws_bytes,
                  void *hip_stream);

/* H[M x Kl] = act(G) * U, element by element, from bf16 G and U.  p: the layer that reads H.
 * Errors: as axo_gated_fwd, without WORKSPACE. */
int axo_gated_act(const axo_problem_t *p, const void *G, const void *U, int64_t ldz, int gate, void *H, int64_t ldh, void *hip_stream);

/* dG = dH * U * act'(G), dU = dH * act(G), element by element [M x Kl].  p: the layer that reads H. */
int axo_gated_dact(const axo_problem_t *p, const void *dH, int64_t lddh, const void *G, const void *U, int64_t ldz, int gate, void *dG,
                   void *dU, int64_t lddz, void *hip_stream);

/* The same with dH = dY[M x Nl] . W[Kl x Nl]^T, the data gradient of the layer that reads H (p, weights W), not rounded in between. */
int axo_gated_dgrad_act(const axo_problem_t *p, const void *dY, int64_t lddy, const void *W, int64_t ldw, const void *G, const void *U,
                        int64_t ldz, int gate, void *dG, void *dU, int64_t lddz, void *ws, size_t ws_bytes, void *hip_stream);

/* dX[M x Kl] = dG . Wg^T + dU . Wu^T, rounded once. */
int axo_gated_dgrad(const axo_problem_t *p, const void *dG, const void *dU, int64_t lddz, const void *Wg, const void *Wu, int64_t ldw,
                    void *dX, int64_t lddx, void *ws, size_t ws_bytes, void *hip_stream);

/* dWg[Kl x Nl] = X^T . dG and dWu = X^T . dU, rounded once.  The bits of two axo_fc_wgrad, but where workgroups share a tile's reduction (many tokens and few
 * outputs; axo_gated_tiles), which sum in another order, the same for every call. */
int axo_gated_wgrad(const axo_problem_t *p, const void *X, int64_t ldx, const void *dG, const void *dU, int64_t lddz, void *dWg, void *dWu,
                    int64_t lddw, void *ws, size_t ws_bytes, void *hip_stream);

/* The same added into fp32 matrices (lddw a multiple of 4), as axo_fc_wgrad_acc. */
int axo_gated_wgrad_acc(const axo_problem_t *p, const void *X, int64_t ldx, const void *dG, const void *dU, int64_t lddz, float *dWg,
                        float *dWu, int64_t lddw, void *ws, size_t ws_bytes, void *hip_stream);

/* Host only.  The largest workspace that any gated entry point needs when it is called with this problem; 0 for an invalid one. */
size_t axo_gated_workspace_bytes(const axo_problem_t *p);

/* The products of the block that have kernels of their own. */
typedef enum axo_gated_op { AXO_GATED_OP_FWD = 0, AXO_GATED_OP_DGRAD_ACT = 1, AXO_GATED_OP_DGRAD = 2, AXO_GATED_OP_WGRAD = 3 } axo_gated_op_t;

/* Host only.  How such a product is cut: rows and output columns of its tiles (of the largest, where there are two kinds), and the workgroups that share a
 * tile's reduction (1: one).  Rows of 16 and 32 are those of tiles whose waves split the reduction; 0 rows, with 0 columns and 0 slices: an empty output, or the
 * general kernel, which also takes operands whose spans pass 4 GiB, whatever is reported here.  For WGRAD 0 rows and columns and 1 slice: the tiles of
 * axo_fc_wgrad.  A function of the shard's sizes alone, chosen by estimated time, so
 * that the answer may change from one version to the next.  Errors: those of axo_shard_dims; BAD_ARG (op); NULL_PTR. */
int axo_gated_tiles(const axo_problem_t *p, int op, int *rows, int *cols, int *slices);

#ifdef __cplusplus
}
#endif
#endif /* AXO_BLOCK_H */
