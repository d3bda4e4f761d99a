/*
 * axo_residual.h -- C ABI of what writes a sublayer's output into the residual stream on MI355X (gfx950): the product that adds to it, and the norms either side
 * of the addition with its gate and scale, forward and backward.
 *
 *   s = r + scale act(h W + b)                           axo_fc_add        (the sublayer's last layer)
 *   s = x + scale gate norm_a(y),  n = norm_b(s)         axo_resnorm_fwd   (behind it, and ahead of the next sublayer)
 *
 * and back: axo_resnorm_bwd takes the gradients of n and s to those of x and y, axo_fc_add_dact gives the gradient behind the bias, which axo_fc_dgrad, axo_fc_wgrad and
 * axo_bias_grad read.
 *
 * Problems, shards, data, ownership, checks and arithmetic are those of axo_block.h: no output may share a byte with an input or with another output of the same
 * call (AXO_ERR_BAD_ARG), statistics, sums and activations are fp32, every bf16 result is rounded once, results are a fixed function of the inputs.
 */
#ifndef AXO_RESIDUAL_H
#define AXO_RESIDUAL_H

#include "axo_block.h" /* axo_type_t */

#ifdef __cplusplus
extern "C" {
#endif

/* ---- product with a residual -------------------------------------------------------------------
 * p is the problem of the layer, K -> N.  The residual R and the output Y are the residual stream, of `type` (axo_type_t). */

/* Y[M x Nl] = R + scale * act(X . W + bias), `epilogue` an axo_epilogue_t (AXO_EPI_NONE: no bias, AXO_EPI_BIAS: no activation), formed from the unrounded sum and
 * rounded to `type` once.  Z, or NULL: the pre-activation X . W + bias rounded to bf16, which axo_fc_add_dact reads; only with an activation.
 * On a grid that splits K, R and bias are added on shards whose coordinate on the K axis is 0 and are not read on the others (R may be NULL there), so that the sum over
 * that axis adds them once; an activation belongs behind that sum, and its epilogues take grids whose K axis has size 1 (BAD_GRID).  Kl == 0 gives R + scale * act(bias).
 * ws: axo_fc_add_workspace_bytes(p) bytes of device memory, 16-byte aligned (may be NULL when that is 0).  It begins with arrival counters: zero-fill it once after
 * allocating it and leave it to calls of axo_fc_add, which must not overlap in time on one workspace.
 * Errors: those of axo_shard_dims; BAD_EPILOGUE (unknown, or one with bias == NULL); BAD_ARG (type, scale not finite, Z without an activation, shared bytes); BAD_GRID;
 * NULL_PTR, BAD_LD, MISALIGNED; WORKSPACE; BAD_SIZE as axo_gated_fwd; HIP; NO_MEMORY. */
int axo_fc_add(const axo_problem_t *p, const void *X, int64_t ldx, const void *W, int64_t ldw, const void *bias, int epilogue, const void *R, int64_t ldr,
               int type, float scale, void *Z, int64_t ldz, void *Y, int64_t ldy, void *ws, size_t ws_bytes, void *hip_stream);

/* dZ[M x Nl] = scale * dY * act'(Z), element by element, rounded to bf16: from the gradient of Y, of `type`, to what axo_fc_dgrad, axo_fc_wgrad and axo_bias_grad take.
 * (The gradient of R is dY itself.)  Without an activation Z is NULL and dZ = scale * dY.  Errors as axo_fc_add, without WORKSPACE. */
int axo_fc_add_dact(const axo_problem_t *p, const void *dY, int64_t lddy, int type, const void *Z, int64_t ldz, int epilogue, float scale, void *dZ,
                    int64_t lddz, void *hip_stream);

/* Host only.  Bytes of device workspace that axo_fc_add needs for this problem; 0 for an invalid one. */
size_t axo_fc_add_workspace_bytes(const axo_problem_t *p);

/* ---- norms either side of a residual addition --------------------------------------------------------
 * p is the problem of the layer that reads Y: rows of K values, T tokens; N is not used.  The grid's K axis has size 1 (BAD_GRID otherwise): both norms need whole rows.
 * The residual stream (X, S, dS, dX) is of `type` (axo_type_t), everything else bf16 but for statistics and the gradients of vectors, which are fp32. */

/* What a norm divides by, with d = v (rms) or v - mean(v) (layer):  1 / sqrt(mean(d^2) + eps). */
typedef enum axo_norm {
    AXO_NORM_NONE = 0,  /* z = v gamma + beta                                                  */
    AXO_NORM_LAYER = 1, /* z = (v - mean) rstd gamma + beta                                    */
    AXO_NORM_RMS = 2    /* z = v rstd gamma + beta                                             */
} axo_norm_t;

/* S[M x K] = X + scale * gate * norm_a(B), rounded to `type` once, and Y[M x K] = norm_b(S) of the rounded values.
 * B: a block's output.  norm_a an axo_norm_t, norm_b AXO_NORM_LAYER or AXO_NORM_RMS.  gamma_a, beta_a, gate, gamma_b, beta_b: K bf16 values each, or NULL for ones, zeros, ones,
 * ones and zeros.  stats: M times (mean_a, rstd_a, mean_b, rstd_b) in fp32 for the backward pass, 16-byte aligned, or NULL; a mean that a norm has not is 0, a
 * rstd 1.  eps >= 0 and finite.  K == 0: nothing is written.
 * Errors: those of axo_shard_dims; BAD_GRID; BAD_ARG (type, norms, scale or eps, shared bytes); NULL_PTR, BAD_LD, MISALIGNED; HIP.
 * Speed: one pass over the data for rows of up to 16384 values, forward and backward. */
int axo_resnorm_fwd(const axo_problem_t *p, const void *B, int64_t ldb, const void *X, int64_t ldx, int type, int norm_a, const void *gamma_a, const void *beta_a,
                    const void *gate, float scale, int norm_b, const void *gamma_b, const void *beta_b, float eps, void *S, int64_t lds, void *Y, int64_t ldy,
                    float *stats, void *hip_stream);

/* Backward, from dY and from dS, the gradient that reaches S from behind (NULL: none):
 *   dX = dS + the gradient of S through norm_b;  dB = the gradient of B through norm_a, gate and scale, from the unrounded dX
 *   dgamma_a, dbeta_a, dgate, dgamma_b, dbeta_b: K fp32 values each, 4-byte aligned (accumulate == 1: added to what is there); any may be NULL and is not formed then.
 * B, S, stats: as axo_resnorm_fwd read and left them.  ws: axo_resnorm_workspace_bytes(p) bytes of device memory, 16-byte aligned, need not be initialised (may be
 * NULL when none of the five is formed).  With M == 0 the sums are zero.
 * Errors: as axo_resnorm_fwd; BAD_ARG (accumulate not 0 or 1); WORKSPACE. */
int axo_resnorm_bwd(const axo_problem_t *p, const void *dY, int64_t lddy, const void *dS, int64_t ldds, const void *B, int64_t ldb, const void *S, int64_t lds,
                    int type, int norm_a, const void *gamma_a, const void *beta_a, const void *gate, float scale, int norm_b, const void *gamma_b,
                    const float *stats, void *dX, int64_t lddx, void *dB, int64_t lddb, float *dgamma_a, float *dbeta_a, float *dgate, float *dgamma_b,
                    float *dbeta_b, int accumulate, void *ws, size_t ws_bytes, void *hip_stream);

/* Host only.  Bytes of device workspace that axo_resnorm_bwd needs for this problem; 0 for one that it refuses. */
size_t axo_resnorm_workspace_bytes(const axo_problem_t *p);

#ifdef __cplusplus
}
#endif
#endif /* AXO_RESIDUAL_H */
