/*
 * ones_train.h — C ABI of the training-step operators.
 *
 * The search (ones.h) needs a profiled step time for every job: seconds per iteration at each batch size (Eq. 5 and
 * the text after it).  These operators are the part of a language-model job's training step that depends on the batch
 * and is not a plain matrix product: layer norm, the cross entropy of a projection on a large vocabulary, both with
 * their gradients, and the orthogonalised update of a matrix parameter.  With them a job can be run, resized and
 * timed on the GPU that the search plans for.
 *
 * Conventions: those of ones.h.  Pointers named d_* are device memory of the current device; the caller owns every
 * buffer, the device workspace among them; nothing here allocates or frees device memory, prints or aborts.  All work
 * is enqueued on `cuda_stream` (a cudaStream_t, NULL = the default stream) and nothing synchronises, except
 * ones_train_status.  Arguments are checked before anything is launched, pointers for the alignment of their elements at
 * least (ONES_ERR_ALIGN).  Results do not depend on the order in which
 * blocks run: the same inputs give the same bits.  Rows are `ld` values apart, ld >= the row's length; values between
 * two rows are not written and do not matter, but where rows start on no 16-byte boundary they may be read along with
 * the 16-byte blocks around a row.  Nothing before a matrix's first value or after its last is read.
 */
#ifndef ONES_TRAIN_H
#define ONES_TRAIN_H
#include "ones.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define ONES_F32 0
#define ONES_BF16 1
#define ONES_F16 2

/* Layer norm over the last dimension:
 *   mean = sum_c x / cols,  rstd = 1 / sqrt(sum_c (x - mean)^2 / cols + eps),  y = (x - mean) * rstd * weight + bias.
 *   d_x, d_y        [rows][cols] of `type`;  d_weight, d_bias [cols] of `wtype`, each NULL for 1 and 0.
 *   d_mean, d_rstd  float[rows], for the backward pass; either may be NULL.
 * 0 <= rows <= ONES_NORM_MAX_ROWS, 1 <= cols <= ONES_NORM_MAX_COLS, eps > 0.  wtype is ONES_F32 or `type`.  Sums are in 32
 * bits. */
#define ONES_NORM_MAX_ROWS 0x7FFF0000 /* 2^31 - 2^16 */
#define ONES_NORM_MAX_COLS 65536
int ones_layer_norm(const void* d_x, int64_t ldx, const void* d_weight, const void* d_bias, int32_t rows, int32_t cols,
                    float eps, int32_t type, int32_t wtype, void* d_y, int64_t ldy, float* d_mean, float* d_rstd,
                    void* cuda_stream);

/* Its gradients: with xh = (x - mean) * rstd and g = dy * weight,
 *   dx = rstd * (g - sum_c g / cols - xh * sum_c (g * xh) / cols),   dweight = sum_rows dy * xh,   dbias = sum_rows dy.
 *   d_dx [rows][cols] of `type`; d_dweight, d_dbias [cols] of `wtype`, each may be NULL.
 *   d_workspace  at least ones_layer_norm_workspace_bytes(rows, cols) bytes, 256-byte aligned (not needed, and may be
 *   NULL, when both d_dweight and d_dbias are NULL).  rows = 0 gives dweight = dbias = 0. */
size_t ones_layer_norm_workspace_bytes(int32_t rows, int32_t cols);
int ones_layer_norm_backward(const void* d_dy, int64_t lddy, const void* d_x, int64_t ldx, const float* d_mean,
                             const float* d_rstd, const void* d_weight, int32_t rows, int32_t cols, int32_t type,
                             int32_t wtype, void* d_dx, int64_t lddx, void* d_dweight, void* d_dbias, void* d_workspace,
                             size_t workspace_bytes, void* cuda_stream);

/* Cross entropy of logits = hidden * weight^T without keeping the logits:
 *   lse[i] = log sum_v exp(logits[i][v]),   loss[i] = lse[i] - logits[i][target[i]].
 * A row whose target lies outside [0, vocab) takes no part: its loss is 0 (its lse is still written).
 *   d_hidden [rows][cols], d_weight [vocab][cols] of `type` (ONES_BF16 or ONES_F16), 16-byte aligned, ldh and ldw
 *   multiples of 8 (else ONES_ERR_ALIGN); d_target int64[rows]; d_loss, d_lse float[rows].
 *   rows >= 0, cols >= 1, vocab >= 1, each at most 2^30; any sizes otherwise.
 *   d_workspace  at least ones_linear_ce_workspace_bytes(rows, vocab) bytes, 256-byte aligned.
 * Logits are accumulated and reduced in 32 bits.  The tensor cores cut their sums off towards zero; what dense rows lose by
 * that in the mean, 2^-30 of a logit per column, is given back for up to 4096 columns, whatever the row: a logit that comes
 * from few columns is too large by up to 2^-18 of itself then, and dense rows of more columns are too small by the rest. */
size_t ones_linear_ce_workspace_bytes(int32_t rows, int32_t vocab);
/* Copies rows that start anywhere to rows on 16-byte boundaries, as ones_linear_ce needs them: d_dst 16-byte aligned, ldd
 * a multiple of 8, both [rows][cols] of ONES_BF16 or ONES_F16.  Zeros follow each row up to the next multiple of 8. */
int ones_align_rows(const void* d_src, int64_t lds, int32_t rows, int32_t cols, int32_t type, void* d_dst, int64_t ldd,
                    void* cuda_stream);
int ones_linear_ce(const void* d_hidden, int64_t ldh, const void* d_weight, int64_t ldw, const int64_t* d_target,
                   int32_t rows, int32_t cols, int32_t vocab, int32_t type, float* d_loss, float* d_lse,
                   void* d_workspace, size_t workspace_bytes, void* cuda_stream);

/* Its gradients for the gradient d_dloss float[rows] of the loss and the lse of the forward call:
 *   dlogits[i][v] = (exp(logits[i][v] - lse[i]) - [v == target[i]]) * dloss[i]   (0 in rows that take no part),
 *   dhidden = dlogits * weight,   dweight = dlogits^T * hidden.
 * Rows that take no part cost next to nothing: the others are gathered first, so nothing of them, not even a NaN in
 * hidden, reaches dweight.  The vocabulary is taken in pieces of `piece` entries (a multiple of 256; 0: a default that keeps the piece's
 * gradient near 256 MiB): the logits of a piece are computed again, and their gradient is kept in the workspace, as
 * 16 bits of `type` scaled so that the largest |dloss| is 1, or 2^15 for ONES_F16 (with up to 64 rows as two such terms, the
 * second what the rounding of the first left), until both products have used it.  ONES_F16 holds it in
 * steps of 2^-39 of the largest |dloss| where those are larger than its 11 bits.
 *   d_dhidden [rows][cols] of `type`; d_dweight [vocab][cols] of `wtype` (`type` or ONES_F32), any alignment of their
 *   elements (16-byte aligned rows are written faster), hidden too; weight aligned as above.
 *   d_workspace  at least ones_linear_ce_backward_workspace_bytes(rows, cols, vocab, piece) bytes. */
size_t ones_linear_ce_backward_workspace_bytes(int32_t rows, int32_t cols, int32_t vocab, int32_t piece);
int ones_linear_ce_backward(const float* d_dloss, const void* d_hidden, int64_t ldh, const void* d_weight, int64_t ldw,
                            const int64_t* d_target, const float* d_lse, int32_t rows, int32_t cols, int32_t vocab,
                            int32_t type, int32_t wtype, int32_t piece, void* d_dhidden, int64_t lddh, void* d_dweight,
                            int64_t lddw, void* d_workspace, size_t workspace_bytes, void* cuda_stream);

/* Orthogonalised update of `count` matrices [m][n], one every `stride` values, by Newton-Schulz products:
 *   X = G / (|G|_F + eps);   `steps` times:  A = X X^T,  X <- (a I + b A + c A^2) X      (on the shorter side)
 * which moves every singular value of G towards 1 (for the usual coefficients a, b, c: into about [0.7, 1.2]).
 *   d_g of `type` (any of the three), any alignment of its elements; d_out [count][m][n] of bfloat16, rows n apart.
 *   1 <= steps <= ONES_UPDATE_MAX_STEPS (one launch runs them all), eps > 0, finite coefficients, sizes >= 1;
 *   count <= 65535, m and n <= 2^20.
 * Products run on 16-bit operands (11 significant bits, scaled into range, also where |G| is down to 2^-50 of eps) with
 * 32-bit accumulators; the norm is summed in 64 bits.
 *   d_workspace  at least ones_orthogonalize_workspace_bytes(count, m, n) bytes, 256-byte aligned. */
#define ONES_UPDATE_MAX_STEPS 1024
size_t ones_orthogonalize_workspace_bytes(int32_t count, int32_t m, int32_t n);
int ones_orthogonalize(const void* d_g, int64_t ldg, int64_t stride, int32_t count, int32_t m, int32_t n, int32_t type,
                       int32_t steps, float a, float b, float c, float eps, void* d_out, void* d_workspace,
                       size_t workspace_bytes, void* cuda_stream);

/* Synchronises `cuda_stream` and says whether every wait inside the kernels above ended as it should since the last
 * call on this device: ONES_OK, ONES_ERR_TIMEOUT (a kernel gave up waiting; its results are void) or ONES_ERR_CUDA. */
int ones_train_status(void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif
