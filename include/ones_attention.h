/*
 * ones_attention.h — C ABI of the operators that a transformer job's training step adds to those of ones_train.h.
 *
 * Norms of queries and keys with the rotation of their positions, causal attention over packed sequences with grouped
 * heads, both with their gradients, and the norm and the clipping of all gradients.  With them a job with attention can be
 * run, resized and timed on the GPU that the search plans for (profile_job.py).
 *
 * Conventions: those of ones_train.h; ones_train_status covers these kernels too.
 */
#ifndef ONES_ATTENTION_H
#define ONES_ATTENTION_H
#include "ones_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Vectors of `dim` values, one for each token and head: value c of head h of token t lies at
 * d_data[t * token + h * head + c].  head >= dim where there are several heads, and token >= 0 where there are several
 * tokens.  Outputs overlap neither one another nor an input, except where an operator says so. */
typedef struct ones_heads {
    void* d_data;
    int64_t token, head; /* strides in values */
    int32_t heads;
} ones_heads;

/* Root-mean-square norm of every query and key vector and the rotation of its position, in one pass:
 *   r = 1 / sqrt(sum_c x_c^2 / dim + eps),  n_c = x_c r weight_c,  y = n turned by its token's angles:
 *   pair i of the first `rotary` values turns by positions[t] * frequencies[i], i < rotary / 2; the values of a pair are
 *   i and i + rotary / 2, or 2 i and 2 i + 1 where `interleaved`; values from `rotary` on stay as they are.
 *   q, k, q_out, k_out  of `type`; the outputs may be the inputs (same strides).  Sides with heads = 0 are left out.
 *   d_positions int64[tokens], d_frequencies double[rotary / 2] (radians for one step of the position): the angle is
 *   formed and reduced to one turn in 64 bits.
 *   d_q_weight, d_k_weight  [dim] of `wtype`, each NULL for 1.
 * 0 <= tokens < 2^31, 1 <= dim <= ONES_QK_NORM_MAX_DIM, rotary even, 0 <= rotary <= dim, heads <= ONES_MAX_HEADS, eps >= 0.
 * wtype is ONES_F32 or `type`.  Sums are in 32 bits, of values times a power of two where their squares leave that range. */
#define ONES_QK_NORM_MAX_DIM 256
#define ONES_MAX_HEADS 1024
int ones_qk_norm(const ones_heads* q, const ones_heads* k, const int64_t* d_positions, const double* d_frequencies,
                 const void* d_q_weight, const void* d_k_weight, int32_t tokens, int32_t dim, int32_t rotary,
                 int32_t interleaved, float eps, int32_t type, int32_t wtype, const ones_heads* q_out,
                 const ones_heads* k_out, void* cuda_stream);

/* Its gradients: g = dy turned back,
 *   dx_c = r (g_c weight_c - x_c r^2 sum_e (g_e weight_e x_e) / dim),   dweight_c = sum_{tokens, heads} g_c x_c r.
 *   dq, dk (in) and q, k as in the forward call; dq_out, dk_out may be dq, dk.  d_dq_weight, d_dk_weight [dim] of `wtype`,
 *   each may be NULL; tokens = 0 gives 0 there.
 *   d_workspace  at least ones_qk_norm_workspace_bytes(dim) bytes, 256-byte aligned (may be NULL when both are NULL). */
size_t ones_qk_norm_workspace_bytes(int32_t dim);
int ones_qk_norm_backward(const ones_heads* dq, const ones_heads* dk, const ones_heads* q, const ones_heads* k,
                          const int64_t* d_positions, const double* d_frequencies, const void* d_q_weight,
                          const void* d_k_weight, int32_t tokens, int32_t dim, int32_t rotary, int32_t interleaved,
                          float eps, int32_t type, int32_t wtype, const ones_heads* dq_out, const ones_heads* dk_out,
                          void* d_dq_weight, void* d_dk_weight, void* d_workspace, size_t workspace_bytes,
                          void* cuda_stream);

/* Causal attention of packed sequences, query heads in groups that share a key and value head (head h reads head
 * h / (q->heads / k->heads)):
 *   s_ij = scale q_i . k_j for tokens j <= i of one sequence,  lse_i = log sum_j exp s_ij,  out_i = sum_j exp(s_ij - lse_i) v_j.
 *   q, out  `heads` heads; k, v  `kv` heads each, heads a multiple of kv, heads / kv <= 128; of `type` (ONES_BF16 or ONES_F16).
 *   q, k, v 16-byte aligned, strides multiples of 8 (else ONES_ERR_ALIGN); out any alignment of its elements.
 *   d_offsets int64[sequences + 1]: sequence n is tokens [d_offsets[n], d_offsets[n + 1]), read on the device.  NULL: all
 *   `sequences` are tokens / sequences long.  Offsets outside [0, tokens] count as its ends, and one below those before it
 *   as the largest of them.  Tokens of no sequence get out = 0, lse = 0, and nothing of them, not even a NaN, reaches others.
 *   Nothing of one sequence reaches another either.  Within a sequence, what is not finite in k or v of a token (backward: in
 *   q, k, v or dout) may also reach earlier tokens of the same 128 keys, or tokens of the same 128 rows of queries: hidden
 *   scores count as products with 0, as in a plain matrix product.
 *   d_lse float[tokens][heads].
 * Scores are in 32 bits before the factor: what does not fit is an infinity. Keys that score -infinity have no part in their row; a
 * row whose keys all do has lse = -infinity and out = NaN (and its gradients, and those of its keys, are NaN).
 * 0 <= tokens < 2^30, 0 <= sequences <= 2^22, 1 <= dim <= ONES_ATTENTION_MAX_DIM, scale > 0 and finite; tiles of
 * queries (128 / (heads / kv) tokens of a sequence each, rounded down) times kv have to be below 2^31 (ONES_ERR_BAD_PARAM).
 *   d_workspace  at least ones_attention_workspace_bytes(tokens, sequences, heads, kv) bytes, 256-byte aligned.
 * Scores, their statistics and all sums are in 32 bits; the probabilities are rounded to `type` for the product with v (ONES_F16: in steps of
 * 2^-31 of the row's largest at most). */
#define ONES_ATTENTION_MAX_DIM 128
size_t ones_attention_workspace_bytes(int32_t tokens, int32_t sequences, int32_t heads, int32_t kv);
int ones_attention(const ones_heads* q, const ones_heads* k, const ones_heads* v, const int64_t* d_offsets,
                   int32_t tokens, int32_t sequences, int32_t dim, float scale, int32_t type, const ones_heads* out,
                   float* d_lse, void* d_workspace, size_t workspace_bytes, void* cuda_stream);

/* Its gradients for the gradient dout of out, with p_ij = exp(s_ij - lse_i):
 *   dp_ij = dout_i . v_j,  ds_ij = p_ij (dp_ij - dout_i . out_i),
 *   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij dout_i   (i over the heads of the group).
 *   dout aligned as q; out and d_lse what the forward call gave; dq, dk, dv any alignment of their elements.  Tokens of no
 *   sequence get gradients of 0.
 *   d_workspace  at least ones_attention_backward_workspace_bytes(tokens, sequences, heads, kv, dim) bytes.
 * p and ds are rounded to `type` for their products, ONES_F16 times a power of two (p 2^12, ds what follows from the largest |dout| of its
 * row for dq, of the sequence and group of heads for dk, and the largest |v| of these): ds keeps 11 bits down to 2^-21 of their product, and
 * steps of 2^-31 of it below.  A row whose |lse| is 2^24 or more and finite, which has only seen keys that a mask's lowest value
 * hides, has p = 0. */
size_t ones_attention_backward_workspace_bytes(int32_t tokens, int32_t sequences, int32_t heads, int32_t kv, int32_t dim);
int ones_attention_backward(const ones_heads* dout, const ones_heads* q, const ones_heads* k, const ones_heads* v,
                            const ones_heads* out, const float* d_lse, const int64_t* d_offsets, int32_t tokens,
                            int32_t sequences, int32_t dim, float scale, int32_t type, const ones_heads* dq,
                            const ones_heads* dk, const ones_heads* dv, void* d_workspace, size_t workspace_bytes,
                            void* cuda_stream);

/* Euclidean norm of all values of `count` tensors together, and the tensors scaled down to a norm of at most max_norm:
 *   norm = sqrt(sum g^2),   out = g * min(1, max_norm / (norm + eps))    (a NaN of the norm reaches every value).
 *   d_g, d_out  host arrays of `count` device pointers; size, type  host arrays: values of each tensor and their type (any of
 *   the three; out has the type of g).  d_out may be d_g, or hold single tensors of it: where the factor is 1 such tensors are
 *   not touched.  Otherwise tensors must not overlap.  d_norm float[1].
 * 0 <= count <= 2^20, size >= 0, at most 2^44 bytes together; max_norm and eps finite and >= 0.  Squares are summed in 32 bits
 * for 32 values at most, then in 64.
 *   d_workspace  at least ones_gradient_norm_workspace_bytes(count) bytes, 256-byte aligned. */
size_t ones_gradient_norm_workspace_bytes(int32_t count);
int ones_gradient_norm(const void* const* d_g, const int64_t* size, const int32_t* type, int32_t count, float* d_norm,
                       void* d_workspace, size_t workspace_bytes, void* cuda_stream);
int ones_clip_gradients(const void* const* d_g, void* const* d_out, const int64_t* size, const int32_t* type, int32_t count,
                        double max_norm, double eps, float* d_norm, void* d_workspace, size_t workspace_bytes,
                        void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif
