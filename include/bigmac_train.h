/*
 * bigmac_train.h -- C-ABI of the operators at the two ends of a training step around the blocks of
 * bigmac_block.h: token ids become the rows that the first block reads, the last block's logits
 * become a loss and its gradient, and a weight's accumulated gradient becomes an update.
 *
 *   bm_embedding_forward    y[t] = scale * table[id[t]]                            (text rows of embed_preprocess,
 *   bm_embedding_backward   dtable[v] += scale * sum over t with id[t] = v of dy[t]   Sec. 3.2 "Module handoff")
 *   bm_cross_entropy        loss[t] = w[t] (log sum_v exp z[t,v] - z[t,label[t]]) and its gradient
 *   bm_orthogonalize        Newton-Schulz: the nearest (semi-)orthogonal matrix of a gradient, roughly
 *
 * Conventions of bigmac_block.h: caller-owned device buffers, 16-byte aligned pointers, row-major
 * tensors, work on the given stream without host synchronisation, error codes, dtype BM_DTYPE_BF16 or
 * BM_DTYPE_FP32 for activations and parameters, fp32 for gradients of parameters, which are ADDED to.
 * Leading dimensions are in elements and free of alignment rules, but rows of whole 16 bytes are
 * faster.  No call uses floating-point atomics: the same arguments give the same bits.
 * Buffers do not overlap unless said otherwise.  Calls that share a workspace follow one another on a
 * stream; captured graphs that may replay at the same time have workspaces of their own.
 */
#ifndef BIGMAC_TRAIN_H
#define BIGMAC_TRAIN_H

#include "bigmac_block.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- token embeddings ---------------------------------------------------------------
 *   V, d       rows and columns of the table
 *   table dev  [V, ld_table >= d]  storage dtype
 *   ids   dev  [T] int32.  Negative: the row is no text token (an image row, padding): its y is left
 *              as it was, its dy is not read.  An id of V or more is the caller's mistake: its y is
 *              NaN, its dy is not read.
 *   y, dy dev  [T, ld >= d]  storage dtype
 * T may be 0 (nothing is done, and pointers may be NULL).  T and d are 2^30 at most. */
bm_status bm_embedding_forward(int32_t dtype, int32_t V, int32_t d, const void* table, int32_t ld_table,
                               const int32_t* ids, int32_t T, float scale, void* y, int32_t ld_y,
                               void* hip_stream);

/* dtable dev [V, ld_dtable >= d] fp32; rows of words that do not occur are neither read nor written.
 * The rows of a word are summed in fp32 in an order that depends on T, d and the ids alone.
 * scratch: bm_embedding_backward_scratch_bytes(T, d) bytes (0 for sizes that are refused). */
size_t    bm_embedding_backward_scratch_bytes(int32_t T, int32_t d);
bm_status bm_embedding_backward(int32_t dtype, int32_t V, int32_t d, const void* dy, int32_t ld_dy,
                                const int32_t* ids, int32_t T, float scale, float* dtable, int32_t ld_dtable,
                                void* scratch, size_t scratch_bytes, void* hip_stream);

/* ---- cross-entropy of a vocabulary, with its gradient ----------------------------------
 *   logits  dev [T, ld >= V]  storage dtype
 *   labels  dev [T] int32.  Negative: the row is ignored -- loss 0, gradient 0, whatever its logits
 *               hold (they are not read).  V or more: loss and gradient are NaN.
 *   weight  dev [T] fp32 factor of every row's loss and gradient (1 / rows of the batch, say), NULL: 1
 *   loss    dev [T] fp32, or NULL
 *   dlogits dev [T, ld_d >= V] storage dtype, or NULL:  w (softmax(z) - onehot(label)).
 *               May be logits itself with ld_d == ld.  Not both loss and dlogits are NULL.
 * Logits of -inf (masked words) have probability and gradient 0; a row of nothing else, or one that
 * holds +inf or NaN, gives NaN.  Statistics are fp32; a gradient is rounded once.
 * scratch: bm_cross_entropy_scratch_bytes(dtype, T, V) bytes (NULL where that is 0).  T may be 0. */
size_t    bm_cross_entropy_scratch_bytes(int32_t dtype, int32_t T, int32_t V);
bm_status bm_cross_entropy(int32_t dtype, int32_t T, int32_t V, const void* logits, int32_t ld,
                           const int32_t* labels, const float* weight, float* loss, void* dlogits, int32_t ld_d,
                           void* scratch, size_t scratch_bytes, void* hip_stream);

/* ---- orthogonalised update ----------------------------------------------------------------
 * For every matrix b of a batch, with G_b [M, N] and m = min(M, N):
 *   X = G_b / (|G_b|_F + eps),  then `steps` times  X <- a X + (b A + c A^2) X  with A = X X^T
 *   (X^T X for a matrix that is taller than wide), and O_b = X.
 * The iteration moves every singular value of G_b towards the fixed points of
 * a s + b s^3 + c s^5; with (3.4445, -4.7750, 2.0315) and 5 steps all but the smallest end between 0.7 and 1.2.
 *   grad dev  fp32, matrix b at grad + b*stride_g, rows of ld_g >= N elements
 *   out  dev  dtype, matrix b at out + b*stride_o, rows of ld_o >= N elements; overwritten
 *   coefficients host [3]: a, b, c.  steps 1..64.  eps >= 0; with eps = 0 a matrix of zeros gives NaN.
 * Strides are in elements and not negative; stride_g may be 0; matrices of `out` lie one behind the other or side by
 * side.  out may be grad itself with the same strides (BM_DTYPE_FP32); otherwise the memory from the first to the last element of
 * the one and that of the other do not overlap.
 * The products run on the matrix cores.  For BM_DTYPE_BF16 their operands are 11-bit significands (fp16, scaled); X itself is kept
 * in 22 bits until the last two steps, in which only singular values near the fixed points are still moved, and up to 128
 * rows or columns so are A and B, up to 32 all of them.  For BM_DTYPE_FP32 everything has 22 bits.  Sums are fp32, the norm fp64.
 * BM_ERR_UNSUPPORTED for coefficients under which a singular value of [0, 1] exceeds 8 within `steps` steps.
 * A matrix that holds an infinity or a NaN gives NaN; other matrices of the batch are not affected.
 * scratch: bm_orthogonalize_scratch_bytes(dtype, batch, M, N) bytes.  batch may be 0. */
size_t    bm_orthogonalize_scratch_bytes(int32_t dtype, int32_t batch, int32_t M, int32_t N);
bm_status bm_orthogonalize(int32_t dtype, int32_t batch, int32_t M, int32_t N, const float* grad, int32_t ld_g,
                           int64_t stride_g, void* out, int32_t ld_o, int64_t stride_o, const float* coefficients,
                           int32_t steps, float eps, void* scratch, size_t scratch_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
