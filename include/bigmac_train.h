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
 * T may be 0 (nothing is done, and pointers may be NULL). */
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

#ifdef __cplusplus
}
#endif
#endif
