/*
 * bigmac_window_attention.h -- C-ABI of what stands around the attention of a block whose tokens have
 * positions on several axes and see only a part of what lies before them:
 *
 *   bm_qk_rotary_forward / _backward         queries and keys turned by their positions (time, row, column),
 *                                            with the RMS norm of every head in the same pass or without
 *   bm_window_attention_forward / _backward  attention to the last `window` tokens and to a few first ones
 *
 * Used one after the other: packed q|k|v rows of a projection -> bm_qk_rotary_forward in place (or into rows
 * of their own, where the norm's backward needs the rows before it) -> bm_window_attention_forward.
 *
 * Conventions of bigmac_block.h: caller-owned device buffers, 16-byte aligned pointers, row-major
 * token-major tensors, work on the given stream without host synchronisation, error codes, dtype
 * BM_DTYPE_BF16 or BM_DTYPE_FP32 for activations and gains, fp32 for gradients of gains, which are ADDED
 * to.  Row strides are in elements and whole multiples of 16 bytes.  No call uses floating-point atomics:
 * the same arguments give the same bits.  Buffers do not overlap unless said otherwise.  Calls that share a
 * workspace follow one another on a stream; captured graphs that may replay at the same time have
 * workspaces of their own.
 */
#ifndef BIGMAC_WINDOW_ATTENTION_H
#define BIGMAC_WINDOW_ATTENTION_H

#include "bigmac_block.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotation of queries and keys over several axes, with the norm of every head ----------
 * For every token t and head (rows of n_q_heads query heads and n_kv_heads key heads):
 *   y = x                                          norm = 0
 *   y = x / sqrt(mean(x^2) + eps) * gain           norm = 1, gain [head_dim] of the queries or of the keys
 *   z[i]      = y[i] cos a - y[i + h] sin a        h = head_dim / 2, i < h
 *   z[i + h]  = y[i + h] cos a + y[i] sin a
 *   a = positions[axis(i)][t] * base^(-2 i / head_dim)      own_frequencies = 0
 *                             * base^(-j / pairs[axis(i)])  own_frequencies = 1, pair i the j-th of its axis
 * The first pairs[0] pairs belong to axis 0, the next pairs[1] to axis 1, and so on; together they are
 * head_dim / 2 (an axis may have none; an axis whose positions are all 0 leaves its pairs as they are).
 * With one axis of head_dim / 2 pairs and positions that count up in every sequence this is the rotation
 * that a block with rope = 1 makes.  Angles are formed and reduced in fp64, off by at most 2^-50 of the position
 * for bases of 1 and more: 2^-24 at position 2^26.  Squares are summed in fp32. */
#define BM_ROTARY_MAX_AXES 4
typedef struct {
  int32_t dtype, n_q_heads, n_kv_heads, head_dim;  /* head_dim: a multiple of 8 up to 256; one of the head counts may be 0 */
  int32_t n_axes, pairs[BM_ROTARY_MAX_AXES];       /* 1..4 axes                                          */
  int32_t own_frequencies;                         /* 0/1                                                */
  float   base;                                    /* > 0                                                */
  int32_t norm;                                    /* 0/1                                                */
  float   eps;                                     /* >= 0; with 0 a head of zeros gives NaN             */
} bm_qk_rotary_desc;

/*   q, k           dev  rows of ld elements: n_q_heads*head_dim and n_kv_heads*head_dim from either pointer on
 *   positions      dev  [n_axes, T] int32, any values
 *   q_gain, k_gain dev  [head_dim] storage dtype (norm = 1, else NULL)
 *   q_out, k_out   dev  rows of ld_out elements; may be q and k themselves with ld_out == ld
 * Pointers that belong to no head are NULL or not read.  T may be 0 (nothing is done). */
bm_status bm_qk_rotary_forward(const bm_qk_rotary_desc* desc, int32_t T, const void* q, const void* k, int32_t ld,
                               const int32_t* positions, const void* q_gain, const void* k_gain, void* q_out,
                               void* k_out, int32_t ld_out, void* hip_stream);

/*   q, k             as given to the forward call: rows BEFORE norm and rotation (norm = 1; not read, and may be
 *                    NULL, without)
 *   dq_out, dk_out   dev  gradients of q_out and k_out, rows of ld_dout elements
 *   dq, dk           dev  gradients of q and k, rows of ld_dqk elements, overwritten; may take the place of dq_out
 *                         and dk_out, or of q and k, in rows of the same stride
 *   dq_gain, dk_gain dev  [head_dim] fp32, added to (norm = 1); may be one buffer where both share a gain
 * scratch: bm_qk_rotary_backward_scratch_bytes(desc, T) bytes (0 without norm), the same for every T. */
size_t    bm_qk_rotary_backward_scratch_bytes(const bm_qk_rotary_desc* desc, int32_t T);
bm_status bm_qk_rotary_backward(const bm_qk_rotary_desc* desc, int32_t T, const void* q, const void* k, int32_t ld,
                                const int32_t* positions, const void* q_gain, const void* k_gain,
                                const void* dq_out, const void* dk_out, int32_t ld_dout, void* dq, void* dk,
                                int32_t ld_dqk, float* dq_gain, float* dk_gain, void* scratch,
                                size_t scratch_bytes, void* hip_stream);

/* ---- attention with a sliding window and first tokens that stay visible ------------------
 * Query i of a sequence with Lq queries and Lk keys stands at position p = Lk - Lq + i: the queries are the
 * sequence's last Lq tokens (all of them in training, one when tokens are generated one by one).  It sees
 * key j where j <= p and (p - j < window or j < sinks); window >= 1, so every query sees its own key.
 *     o = softmax(q k^T / sqrt(dh)) v,   lse = log sum exp of the scaled scores
 *   sinks            0..BM_WINDOW_MAX_SINKS
 *   q         dev    rows of ld_q elements, Hq heads of dh, sequences one behind the other by cu_q [S+1]
 *   k, v      dev    rows of ld_kv elements, Hkv heads; sequence s holds rows k_begin[s] .. k_end[s]-1.  The four
 *                    arrays are NULL where keys have the queries' packing.  Rows may lie between the sequences
 *                    (slots of a cache), which are neither read nor written.  The forward pass takes sequences in
 *                    any order, and ones that share rows (a common beginning); the backward pass takes them one
 *                    behind the other
 *   cu_q, k_begin, k_end are given twice, in device and in host memory, with the same values
 *   o, d_o    dev    [Tq, Hq*dh], lse dev [Hq, Tq] fp32, Tq = cu_q[S]
 * Limits: S < 65536, Hq < 65536, Tq x Hq and Tk x Hkv below 2^26, S x Hq below 2^22, row strides below 2^24.
 * The backward pass in bf16 at head size 128 refuses packs that come to 2^23 workgroups, one for each 128 keys and
 * each 256 queries of a head, which takes S x Hq of 2^21 and more.
 * Lq <= Lk for every sequence; Lq = 0 is allowed (its dk, dv are 0), and so is Lk = 0 with it.
 * The forward pass does not read keys and values that no query of the call sees: they may be anything.  A key or
 * value that some queries see and others do not has weight 0 for the latter and is finite, in the backward pass all
 * of them are.
 * dh is 8, 16, 32, 64, 72 or 128; q head a uses kv head a / (Hq/Hkv).  bf16 with head sizes 64, 72 and 128 runs on
 * the matrix cores: probabilities, and dS in the backward pass, are rounded to bf16 before the products that they
 * enter.  Everything else is fp32 arithmetic.
 * Where every sequence of a call has Lq x (Hq/Hkv) <= 32, the keys are split over the chip and the parts joined in a
 * fixed order.  One sequence with more sends all of the call through tiles of 128 queries (16 in fp32 arithmetic), in
 * which a workgroup walks all the keys that its queries see: chunks of queries and single ones take separate calls. */
#define BM_WINDOW_MAX_SINKS 128
/* Tq = cu_q[S], Tk = the largest k_end.  0 for sizes that are refused.  A size that is enough for S sequences and Tq
 * queries is enough for fewer of either, whatever their lengths. */
size_t    bm_window_attention_scratch_bytes(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv,
                                            int32_t dh, int32_t S, int32_t Tq, int32_t Tk);
bm_status bm_window_attention_forward(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv, int32_t dh,
                                      const void* q, int32_t ld_q, const void* k, const void* v, int32_t ld_kv,
                                      const int32_t* cu_q_dev, const int32_t* cu_q_host,
                                      const int32_t* k_begin_dev, const int32_t* k_end_dev,
                                      const int32_t* k_begin_host, const int32_t* k_end_host, int32_t S,
                                      void* o, float* lse, void* scratch, size_t scratch_bytes, void* hip_stream);

/* The scratch is that of exactly these sizes.  Gradients from d_o and the forward's q, k, v, o and lse, which belong
 * together: an lse below that of these q and k makes probabilities above 1, which are held to 1 in some sums and not
 * in others.  dq in rows of ld_dq elements, dk and dv (rows k_begin .. k_end-1 of every sequence) in rows of ld_dkv;
 * overwritten.  Gradients that lie over an input are refused; columns of the same rows beside it are not. */
size_t    bm_window_attention_backward_scratch_bytes(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq,
                                                     int32_t Hkv, int32_t dh, int32_t S, int32_t Tq, int32_t Tk);
bm_status bm_window_attention_backward(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv, int32_t dh,
                                       const void* q, int32_t ld_q, const void* k, const void* v, int32_t ld_kv,
                                       const void* o, const void* d_o, const float* lse,
                                       const int32_t* cu_q_dev, const int32_t* cu_q_host,
                                       const int32_t* k_begin_dev, const int32_t* k_end_dev,
                                       const int32_t* k_begin_host, const int32_t* k_end_host, int32_t S,
                                       void* dq, int32_t ld_dq, void* dk, void* dv, int32_t ld_dkv, void* scratch,
                                       size_t scratch_bytes, void* hip_stream);

/* What such calls launch (host only, nothing is launched).
 *   forward [4]   host  0: tiles in fp32 arithmetic, 1: tiles on the matrix cores, 2: few queries, their keys in parts;
 *                       of 2, else 0: workgroups, 1 if keys and values go past the caches, 1 if the kv heads of a part
 *                       share an XCD
 *   backward [4]  host  keys of a workgroup of dK/dV, rows of one of dQ, launches of both (1 or 2), workgroups for parts
 *                       of first tokens' keys; 0 in fp32 arithmetic */
bm_status bm_probe_window_plan(int32_t dtype, int32_t window, int32_t sinks, int32_t Hq, int32_t Hkv, int32_t dh,
                               const int32_t* cu_q_host, const int32_t* k_begin_host, const int32_t* k_end_host, int32_t S,
                               int32_t* forward, int32_t* backward);

#ifdef __cplusplus
}
#endif
#endif
