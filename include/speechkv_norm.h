/*
 * speechkv_norm.h - norms of queries and keys for each head and the rotation by
 * position, in one pass (libspeechkv.so, beside the calls of speechkv.h).
 *
 * The pooling, the attention and the cache take queries and keys as the model's
 * attention sees them.  Models that norm each head of a query or key before
 * they rotate it reach that form here from the projection's output:
 *   speechkv_norm_rope       into tensors (a prompt: speechkv_pool_kv and
 *                            speechkv_prefill_attn come next; a decoding step
 *                            of speechkv_decode_attn)
 *   speechkv_norm_rope_bwd   its gradients (training)
 *   speechkv_norm_append_kv  keys and values straight behind the entries of a
 *                            cache, as speechkv_append_kv does without a norm
 *
 * Of a row x of one head (head_dim elements, D):
 *   r = 1 / sqrt(sum_e x_e^2 / D + eps)        (1 without a norm)
 *   y = R (gamma o r x)                        (gamma 1 without one)
 * where the rotation R takes the element pair number j < rot_dim / 2 (see the
 * SPEECHKV_ROPE constants of speechkv_draft.h) with the angle
 * a_j = positions[axis[j]] * inv_freq[j]
 *     (u, w)  to  (u cos a_j - w sin a_j,  u sin a_j + w cos a_j)
 * and leaves the elements from rot_dim on as they are.  Sums, norms and the
 * rotation are fp32, angles are reduced in 64 bits, and y is rounded once.  A
 * row whose squares sum past the range of fp32 counts as infinitely long (r is
 * 0); a row with an infinity or a NaN is wrong as a whole, other rows are not.
 *
 * The conventions of speechkv.h hold: ownership, streams, errors before
 * anything is enqueued, element types.  head_dim is 64 or 128.
 */
#ifndef SPEECHKV_NORM_H
#define SPEECHKV_NORM_H

#include "speechkv_draft.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rows of head_dim elements, one for each (sequence b, row i, head h): element
 * e of it is at data + b*stride_b + i*stride_s + h*stride_h + e (device memory;
 * strides in elements, >= 0, keeping each row 16-byte aligned).  The views of a
 * call may be parts of one tensor, such as the output of a fused projection.
 * In a tensor that is written, the axes longer than 1 must be nested: sorted by
 * stride, each stride is at least what the axes before it span.
 */
typedef struct speechkv_heads {
  void* data;
  int64_t stride_b, stride_s, stride_h;
  int32_t num_heads;
} speechkv_heads;

/*
 * The norm of a call.  gamma_q, gamma_k: device fp32 [head_dim], 16-byte
 * aligned, or NULL: 1.  eps: finite, at least 2^-126.
 */
typedef struct speechkv_head_norm {
  const float* gamma_q;
  const float* gamma_k;
  float eps;
} speechkv_head_norm;

/*
 * The rotation of a call.
 * positions      device int32 [num_axes][batch][rows]: a row's position on each
 *                axis (any int32).
 * inv_freq       device fp32 [rot_dim / 2], radians per position.
 * axis           device int32 [rot_dim / 2], which axis turns pair j (values
 *                outside [0, num_axes) count as the nearest inside), or NULL:
 *                the first.
 * num_axes       1 .. 16.
 * rot_dim        rotated elements of a head, a multiple of 16 in 16 .. head_dim.
 * layout         SPEECHKV_ROPE_HALVES or SPEECHKV_ROPE_PAIRS.
 */
typedef struct speechkv_rope {
  const int32_t* positions;
  const float* inv_freq;
  const int32_t* axis;
  int32_t num_axes, rot_dim, layout;
} speechkv_rope;

/*
 * speechkv_norm_rope - y as above for the queries and the keys.
 *
 * q, k           host pointers to the inputs' descriptions; either may be NULL,
 *                not both.
 * batch          sequences (1 .. 65535).
 * num_rows       rows per sequence (>= 1); batch * num_rows < 2^24, otherwise
 *                UNSUPPORTED.
 * row_len        device int32 [batch], how many rows sequence b has (0 ..
 *                num_rows), or NULL: all.  The rows behind them are neither
 *                read nor written.
 * head_dim, dtype  of all of them (UNSUPPORTED if not listed above).
 * norm           host pointer, or NULL: no norm.
 * rope           host pointer, or NULL: no rotation.  (Without either, rows are
 *                copied bitwise.)
 * q_out, k_out   host pointers to the outputs' descriptions, NULL where q or k
 *                is; num_heads as in the input.  An output may be its own input
 *                (one address and one set of strides).
 * Errors: INVALID_ARG, UNSUPPORTED, HIP; ALIAS when an output overlaps anything
 *         read or the other output (but for its own input as above, and heads
 *         of one tensor, in any order of its axes, that lie beside each
 *         other).
 */
int speechkv_norm_rope(const speechkv_heads* q, const speechkv_heads* k, int32_t batch,
                       int32_t num_rows, const int32_t* row_len, int32_t head_dim,
                       int32_t dtype, const speechkv_head_norm* norm,
                       const speechkv_rope* rope, const speechkv_heads* q_out,
                       const speechkv_heads* k_out, void* stream);

/*
 * speechkv_norm_rope_bwd - gradients of speechkv_norm_rope.  With the gradient
 * dy of y, turned back (g = R^-1 dy), and h = gamma o g:
 *   dgamma = sum over rows and heads of g o r x
 *   dx     = r (h - r x (sum_e h_e r x_e) / D)
 * (dx = g without a norm).  r is computed again from x.
 *
 * q, k           the forward's inputs; dq_out, dk_out the gradients of its
 *                outputs; dq, dk receive those of its inputs.  The three of the
 *                queries, or the three of the keys, may be NULL.  dq may be
 *                dq_out (one address and one set of strides), dk may be dk_out.
 * batch .. rope  as for the forward.  Rows behind a sequence's last are neither
 *                read nor written and add nothing to dgamma.
 * dgamma_q, dgamma_k  device fp32 [head_dim], or NULL.  NULL without a norm and
 *                where the queries or keys are.
 * workspace      device, >= speechkv_norm_rope_bwd_workspace_bytes bytes,
 *                16-byte aligned, when a dgamma is asked for (partial sums,
 *                added in a fixed order: the same call gives the same bits).
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, HIP; ALIAS as for the forward.
 */
int speechkv_norm_rope_bwd(const speechkv_heads* q, const speechkv_heads* k,
                           const speechkv_heads* dq_out, const speechkv_heads* dk_out,
                           int32_t batch, int32_t num_rows, const int32_t* row_len,
                           int32_t head_dim, int32_t dtype, const speechkv_head_norm* norm,
                           const speechkv_rope* rope, const speechkv_heads* dq,
                           const speechkv_heads* dk, float* dgamma_q, float* dgamma_k,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Workspace bytes of speechkv_norm_rope_bwd with a dgamma (num_q_heads or
 * num_kv_heads 0: without the queries or the keys), or 0 for invalid or
 * unsupported arguments.  The size for the most sequences and rows of a program
 * is enough for fewer.  Host only. */
size_t speechkv_norm_rope_bwd_workspace_bytes(int32_t batch, int32_t num_rows,
                                              int32_t num_q_heads, int32_t num_kv_heads,
                                              int32_t head_dim);

/*
 * speechkv_norm_append_kv - speechkv_norm_rope with the keys, and the values as
 * they are, stored behind a sequence's cache entries.  For every sequence b and
 * row i < row_len[b]:
 *   cache slot cache_len[b] + i  <-  y of k[b][i],  v[b][i] (bitwise)
 *   q_out[b][i]                  <-  y of q[b][i]
 *   cache_len_out[b]             <-  cache_len[b] + row_len[b]
 *
 * q, q_out       as above, or both NULL.
 * k, v           host pointers to their descriptions; num_heads of both is the
 *                cache's num_kv_heads.
 * batch .. rope  as above; head_dim and dtype are the cache's.
 * cache_len      device int32 [batch], entries the cache holds.
 * cache          host pointer to the cache description.  Slots without a page
 *                (past the block table, or a table entry out of range) are not
 *                written.
 * cache_len_out  device int32 [batch], or NULL.  Must not be cache_len.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP; ALIAS when a page pool, q_out or
 *         cache_len_out overlaps anything read or another of the four (but for
 *         q_out as above).
 */
int speechkv_norm_append_kv(const speechkv_heads* q, const speechkv_heads* k,
                            const speechkv_heads* v, int32_t batch, int32_t num_rows,
                            const int32_t* row_len, const speechkv_head_norm* norm,
                            const speechkv_rope* rope, const int32_t* cache_len,
                            const speechkv_paged_kv* cache, const speechkv_heads* q_out,
                            int32_t* cache_len_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SPEECHKV_NORM_H */
