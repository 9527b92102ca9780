/*
 * speechkv_shared.h - many questions about one recording, within a budget of
 * cache entries (libspeechkv.so, beside the calls of speechkv.h).
 *
 *   speechkv_shared_attn   single tokens of a batch whose sequences share long
 *                          prefixes: each prefix is read once for all of them
 *   speechkv_attn_weights  the attention weight that each cache entry gathers
 *                          from queries, of decoding steps or of a whole prompt
 *   speechkv_evict         keeps the entries that gathered most and moves them
 *                          together, all layers at once
 *
 * The conventions of speechkv.h hold: ownership, streams, errors before
 * anything is enqueued, element types, supported shapes.  Values in device
 * memory are the caller's obligation.  The kernels clamp every index they
 * derive from them: an entry that would lie past a block table or whose page is
 * out of range is neither read nor written, and counts as one that is not
 * there.
 */
#ifndef SPEECHKV_SHARED_H
#define SPEECHKV_SHARED_H

#include "speechkv_norm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most layers of one speechkv_evict (their buffers are checked against each
 * other, pair by pair). */
#define SPEECHKV_MAX_EVICT_LAYERS 256

/*
 * speechkv_shared_attn - one decoding step of attention for a batch whose
 * sequences come in groups, each with a prefix that its members share (the
 * recording that they ask about) before the entries of their own.
 *
 * Group j is the sequences b in [group_start[j], group_start[j + 1]) and its
 * prefix the first prefix_len[j] entries of row j of the prefix cache's block
 * table.  Query head h of sequence b (KV head g = h / G) attends to its group's
 * prefix and to the first cache_len[b] entries of its own cache:
 *   out[b][h] = sum_c softmax_c(scale * q[b][h] . K[c, g]) V[c, g]
 * over both, and 0 if it sees nothing.  A sequence of no group sees its own
 * entries alone.  The newest token's key and value are stored before the call
 * (speechkv_append_kv, speechkv_norm_append_kv) and counted in cache_len.  With
 * bf16 the softmax weights are rounded to bf16 (by 2^-8 of each at most) before
 * their products with V, as in speechkv_decode_attn; maxima, sums and the
 * outputs before their rounding are fp32, and so is everything with fp32.
 *
 * q, out         device, element type cache->dtype, [batch][num_q_heads]
 *                [head_dim], dense.
 * batch          sequences (1 .. 65535).
 * prefix         host pointer to the prefixes' cache description (block table
 *                [num_groups][max_pages_per_seq]).  num_kv_heads, head_dim and
 *                dtype are the cache's; the pools may be the cache's or others.
 * prefix_len     device int32 [num_groups], 0 <= prefix_len[j] <= max_prefix_len.
 * max_prefix_len host bound on prefix_len (it sizes the grid).
 * group_start    device int32 [num_groups + 1], non-decreasing, 0 <=
 *                group_start[0], group_start[num_groups] <= batch.
 * num_groups     1 .. 65535.
 * max_group      host bound on the members of a group, 1 .. batch.
 * cache          host pointer to the description of the sequences' own caches.
 * cache_len      device int32 [batch], 0 <= cache_len[b] <= max_cache_len.
 * max_cache_len  host bound on cache_len.
 * scale          logit scale, finite and > 0.
 * num_splits     key ranges that a prefix is split into, 1 .. 1024; 0 selects
 *                speechkv_shared_num_splits(), or the best count that the
 *                workspace holds.  Partial results are merged in a fixed order:
 *                the same call, with a workspace of the same size, gives the
 *                same bits.
 * lse            device fp32 [batch][num_q_heads] receiving the natural-log
 *                log-sum-exp of each row's scaled logits (-inf where it sees
 *                nothing), or NULL.
 * workspace      device scratch, 16-byte aligned; any contents.  With num_splits
 *                = 0 any size from batch * num_q_heads * (head_dim + 2) * 8 bytes
 *                on does; a call that has less than
 *                speechkv_shared_workspace_bytes(...) takes fewer splits, which
 *                may be slower.  With a given count it must hold that size.
 *                Calls that overlap in time need one each.
 * Errors: INVALID_ARG, WORKSPACE, HIP; UNSUPPORTED also where a launch would
 *         need 2^24 blocks or more, or for caches of 2^31 - 8191 entries and
 *         more; ALIAS when out, lse or the workspace overlaps anything read or
 *         each other.
 */
int speechkv_shared_attn(const void* q, int32_t batch, int32_t num_q_heads,
                         const speechkv_paged_kv* prefix, const int32_t* prefix_len,
                         int32_t max_prefix_len, const int32_t* group_start,
                         int32_t num_groups, int32_t max_group,
                         const speechkv_paged_kv* cache, const int32_t* cache_len,
                         int32_t max_cache_len, float scale, int32_t num_splits, void* out,
                         float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* The split count speechkv_shared_attn takes for num_splits = 0 with workspace
 * enough (-1 for invalid arguments), and the workspace it needs for num_splits
 * (0: enough for its own choice with either element type; the size 0 stands for
 * invalid arguments).  The choice falls where more members or entries fill the
 * chip, so a larger call may need less: a program whose calls vary asks for
 * every one of them, or keeps the largest size that it is ready to spend.  Host
 * only. */
int32_t speechkv_shared_num_splits(int32_t batch, int32_t num_groups, int32_t max_group,
                                   int32_t num_q_heads, int32_t num_kv_heads,
                                   int32_t head_dim, int32_t dtype, int32_t max_prefix_len,
                                   int32_t max_cache_len);
size_t speechkv_shared_workspace_bytes(int32_t batch, int32_t num_groups, int32_t max_group,
                                       int32_t num_q_heads, int32_t num_kv_heads,
                                       int32_t head_dim, int32_t max_prefix_len,
                                       int32_t max_cache_len, int32_t num_splits);

/*
 * speechkv_attn_weights - the attention weight that cache entries gather from
 * queries, added to what they have.
 *
 * For every sequence b, KV head g and cache entry c < cache_len[b]:
 *   weights_out[b][g][c] = weights[b][g][c] +
 *       sum over the query heads h of g and the rows i that see c of
 *       exp(scale * q[b][i][h] . K[b, c, g] - lse[b][h][i])
 * Each row sees a prefix of the cache: its first visible[b][i] entries.  With
 * the lse of an attention over those entries a row gives 1 in all; with that of
 * speechkv_shared_attn it gives 1 in all to the prefix and the own entries
 * together.  The lse of a prompt is speechkv_prefill_attn's, that of a decoding
 * step speechkv_shared_attn's (with one empty group where nothing is shared):
 * speechkv_decode_attn and speechkv_tree_attn return none.  A row whose lse is -inf (one that sees nothing) gives nothing.
 * Products and sums are fp32.
 *
 * q              host pointer to the queries' description (batch, num_rows,
 *                G * num_kv_heads heads; speechkv_norm.h), dtype the cache's.
 * batch          sequences (1 .. 65535).
 * num_rows       queries of a sequence (1 .. 2^24 - 1).
 * lse            device fp32, that of row i of head h of sequence b at
 *                lse + b*lse_stride_b + h*lse_stride_h + i*lse_stride_s (strides
 *                >= 0, in elements).
 * visible        device int32 [batch][num_rows], the entries that each row sees
 *                (any value: below 0 none, at most cache_len[b]), or NULL: the
 *                rows are the last num_rows tokens of the sequence, row i sees
 *                the entries c < cache_len[b] - (num_rows - 1 - i).
 * cache          host pointer to the cache description (only keys are read).
 * cache_len      device int32 [batch], 0 <= cache_len[b] <= max_cache_len.
 * max_cache_len  host bound on cache_len (it sizes the grid), at most capacity.
 * scale          logit scale, finite and > 0.
 * weights        device fp32 [batch][num_kv_heads][capacity], or NULL: zeros.
 * weights_out    the same shape, possibly weights itself.  Entries from
 *                cache_len[b] on are not written; those whose page is out of
 *                range keep their weight.
 * capacity       entries of a row of weights (>= 1).
 * Errors: INVALID_ARG, UNSUPPORTED (also where the launch would need 2^32
 *         threads or more, or for caches of 2^31 - 8191 entries and more), HIP;
 *         ALIAS when weights_out overlaps anything read but for weights =
 *         weights_out.
 */
int speechkv_attn_weights(const speechkv_heads* q, int32_t batch, int32_t num_rows,
                          const float* lse, int64_t lse_stride_b, int64_t lse_stride_h,
                          int64_t lse_stride_s, const int32_t* visible,
                          const speechkv_paged_kv* cache, const int32_t* cache_len,
                          int32_t max_cache_len, float scale, const float* weights,
                          float* weights_out, int32_t capacity, void* stream);

/*
 * One layer of speechkv_evict.
 * cache_len      device int32 [batch], entries before.
 * cache_len_out  device int32 [batch], entries after, or NULL.  Must not be
 *                cache_len.
 * weights        device fp32 [batch][num_kv_heads][capacity].
 * weights_out    the same shape, possibly weights itself.
 * kept           device int32 [batch][num_kv_heads][max_keep].
 */
typedef struct speechkv_evict_layer {
  speechkv_paged_kv cache;
  const int32_t* cache_len;
  int32_t* cache_len_out;
  const float* weights;
  float* weights_out;
  int32_t* kept;
} speechkv_evict_layer;

/*
 * speechkv_evict - shortens caches to the entries that gathered most weight, in
 * all layers with one or two launches (per 32 layers).
 *
 * For every layer, sequence b and KV head g, with L = cache_len[b]:
 *   n = min(L, keep_len[b]) entries stay: the first f = min(num_first, n), the
 *   last r = min(num_recent, n - f), and of those between them the n - f - r
 *   with the largest weight; between equal weights (0 and -0 are equal) the
 *   lower slot stays, and a NaN counts as less than every number.
 * With s_0 < s_1 < .. < s_(n-1) their slots:
 *   kept[b][g][j]        <-  s_j
 *   cache slot j         <-  cache slot s_j   (keys and values, bitwise, of g)
 *   weights_out[b][g][j] <-  weights[b][g][s_j], and 0 for n <= j < L
 *   cache_len_out[b]     <-  n
 * as if every slot were read before the first is written.  The heads of a cache
 * may keep different slots; their number is the same.  Entries from L on of the
 * weights and from n on of kept are not written.  A slot s_j without a page, or
 * whose place j has none, is not moved.
 *
 * After it a sequence's cache is shorter: decoding goes on behind its n
 * entries (the pages from ceil(n / page_size) on are free), and new entries
 * start with weight 0.  Positions of new tokens count as before.
 *
 * layers         host pointer to the layers' descriptions.  All have the same
 *                num_kv_heads, head_dim and dtype; lengths, pools, tables and
 *                page sizes may differ.  Layers may share pools (caller
 *                obligation: not pages, and no page twice in a block table).
 * num_layers     1 .. SPEECHKV_MAX_EVICT_LAYERS.
 * batch          sequences (1 .. 65535).
 * keep_len       device int32 [batch], 0 <= keep_len[b] <= max_keep.
 * max_keep       entries of a row of kept (>= 1), a bound on keep_len.
 * capacity       entries of a row of weights (>= 1), a bound on cache_len.
 * num_first, num_recent  >= 0.
 * Errors: INVALID_ARG, HIP; UNSUPPORTED also for a capacity of 2^31 - 8191 and
 *         more; ALIAS when a buffer written (pools, weights_out, kept,
 *         cache_len_out) overlaps one read or another written, of any layers
 *         (but for pools of the same kind, and weights = weights_out).
 */
int speechkv_evict(const speechkv_evict_layer* layers, int32_t num_layers, int32_t batch,
                   const int32_t* keep_len, int32_t max_keep, int32_t capacity,
                   int32_t num_first, int32_t num_recent, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SPEECHKV_SHARED_H */
