/*
 * speechkv_draft.h - steps of several new tokens over the compressed cache
 * (libspeechkv.so, beside the calls of speechkv.h).
 *
 * speechkv_decode_attn attends one new token per sequence.  A program that
 * drafts several tokens and has the model check them in one pass, or that
 * feeds a typed follow-up of some tokens into a running conversation, needs
 * the same for n tokens at once.  Four steps make up such a pass:
 *   speechkv_append_kv    per layer: rotates the new keys and queries by their
 *                         positions and stores keys and values behind the
 *                         entries that the cache holds
 *   speechkv_tree_attn    per layer: every new token attends to the whole cache
 *                         and to those new tokens that its row of a mask names
 *   (the program picks the tokens it accepts)
 *   speechkv_tree_commit  all layers at once: moves the accepted tokens'
 *                         entries together, behind the cache
 * After it the cache is what appending the accepted tokens alone would have
 * left, and the next pass begins.
 *
 * The conventions of speechkv.h hold: ownership, streams, errors before
 * anything is enqueued, element types, supported shapes.  In all three calls
 * cache_len[b] is the number of entries the cache holds BEFORE the new tokens,
 * whose slots are cache_len[b], cache_len[b] + 1, ...  It counts cache entries;
 * positions count full-resolution rows, so the two differ by what the pooling
 * of the speech saved.
 *
 * Values in device memory are the caller's obligation.  The kernels clamp
 * every index they derive from them: an entry that would lie past a sequence's
 * block table or whose page is out of range is neither read nor written.
 */
#ifndef SPEECHKV_DRAFT_H
#define SPEECHKV_DRAFT_H

#include "speechkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most new tokens per sequence that speechkv_tree_attn and
 * speechkv_tree_commit take. */
#define SPEECHKV_MAX_TREE_NODES 1024

/* Most layers of one speechkv_tree_commit (their buffers are checked against
 * each other, pair by pair). */
#define SPEECHKV_MAX_COMMIT_LAYERS 256

/* Which elements of a head speechkv_append_kv rotates together. */
#define SPEECHKV_ROPE_HALVES 0 /* (j, j + rot_dim / 2), j < rot_dim / 2 */
#define SPEECHKV_ROPE_PAIRS 1  /* (2 j, 2 j + 1),       j < rot_dim / 2 */

/*
 * speechkv_append_kv - stores new keys and values behind a sequence's cache
 * entries, with the keys (and the queries) rotated by their positions.
 *
 * For every sequence b, new token i < new_len[b] and head, with the angle
 * a_j = positions[b][i] * inv_freq[j], the rotation R takes the element pair
 * number j < rot_dim / 2 of a head (see the SPEECHKV_ROPE constants)
 *     (x, y)  to  (x cos a_j - y sin a_j,  x sin a_j + y cos a_j)
 * and leaves the elements from rot_dim on as they are:
 *   cache slot cache_len[b] + i  <-  R k[b][i],  v[b][i] (bitwise)
 *   q_out[b][i]                  <-  R q[b][i]
 *   cache_len_out[b]             <-  cache_len[b] + new_len[b]
 * Angles are reduced in 64 bits, so far positions lose nothing; the rotation
 * is done in fp32 and rounded once.  With rot_dim = 0 keys and queries are
 * copied bitwise.
 *
 * q              device, element type cache->dtype, or NULL when no queries
 *                are to be rotated (q_out is then NULL too).  Element
 *                (b, i, h, e) is at b*q_stride_b + i*q_stride_s + h*q_stride_h
 *                + e.  Strides are in elements, >= 0, and keep each row
 *                16-byte aligned; q, k and v may be views of one tensor.
 * num_q_heads    query heads (not read without q).
 * k, v           device, as q with num_kv_heads heads and the strides
 *                stride_b, stride_s, stride_h.
 * batch          sequences (1 .. 65535).
 * num_new        new tokens per sequence in q, k, v and q_out (1 .. 2^24 - 1).
 * new_len        device int32 [batch], how many of them sequence b has (0 ..
 *                num_new), or NULL: all.  The rows behind them are neither
 *                read nor written.
 * positions      device int32 [batch][num_new], each token's position (any
 *                int32; tokens of a tree that share a depth share a position).
 *                May be NULL when rot_dim is 0.
 * inv_freq       device fp32 [rot_dim / 2], radians per position.  May be NULL
 *                when rot_dim is 0.
 * rot_dim        rotated elements of a head, a multiple of 16 in 0 .. head_dim.
 * rope           SPEECHKV_ROPE_HALVES or SPEECHKV_ROPE_PAIRS.
 * cache_len      device int32 [batch], entries the cache holds.
 * cache          host pointer to the cache description.
 * q_out          device [batch][num_new][num_q_heads][head_dim], dense.  It may
 *                be q itself when q is dense like it.
 * cache_len_out  device int32 [batch], or NULL.  Must not be cache_len.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP; ALIAS when a page pool, q_out or
 *         cache_len_out overlaps anything read or another of the four (but for
 *         q_out = q as above).
 */
int speechkv_append_kv(const void* q, int64_t q_stride_b, int64_t q_stride_s,
                       int64_t q_stride_h, int32_t num_q_heads, const void* k,
                       const void* v, int64_t stride_b, int64_t stride_s,
                       int64_t stride_h, int32_t batch, int32_t num_new,
                       const int32_t* new_len, const int32_t* positions,
                       const float* inv_freq, int32_t rot_dim, int32_t rope,
                       const int32_t* cache_len, const speechkv_paged_kv* cache,
                       void* q_out, int32_t* cache_len_out, void* stream);

/*
 * speechkv_tree_attn - attention of several new tokens per sequence, the nodes
 * of a tree (or any order), over the cache and over each other.
 *
 * With L = cache_len[b] and n = num_nodes_of[b], cache slots [0, L) hold what
 * came before and slot L + j holds node j (stored by speechkv_append_kv).
 * Node i < n of query head h (KV head g = h / G) sees every slot c < L and the
 * slots L + j, j < n, for which bit j of its mask row is set:
 *   out[b][i][h] = sum_c softmax_c(scale * q[b][i][h] . K[b, c, g]) V[b, c, g]
 * over what it sees, and 0 if it sees nothing (L = 0 and an empty mask row).
 * What a node does not see does not reach its output, whatever it holds
 * (infinities and NaN included).  With bf16 the softmax weights are rounded to
 * bf16 (by 2^-8 of each at most) before their products with V, as in
 * speechkv_decode_attn; maxima, sums and the outputs before their rounding are
 * fp32, and so is everything with fp32.
 *
 * q, out         device, element type cache->dtype,
 *                [batch][num_nodes][num_q_heads][head_dim], dense.  Rows
 *                i >= num_nodes_of[b] are not written.
 * batch          sequences (1 .. 65535).
 * num_nodes      nodes per sequence in q, out and tree_mask, 1 ..
 *                SPEECHKV_MAX_TREE_NODES.
 * num_nodes_of   device int32 [batch], how many of them sequence b has (0 ..
 *                num_nodes), or NULL: all.
 * tree_mask      device uint32, row i of sequence b being the ceil(num_nodes /
 *                32) words at tree_mask + b * mask_stride_b + i * ceil(num_nodes
 *                / 32), bit j % 32 of word j / 32 for node j.  A node sees
 *                itself only if its own bit is set.  Or NULL: node i sees the
 *                nodes j <= i (a chain).
 * mask_stride_b  words from one sequence's mask to the next (>= 0; 0: one mask
 *                for every sequence).
 * cache_len      device int32 [batch], 0 <= cache_len[b] <= max_cache_len.
 *                Block-table entries past the last node's page may hold any
 *                value.
 * max_cache_len  host bound on cache_len (it sizes the grid); max_cache_len +
 *                num_nodes slots may exceed what a block table holds as long
 *                as the sequences' own slots do not.  UNSUPPORTED from 2^31 -
 *                8191 on, and with thousands of splits from up to 2^21 less.
 * scale          logit scale, finite and > 0.
 * num_splits     key ranges each (sequence, KV head) is split into; 0 selects
 *                speechkv_tree_num_splits(), or the best count that the
 *                workspace holds (1 needs none).  Partial results are merged in
 *                a fixed order: the same call, with a workspace of the same
 *                size, gives the same bits.  UNSUPPORTED where a launch would
 *                need 2^24 blocks or more.
 * workspace      device scratch (16-byte aligned; any contents), or NULL with
 *                workspace_bytes not read.  With num_splits = 0 any size does;
 *                a call that has less than speechkv_tree_workspace_bytes(...)
 *                takes fewer splits, which may be slower.  With num_splits > 1
 *                it must hold that size.  Calls that overlap in time need one
 *                each.
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, HIP; ALIAS when out or the
 *         workspace overlaps q, the mask, the lengths, the block table, a page
 *         pool or each other.
 */
int speechkv_tree_attn(const void* q, int32_t batch, int32_t num_nodes,
                       int32_t num_q_heads, const speechkv_paged_kv* cache,
                       const int32_t* cache_len, int32_t max_cache_len,
                       const int32_t* num_nodes_of, const uint32_t* tree_mask,
                       int64_t mask_stride_b, float scale, int32_t num_splits,
                       void* out, void* workspace, size_t workspace_bytes,
                       void* stream);

/* The split count speechkv_tree_attn takes for num_splits = 0 with workspace
 * enough (-1 for invalid arguments), and the workspace it needs for num_splits
 * (0: enough for its own choice with either element type).  The choice falls
 * where more sequences, nodes or keys fill the chip without splits, so a larger
 * call may need less: a program whose calls vary asks for every one of them, or
 * keeps the largest size that it is ready to spend. */
int32_t speechkv_tree_num_splits(int32_t batch, int32_t num_nodes, int32_t num_q_heads,
                                 int32_t num_kv_heads, int32_t head_dim, int32_t dtype,
                                 int32_t max_cache_len);
size_t speechkv_tree_workspace_bytes(int32_t batch, int32_t num_nodes, int32_t num_q_heads,
                                     int32_t num_kv_heads, int32_t head_dim,
                                     int32_t max_cache_len, int32_t num_splits);

/*
 * One layer's cache with its lengths, for speechkv_tree_commit.
 * cache_len      device int32 [batch], entries before the new tokens.
 * cache_len_out  device int32 [batch], or NULL.  Must not be cache_len.
 */
typedef struct speechkv_layer_cache {
  speechkv_paged_kv cache;
  const int32_t* cache_len;
  int32_t* cache_len_out;
} speechkv_layer_cache;

/*
 * speechkv_tree_commit - keeps the accepted nodes of a tree: their entries move
 * together behind the cache, in all layers with one launch (per 32 layers).
 *
 * For every layer, sequence b, KV head and j < path_len[b]:
 *   cache slot cache_len[b] + j  <-  cache slot cache_len[b] + path[b][j]
 *   cache_len_out[b]             <-  cache_len[b] + path_len[b]
 * as if every slot were read before the first is written, so path may name
 * nodes in any order and more than once.  An entry of path outside [0,
 * num_nodes) leaves its slot as it is.
 *
 * layers         host pointer to the layers' descriptions.  All have the same
 *                num_kv_heads, head_dim and dtype; lengths, pools, tables and
 *                page sizes may differ.  Layers may share pools (caller
 *                obligation: not pages).
 * num_layers     1 .. SPEECHKV_MAX_COMMIT_LAYERS.
 * batch          sequences (1 .. 65535).
 * path           device int32 [batch][max_path], accepted nodes.
 * max_path       1 .. num_nodes.
 * path_len       device int32 [batch], 0 .. max_path.
 * num_nodes      nodes per sequence, 1 .. SPEECHKV_MAX_TREE_NODES.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP; ALIAS when a page pool or a
 *         cache_len_out overlaps path, path_len, a cache_len or a block table,
 *         a K pool overlaps a V pool, or two cache_len_out overlap each other
 *         or a pool.
 */
int speechkv_tree_commit(const speechkv_layer_cache* layers, int32_t num_layers,
                         int32_t batch, const int32_t* path, int32_t max_path,
                         const int32_t* path_len, int32_t num_nodes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SPEECHKV_DRAFT_H */
