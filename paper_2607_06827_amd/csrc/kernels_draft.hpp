// Internal interface between the C-ABI host layer and the kernels of the steps
// of several new tokens (include/speechkv_draft.h).
#pragma once

#include "kernels.hpp"

namespace skv {

// x / d and x % d by a multiplication, for x >= 0 and d >= 1 below 2^31: with
// 2^(s-1) < d <= 2^s, mul = floor(2^32 (2^s - d) / d) + 1 gives x / d =
// (mul x / 2^32 + x) / 2^s.
struct FastDivide {
  int32_t d, shift;
  uint32_t mul;
  FastDivide() = default;
  explicit FastDivide(int32_t by) : d(by), shift(0) {
    while (((int64_t)1 << shift) < by) ++shift;
    mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - by)) / by + 1);
  }
  __device__ __forceinline__ void divide(int32_t x, int32_t& q, int32_t& r) const {
    q = (int32_t)((__umulhi((uint32_t)x, mul) + (uint32_t)x) >> shift);
    r = x - q * d;
  }
};

struct AppendArgs {
  const void* q;  // may be null
  int64_t q_stride_b, q_stride_s, q_stride_h;  // elements
  int num_q_heads;  // 0 without q
  const void* k;
  const void* v;
  int64_t stride_b, stride_s, stride_h;
  int num_new;
  const int32_t* new_len;    // may be null: num_new
  const int32_t* positions;  // null with rot = 0
  const float* inv_freq;
  int rot;    // rotated elements of a head
  int pairs;  // neighbouring elements (else halves)
  const int32_t* cache_len;
  void* k_pages;
  void* v_pages;
  const int32_t* table;
  PagedView pv;
  void* q_out;
  int32_t* cache_len_out;  // may be null
};

struct TreeArgs {
  const void* q;
  const void* k_pages;
  const void* v_pages;
  const int32_t* table;
  PagedView pv;
  const int32_t* cache_len;
  int max_len;               // host bound on cache_len
  int num_nodes;             // rows of q, out and the mask per sequence
  const int32_t* nodes_of;   // may be null: num_nodes
  const uint32_t* mask;      // null: a chain
  int64_t mask_stride;       // words
  int mask_words;            // words of a row
  int num_q_heads;
  int group_shift;   // log2 of the query heads per KV head
  int row_groups;    // of a block: 1, 2 or 4
  int row_tiles;     // blocks that share a (sequence, KV head)'s rows
  int num_units;     // (sequence, KV head) pairs times splits (set by the launcher, as the divisors)
  FastDivide by_row_tiles, by_splits, by_heads;
  float scale_log2;  // scale * log2(e)
  int num_splits;
  int tiles_per_split;  // key tiles of a split, from the host's bound
  void* out;
  float* ws_o;   // [B][nodes][Hq][splits][D] unnormalised partial outputs
  float* ws_ml;  // [B][nodes][Hq][splits][2] running max (log2 units) and sum
};

// Layers of one launch of the commit kernel: their descriptions travel as
// kernel arguments (56 bytes each, 4 KB of arguments at most).
constexpr int kCommitLayers = 32;
constexpr int kCommitPath = 1024;  // longest path (SPEECHKV_MAX_TREE_NODES)
struct CommitLayer {
  void* k_pages;
  void* v_pages;
  const int32_t* table;
  const int32_t* cache_len;
  int32_t* cache_len_out;  // may be null
  int32_t num_pages, page_shift, max_pages;
};
struct CommitArgs {
  CommitLayer layer[kCommitLayers];
  const int32_t* path;
  const int32_t* path_len;
  int max_path;
  int num_nodes;
  int kv_heads;
  int heads, parts;    // (KV head, pool) pairs of a block, column parts of a row (set by the launcher)
  FastDivide by_path;  // max_path (set by the launcher)
};
static_assert(sizeof(CommitArgs) <= 4096, "kernel arguments");

// dtype: 0 = fp32, 1 = bf16.  Each launcher returns the launch status.
hipError_t launch_append(const AppendArgs& a, int dtype, int head_dim, int batch, hipStream_t s);
constexpr int kTreeKeys = 32;  // keys of a tile
constexpr int kTreeAhead = 64;  // tiles that a block looks ahead: 16 steps of four streams
constexpr int kMaskWords = 32;  // most words of a mask row (SPEECHKV_MAX_TREE_NODES / 32)
// Blocks that the rows (nodes x heads of a group) of a (sequence, KV head) take,
// of `groups` row groups of 32 each.
inline int tree_row_tiles(int64_t rows, int groups) { return (int)((rows + 32 * groups - 1) / (32 * groups)); }
// Rows (node, query head) of a sequence that a block of the merge takes.
constexpr int kMergeThreads = 256;
constexpr int tree_merge_rows(int head_dim) { return kMergeThreads / (head_dim / 4); }
hipError_t launch_tree(const TreeArgs& a, int dtype, int head_dim, int batch, hipStream_t s);
hipError_t launch_tree_merge(const TreeArgs& a, int dtype, int head_dim, int batch, hipStream_t s);
hipError_t launch_commit(const CommitArgs& a, int dtype, int head_dim, int layers, int batch, hipStream_t s);

}  // namespace skv
