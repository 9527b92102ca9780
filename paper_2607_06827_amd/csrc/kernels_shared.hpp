// Internal interface between the C-ABI host layer and the kernels of shared
// prefixes, entry weights and eviction (include/speechkv_shared.h).
#pragma once

#include "kernels_norm.hpp"

namespace skv {

// A cache that is only read: pools, block table and lengths.
struct KeySource {
  const void* k_pages;
  const void* v_pages;
  const int32_t* table;
  const int32_t* len;
  int max_len;  // host bound on len
  PagedView pv;
};

struct SharedArgs {
  const void* q;
  KeySource prefix, own;       // prefix: rows of table and len by group, own: by sequence
  const int32_t* group_start;  // [groups + 1]
  int batch, groups, max_group;
  int num_q_heads, group_shift;  // log2 of the query heads per KV head
  float scale_log2;              // scale * log2(e)
  int row_tiles;                 // prefix blocks that share a (group, KV head)'s rows
  int prefix_splits, own_splits;
  int prefix_tiles, own_tiles;   // key tiles of a split, from the host's bounds
  int prefix_units;              // (group, KV head)s times splits (set by the launcher,
  int prefix_blocks;             // as their blocks and the divisors)
  FastDivide by_row_tiles, by_prefix_splits, by_own_splits, by_heads;
  void* out;
  float* lse;    // may be null
  float* ws_o;   // [B][Hq][prefix_splits + own_splits][D] unnormalised partial outputs
  float* ws_ml;  // [B][Hq][prefix_splits + own_splits][2] running max (log2 units) and sum
};

struct WeightArgs {
  HeadRows q;
  int num_rows;
  int group_shift;
  const float* lse;
  int64_t lse_b, lse_h, lse_s;
  const int32_t* visible;  // may be null: the rows are the last tokens
  KeySource cache;         // (no values)
  int batch;
  float scale_log2;
  const float* weights;  // may be null: zeros
  float* weights_out;
  int capacity;
  int row_tiles;   // tiles of 16 rows of a (sequence, KV head)
  int steps;       // with few rows: steps of a wave (set by the plan, as key_blocks)
  int stretches;   // with many rows: stretches of keys of a block (as steps)
  int key_blocks;  // blocks of a (sequence, KV head)
  FastDivide by_pairs, by_heads;  // (set by the launcher)
};
constexpr int kWeightFew = 2;     // row tiles that a block keeps in LDS
constexpr int kWeightStep = 32;   // keys of a wave's step with few rows
constexpr int kWeightSteps = 16;  // most steps of a wave
// Keys of a block with many rows.
constexpr int weight_keys(int row_bytes) { return row_bytes > 256 ? 32 : 64; }
void plan_weights(WeightArgs& a, int dim, int elt_size);

// Layers of one launch of the eviction's kernels: their descriptions travel as
// kernel arguments (4 KB at most).
constexpr int kEvictLayers = 32;
struct EvictLayer {
  void* k_pages;
  void* v_pages;
  const int32_t* table;
  const int32_t* cache_len;
  int32_t* cache_len_out;  // may be null
  const float* weights;
  float* weights_out;
  int32_t* kept;
  int32_t num_pages, page_shift, max_pages;
};
struct EvictArgs {
  EvictLayer layer[kEvictLayers];
  const int32_t* keep_len;
  int max_keep, capacity, num_first, num_recent;
  int kv_heads;
  int parts;  // column parts of a row (set by the launcher)
};
static_assert(sizeof(EvictArgs) <= 4096, "kernel arguments");

// dtype: 0 = fp32, 1 = bf16.  Each launcher returns the launch status.
hipError_t launch_shared(const SharedArgs& a, int dtype, int head_dim, hipStream_t s);
hipError_t launch_shared_merge(const SharedArgs& a, int dtype, int head_dim, hipStream_t s);
constexpr int kSharedKeys = 32;  // keys of a tile
constexpr int kSharedRows = 32;  // rows of a prefix block
hipError_t launch_weights(const WeightArgs& a, int dtype, int head_dim, hipStream_t s);
hipError_t launch_evict(const EvictArgs& a, int dtype, int head_dim, int layers, int batch, hipStream_t s);

}  // namespace skv
