// C-ABI host layer of shared prefixes, entry weights and eviction
// (include/speechkv_shared.h): argument validation, grid sizing and dispatch.
// Every check runs before the first HIP call.
#include "../../include/speechkv_shared.h"

#include "head_views.hpp"
#include "kernels_shared.hpp"

namespace {

using namespace skv;

// Longest cache: key numbers, with the tiles that a block looks ahead, stay in 31
// bits.
constexpr int32_t kMaxLen = INT32_MAX - 8191;
constexpr int32_t kMaxSplits = 1024;

int row_tiles_of(int64_t rows) { return (int)((rows + kSharedRows - 1) / kSharedRows); }

// How speechkv_shared_attn cuts a call: splits of a prefix and of the own entries.
struct SharedPlan {
  int splits, own_splits;
};

int64_t tiles_of(int max_len) { return ((int64_t)max_len + kSharedKeys - 1) / kSharedKeys; }

size_t shared_bytes(int32_t batch, int32_t q_heads, int32_t head_dim, const SharedPlan& p) {
  return (size_t)batch * q_heads * (p.splits + p.own_splits) * (head_dim + 2) * sizeof(float);
}

// The plan with the smallest estimated time: with the given prefix splits, or with 0 of
// those whose partial rows fit `room` bytes (or the smallest of all).  (The best counts
// fall where more members or entries fill the chip, so room for the largest call may be
// too little for a smaller one's.)
// The estimate is fitted to a sweep on MI355X over 20 shapes of 1 to 64 sequences
// in 1 to 20 groups, 1 to 8 KV heads of 1 to 8 query heads, prefixes of 126 to 7532
// and own caches of 10 to 5000 entries, both element types and head sizes; its
// choice takes 0.7% longer than the best of the candidates on average, 4.4% at most.
// In us:
//  - a block takes 0.3, a step of its four waves over a 128-wide bf16 tile each 1.21,
//    one of a wave with own entries 1.37; 64-wide heads take 0.58 of it, fp32 5.1 and
//    2.3 times; what runs at once is two blocks a CU (four with 64-wide bf16 heads, one
//    with 128-wide fp32), and a full chip takes 1.5 times as long as its blocks alone;
//  - the blocks that a CU has at first (numbers 0, 256, .. of the launch) take 0.8 of
//    what they take one after the other (1.8% and 9% without this and the next);
//  - (group, KV head, split)s go round the eight XCDs, so the fullest XCD counts for
//    all (1.3% and 12% without this);
//  - keys are read at 6.5 TB/s, once;
//  - each partial row is written and read at 2.3 TB/s.
SharedPlan shared_plan(int batch, int groups, int max_group, int group, int kv_heads, int head_dim, int dtype,
                       int max_prefix, int max_len, int splits, size_t room) {
  const bool f32 = dtype == SPEECHKV_DTYPE_F32, wide = head_dim == 128;
  // members of a group: between the average and the bound
  const double members = 0.5 * (max_group + std::min<double>(max_group, (double)batch / groups));
  const double units = (double)groups * kv_heads, own_units = (double)batch * kv_heads;
  const double row_tiles = std::ceil(members * group / kSharedRows), row_bytes = head_dim * (f32 ? 4.0 : 2.0);
  const int64_t tiles = std::max<int64_t>(1, tiles_of(max_prefix)), own = std::max<int64_t>(1, tiles_of(max_len));
  const int per_cu = f32 && wide ? 1 : !f32 && !wide ? 4 : 2;
  const double slots = 256.0 * per_cu;
  const double size = f32 ? (wide ? 5.08 : 2.29) : wide ? 1.0 : 0.58;
  const double read_us = (units * max_prefix + own_units * max_len) * 2 * row_bytes / 6.5e6;
  static const int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
  SharedPlan best = {splits ? splits : 1, 1};
  double best_us = 1e300;
  for (int count : counts) {
    const int s = splits ? splits : count;
    if (!splits && s > tiles) break;
    const double block_us = 0.31 + 1.21 * size * (double)(((tiles + s - 1) / s + 3) / 4);
    for (int o : counts) {
      if (o > own || o > 32) break;
      if (!splits && shared_bytes(batch, group * kv_heads, head_dim, {s, o}) > room) break;
      const double own_us = 0.31 + 1.37 * size * (double)((own + o - 1) / o);
      const double blocks = std::ceil(units * s / 8) * 8 * row_tiles, own_blocks = std::ceil(own_units * o / 4);
      const double all_us = 1.5 * (blocks * block_us + own_blocks * own_us) / slots;
      double cu_us = 0.0;
      for (int k = 0; k < per_cu && 256.0 * k < blocks + own_blocks; ++k)
        cu_us += 0.8 * (256.0 * k < blocks ? block_us : own_us);
      const double us = std::max({block_us, own_us, all_us, cu_us, 0.31 + read_us}) +
                        own_units * group * (s + o) * head_dim * 8 / 2.34e6;
      if (us < best_us) {
        best_us = us;
        best = {s, o};
      }
    }
    if (splits) break;
  }
  return best;
}

bool shared_sizes_bad(int32_t batch, int32_t num_groups, int32_t max_group, int32_t max_prefix_len,
                      int32_t max_cache_len, int32_t num_splits) {
  return batch < 1 || batch > kMaxGrid || num_groups < 1 || num_groups > kMaxGrid || max_group < 1 ||
         max_group > batch || max_prefix_len < 0 || max_cache_len < 0 || num_splits < 0 || num_splits > kMaxSplits;
}

// Bytes of [batch][heads][n] values of 4 bytes, or -1 when they do not fit 2^62.
int64_t rows_bytes(int32_t batch, int32_t heads, int32_t n) {
  const __int128 bytes = (__int128)batch * heads * n * 4;
  return bytes < ((__int128)1 << 62) ? (int64_t)bytes : -1;
}

int64_t capacity_of(const speechkv_paged_kv* c) { return (int64_t)c->max_pages_per_seq * c->page_size; }

KeySource source_of(const speechkv_paged_kv* c, const int32_t* len, int32_t max_len) {
  return {c->k_pages, c->v_pages, c->block_table, len, max_len, view_of(c)};
}

}  // namespace

extern "C" {

int32_t speechkv_shared_num_splits(int32_t batch, int32_t num_groups, int32_t max_group, int32_t num_q_heads,
                                   int32_t num_kv_heads, int32_t head_dim, int32_t dtype, int32_t max_prefix_len,
                                   int32_t max_cache_len) {
  if (shared_sizes_bad(batch, num_groups, max_group, max_prefix_len, max_cache_len, 0) || num_kv_heads < 1 ||
      num_kv_heads > kMaxGrid || (head_dim != 64 && head_dim != 128) ||
      (dtype != SPEECHKV_DTYPE_F32 && dtype != SPEECHKV_DTYPE_BF16))
    return -1;
  const int group = group_of(num_q_heads, num_kv_heads);
  if (group < 0) return -1;
  return shared_plan(batch, num_groups, max_group, group, num_kv_heads, head_dim, dtype, max_prefix_len, max_cache_len,
                     0, SIZE_MAX)
      .splits;
}

size_t speechkv_shared_workspace_bytes(int32_t batch, int32_t num_groups, int32_t max_group, int32_t num_q_heads,
                                       int32_t num_kv_heads, int32_t head_dim, int32_t max_prefix_len,
                                       int32_t max_cache_len, int32_t num_splits) {
  if (num_splits < 0 || num_splits > kMaxSplits ||
      speechkv_shared_num_splits(batch, num_groups, max_group, num_q_heads, num_kv_heads, head_dim, SPEECHKV_DTYPE_BF16,
                                 max_prefix_len, max_cache_len) < 0)
    return 0;
  size_t most = 0;
  for (int dtype : {SPEECHKV_DTYPE_F32, SPEECHKV_DTYPE_BF16})
    most = std::max(most, shared_bytes(batch, num_q_heads, head_dim,
                                       shared_plan(batch, num_groups, max_group, num_q_heads / num_kv_heads, num_kv_heads,
                                                   head_dim, dtype, max_prefix_len, max_cache_len, num_splits, SIZE_MAX)));
  return most;
}

int speechkv_shared_attn(const void* q, int32_t batch, int32_t num_q_heads, const speechkv_paged_kv* prefix,
                         const int32_t* prefix_len, int32_t max_prefix_len, const int32_t* group_start,
                         int32_t num_groups, int32_t max_group, const speechkv_paged_kv* cache,
                         const int32_t* cache_len, int32_t max_cache_len, float scale, int32_t num_splits, void* out,
                         float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !out || !prefix_len || !group_start || !cache_len) return SPEECHKV_ERR_INVALID_ARG;
  int st = check_cache(prefix);
  if (st || (st = check_cache(cache))) return st;
  if (shared_sizes_bad(batch, num_groups, max_group, max_prefix_len, max_cache_len, num_splits))
    return SPEECHKV_ERR_INVALID_ARG;
  if (prefix->num_kv_heads != cache->num_kv_heads || prefix->head_dim != cache->head_dim ||
      prefix->dtype != cache->dtype || max_prefix_len > capacity_of(prefix) || max_cache_len > capacity_of(cache))
    return SPEECHKV_ERR_INVALID_ARG;
  if (!(scale > 0.f) || scale > 3.0e38f) return SPEECHKV_ERR_INVALID_ARG;  // finite, > 0
  if (num_q_heads < 1 || num_q_heads % cache->num_kv_heads) return SPEECHKV_ERR_INVALID_ARG;
  const int group = group_of(num_q_heads, cache->num_kv_heads), D = cache->head_dim, heads = cache->num_kv_heads;
  if (group < 0 || max_prefix_len > kMaxLen || max_cache_len > kMaxLen) return SPEECHKV_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(out) || !aligned4(lse) || !aligned4(prefix_len) || !aligned4(group_start) ||
      !aligned4(cache_len))
    return SPEECHKV_ERR_INVALID_ARG;
  const SharedPlan plan = shared_plan(batch, num_groups, max_group, group, heads, D, cache->dtype, max_prefix_len,
                                      max_cache_len, num_splits, workspace ? workspace_bytes : 0);
  const size_t need = shared_bytes(batch, num_q_heads, D, plan);
  if (!workspace || workspace_bytes < need || !aligned16(workspace)) return SPEECHKV_ERR_WORKSPACE;
  const int row_tiles = row_tiles_of((int64_t)max_group * group);
  const __int128 blocks = ((__int128)num_groups * heads * plan.splits + 7) * row_tiles +
                          (__int128)batch * heads * plan.own_splits;
  const int64_t merged = (int64_t)batch * num_q_heads / (256 / (D / 4)) + 1;
  if (blocks > kMaxBlocks || merged > kMaxBlocks) return SPEECHKV_ERR_UNSUPPORTED;
  const int64_t qo = (int64_t)batch * num_q_heads * D * elt_size(cache->dtype), lens = (int64_t)batch * 4;
  const int64_t pool = page_pool_bytes(cache), prefix_pool = page_pool_bytes(prefix);
  const Region rd[] = {{q, qo}, {prefix_len, (int64_t)num_groups * 4}, {group_start, (int64_t)(num_groups + 1) * 4},
                       {cache_len, lens}, {prefix->block_table, table_bytes(prefix, num_groups)},
                       {cache->block_table, table_bytes(cache, batch)}, {prefix->k_pages, prefix_pool},
                       {prefix->v_pages, prefix_pool}, {cache->k_pages, pool}, {cache->v_pages, pool}};
  const Region wr[] = {{out, qo}, {lse, (int64_t)batch * num_q_heads * 4}, {workspace, (int64_t)need}};
  if (aliased(wr, 3, rd, 10)) return SPEECHKV_ERR_ALIAS;
  SharedArgs a = {};
  a.q = q;
  a.prefix = source_of(prefix, prefix_len, max_prefix_len);
  a.own = source_of(cache, cache_len, max_cache_len);
  a.group_start = group_start;
  a.batch = batch;
  a.groups = num_groups;
  a.max_group = max_group;
  a.num_q_heads = num_q_heads;
  a.group_shift = log2_exact(group);
  a.scale_log2 = scale * 1.4426950408889634f;
  a.row_tiles = row_tiles;
  a.prefix_splits = plan.splits;
  a.own_splits = plan.own_splits;
  a.prefix_tiles = (int)((tiles_of(max_prefix_len) + plan.splits - 1) / plan.splits);
  a.own_tiles = (int)((tiles_of(max_cache_len) + plan.own_splits - 1) / plan.own_splits);
  a.out = out;
  a.lse = lse;
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = a.ws_o + (size_t)batch * num_q_heads * (plan.splits + plan.own_splits) * D;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = launch_shared(a, cache->dtype, D, s);
  if (e == hipSuccess) e = launch_shared_merge(a, cache->dtype, D, s);
  return status_of(e);
}

int speechkv_attn_weights(const speechkv_heads* q, int32_t batch, int32_t num_rows, const float* lse,
                          int64_t lse_stride_b, int64_t lse_stride_h, int64_t lse_stride_s, const int32_t* visible,
                          const speechkv_paged_kv* cache, const int32_t* cache_len, int32_t max_cache_len, float scale,
                          const float* weights, float* weights_out, int32_t capacity, void* stream) {
  if (!q || !lse || !cache_len || !weights_out) return SPEECHKV_ERR_INVALID_ARG;
  int st = check_cache(cache);
  if (st) return st;
  if (batch < 1 || batch > kMaxGrid || num_rows < 1 || num_rows > kMaxBlocks || capacity < 1 || max_cache_len < 0 ||
      max_cache_len > capacity || max_cache_len > capacity_of(cache))
    return SPEECHKV_ERR_INVALID_ARG;
  if (!(scale > 0.f) || scale > 3.0e38f) return SPEECHKV_ERR_INVALID_ARG;  // finite, > 0
  if (lse_stride_b < 0 || lse_stride_h < 0 || lse_stride_s < 0 || !aligned4(lse) || !aligned4(visible) ||
      !aligned4(cache_len) || !aligned4(weights) || !aligned4(weights_out))
    return SPEECHKV_ERR_INVALID_ARG;
  const Sizes n = {batch, num_rows, cache->head_dim, elt_size(cache->dtype)};
  View vq;
  if ((st = view_of_heads(q, n, false, vq))) return st;
  const int heads = cache->num_kv_heads;
  if (vq.heads % heads) return SPEECHKV_ERR_INVALID_ARG;
  const int group = group_of(vq.heads, heads);
  if (group < 0 || max_cache_len > kMaxLen) return SPEECHKV_ERR_UNSUPPORTED;
  const int64_t lse_bytes = extent(batch, lse_stride_b, num_rows, lse_stride_s, vq.heads, lse_stride_h, 1, 4);
  if (lse_bytes < 0) return SPEECHKV_ERR_INVALID_ARG;
  WeightArgs a = {};
  a.row_tiles = (int)(((int64_t)num_rows * group + 15) / 16);
  a.batch = batch;
  a.cache = source_of(cache, cache_len, max_cache_len);
  plan_weights(a, n.dim, n.esz);
  // (with many rows a block has 512 threads: 2^32 of a launch are too many)
  if (((__int128)batch * heads + 7) * a.key_blocks > (a.row_tiles > kWeightFew ? kMaxBlocks / 2 : kMaxBlocks))
    return SPEECHKV_ERR_UNSUPPORTED;
  const int64_t pool = page_pool_bytes(cache), lens = (int64_t)batch * 4, sums = rows_bytes(batch, heads, capacity);
  if (sums < 0) return SPEECHKV_ERR_INVALID_ARG;
  const Region rd[] = {{vq.p, vq.bytes}, {lse, lse_bytes}, {visible, lens * num_rows}, {cache_len, lens},
                       {cache->block_table, table_bytes(cache, batch)}, {cache->k_pages, pool},
                       {weights == weights_out ? nullptr : weights, sums}};
  const Region wr[] = {{weights_out, sums}};
  if (aliased(wr, 1, rd, 7)) return SPEECHKV_ERR_ALIAS;
  if (max_cache_len == 0) return SPEECHKV_OK;  // (no entries)
  a.q = rows_of(vq);
  a.num_rows = num_rows;
  a.group_shift = log2_exact(group);
  a.lse = lse;
  a.lse_b = lse_stride_b;
  a.lse_h = lse_stride_h;
  a.lse_s = lse_stride_s;
  a.visible = visible;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.weights = weights;
  a.weights_out = weights_out;
  a.capacity = capacity;
  return status_of(launch_weights(a, cache->dtype, cache->head_dim, static_cast<hipStream_t>(stream)));
}

int speechkv_evict(const speechkv_evict_layer* layers, int32_t num_layers, int32_t batch, const int32_t* keep_len,
                   int32_t max_keep, int32_t capacity, int32_t num_first, int32_t num_recent, void* stream) {
  if (!layers || !keep_len) return SPEECHKV_ERR_INVALID_ARG;
  if (num_layers < 1 || num_layers > SPEECHKV_MAX_EVICT_LAYERS || batch < 1 || batch > kMaxGrid || max_keep < 1 ||
      capacity < 1 || num_first < 0 || num_recent < 0 || !aligned4(keep_len))
    return SPEECHKV_ERR_INVALID_ARG;
  const speechkv_paged_kv& first = layers[0].cache;
  for (int32_t i = 0; i < num_layers; ++i) {
    const speechkv_evict_layer& y = layers[i];
    const int st = check_cache(&y.cache);
    if (st) return st;
    if (!y.cache_len || !y.weights || !y.weights_out || !y.kept || !aligned4(y.cache_len) ||
        !aligned4(y.cache_len_out) || !aligned4(y.weights) || !aligned4(y.weights_out) || !aligned4(y.kept))
      return SPEECHKV_ERR_INVALID_ARG;
    if (y.cache.num_kv_heads != first.num_kv_heads || y.cache.head_dim != first.head_dim ||
        y.cache.dtype != first.dtype)
      return SPEECHKV_ERR_INVALID_ARG;
  }
  // every layer's written buffers against every layer's read ones and against the
  // other written ones (layers may share pools, so K pools are checked against V
  // pools only)
  const int64_t lens = (int64_t)batch * 4, sums = rows_bytes(batch, first.num_kv_heads, capacity);
  const int64_t lists = rows_bytes(batch, first.num_kv_heads, max_keep);
  if (sums < 0 || lists < 0) return SPEECHKV_ERR_INVALID_ARG;
  if (capacity > kMaxLen) return SPEECHKV_ERR_UNSUPPORTED;
  const int n = num_layers;
  auto k_pool = [&](int i) { return Region{layers[i].cache.k_pages, page_pool_bytes(&layers[i].cache)}; };
  auto v_pool = [&](int i) { return Region{layers[i].cache.v_pages, page_pool_bytes(&layers[i].cache)}; };
  auto out = [&](int i) { return Region{layers[i].weights_out, sums}; };
  auto in = [&](int i) { return Region{layers[i].weights == layers[i].weights_out ? nullptr : layers[i].weights, sums}; };
  auto kept = [&](int i) { return Region{layers[i].kept, lists}; };
  auto len_out = [&](int i) { return Region{layers[i].cache_len_out, lens}; };
  auto len = [&](int i) { return Region{layers[i].cache_len, lens}; };
  auto table = [&](int i) { return Region{layers[i].cache.block_table, table_bytes(&layers[i].cache, batch)}; };
  auto keep = [&](int) { return Region{keep_len, lens}; };
  auto pools_meet = [&](auto& x) { return meet(n, k_pool, n, x) || meet(n, v_pool, n, x); };
  auto reads_meet = [&](auto& x) { return meet(n, x, n, len) || meet(n, x, n, table) || meet(n, x, 1, keep) || meet(n, x, n, in); };
  if (meet(n, k_pool, n, v_pool) || pools_meet(out) || pools_meet(kept) || pools_meet(len_out) || reads_meet(k_pool) ||
      reads_meet(v_pool) || reads_meet(out) || reads_meet(kept) || reads_meet(len_out) || meet(n, out, n, kept) ||
      meet(n, out, n, len_out) || meet(n, kept, n, len_out))
    return SPEECHKV_ERR_ALIAS;
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (overlaps(out(i).p, sums, out(j).p, sums) || overlaps(kept(i).p, lists, kept(j).p, lists) ||
          (len_out(i).p && len_out(j).p && overlaps(len_out(i).p, lens, len_out(j).p, lens)))
        return SPEECHKV_ERR_ALIAS;
  EvictArgs a = {};
  a.keep_len = keep_len;
  a.max_keep = max_keep;
  a.capacity = capacity;
  a.num_first = num_first;
  a.num_recent = num_recent;
  a.kv_heads = first.num_kv_heads;
  for (int32_t at = 0; at < num_layers; at += kEvictLayers) {
    const int32_t some = std::min(num_layers - at, (int32_t)kEvictLayers);
    for (int32_t i = 0; i < some; ++i) {
      const speechkv_evict_layer& y = layers[at + i];
      EvictLayer& c = a.layer[i];
      c.k_pages = y.cache.k_pages;
      c.v_pages = y.cache.v_pages;
      c.table = y.cache.block_table;
      c.cache_len = y.cache_len;
      c.cache_len_out = y.cache_len_out;
      c.weights = y.weights;
      c.weights_out = y.weights_out;
      c.kept = y.kept;
      c.num_pages = y.cache.num_pages;
      c.page_shift = log2_exact(y.cache.page_size);
      c.max_pages = y.cache.max_pages_per_seq;
    }
    const hipError_t e = launch_evict(a, first.dtype, first.head_dim, some, batch, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return SPEECHKV_ERR_HIP;
  }
  return SPEECHKV_OK;
}

}  // extern "C"
