// C-ABI host layer of the steps of several new tokens
// (include/speechkv_draft.h): argument validation, grid sizing and dispatch.
// Every check runs before the first HIP call.
#include "../../include/speechkv_draft.h"

#include <algorithm>
#include <cmath>

#include "host_checks.hpp"
#include "kernels_draft.hpp"

namespace {

using namespace skv;

// Most blocks of 256 threads along one axis of a launch (its threads are counted
// in 32 bits).
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 1;

// The kernels hold a mask row's words and a path's entries in LDS arrays.
static_assert(32 * kMaskWords >= SPEECHKV_MAX_TREE_NODES && kCommitPath >= SPEECHKV_MAX_TREE_NODES,
              "arrays of a tree's nodes");

// Longest cache of speechkv_tree_attn: the kernel's key numbers, with the nodes
// and the tiles that it looks ahead, stay in 31 bits.  (Splits are whole tiles,
// so many of them reach further; those calls are checked by their own numbers.)
constexpr int32_t kMaxTreeLen = INT32_MAX - 8191;

// Bytes from the first to past the last element of a strided [batch][rows]
// [heads][dim] tensor, or -1 when they do not fit 2^62 (no tensor is so long).
int64_t extent(int64_t batch, int64_t sb, int64_t rows, int64_t ss, int64_t heads, int64_t sh, int64_t dim,
               int64_t elt) {
  const __int128 n = ((__int128)(batch - 1) * sb + (__int128)(rows - 1) * ss + (__int128)(heads - 1) * sh + dim) * elt;
  return n < ((__int128)1 << 62) ? (int64_t)n : -1;
}

bool bad_stride(int64_t s, int64_t per16) { return s < 0 || s % per16; }

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Whether a region of one list overlaps a region of another (null ones take no
// part).  Lists that lie apart as a whole, as pools and lengths mostly do, are
// not compared pair by pair.
template <typename A, typename B>
bool meet(int na, const A& a, int nb, const B& b) {
  uintptr_t a_lo = UINTPTR_MAX, a_hi = 0, b_lo = UINTPTR_MAX, b_hi = 0;
  for (int i = 0; i < na; ++i) {
    const Region x = a(i);
    if (!x.p) continue;
    a_lo = std::min(a_lo, (uintptr_t)x.p);
    a_hi = std::max(a_hi, (uintptr_t)x.p + (uintptr_t)x.n);
  }
  for (int i = 0; i < nb; ++i) {
    const Region x = b(i);
    if (!x.p) continue;
    b_lo = std::min(b_lo, (uintptr_t)x.p);
    b_hi = std::max(b_hi, (uintptr_t)x.p + (uintptr_t)x.n);
  }
  if (a_hi <= b_lo || b_hi <= a_lo) return false;
  for (int i = 0; i < na; ++i) {
    const Region x = a(i);
    for (int j = 0; x.p && j < nb; ++j) {
      const Region y = b(j);
      if (y.p && overlaps(x.p, x.n, y.p, y.n)) return true;
    }
  }
  return false;
}

int64_t table_bytes(const speechkv_paged_kv* c, int32_t batch) { return (int64_t)batch * c->max_pages_per_seq * 4; }

// How speechkv_tree_attn cuts a call: row groups of a block (1, 2 or 4, of 32
// rows each) and splits of the keys.
struct TreePlan {
  int groups, splits;
};

// Bytes of the splits' partial rows: fp32 sums, then (running maximum, weight
// sum) pairs.
size_t tree_partial_bytes(int32_t batch, int32_t nodes, int32_t q_heads, int32_t head_dim, int32_t splits) {
  return splits <= 1 ? 0 : (size_t)batch * nodes * q_heads * splits * (head_dim + 2) * sizeof(float);
}

// The plan with the smallest estimated time: of the given split count, or with
// 0 of those whose partial rows fit `room` bytes.  (The best count falls where a
// longer axis or more sequences fill the chip, so room for the largest call may
// be too little for a smaller one's.)
// The estimate is fitted to a sweep on MI355X over 24 shapes of 1 to 64
// sequences, 1 to 8 KV heads, 4 to 1000 nodes and 30 to 7692 keys (bf16, 128
// wide; the best of 1, 2 or 4 groups and of the split counts below is met
// within 2% on average, 9% at most) and checked on 6 more of fp32 and 64-wide
// heads (14% at most).  In us:
//  - a launch and the first loads take 4.7, a block 1.3 and a step of one tile
//    per stream about 1 (fp32 steps, bound by their products, 4.4 a 128-wide
//    tile); the blocks that fit the chip run at once;
//  - a key is read from HBM at 7 TB/s, and read again by every further row tile
//    at a third of the cost: 64 rows of 7692 keys of 16 sequences take 89 us
//    in one tile of 64, 108 in two of 32;
//  - a wave's tile occupies its SIMD for 0.49;
//  - splits cost 3.2 for the merge and the write and read of their fp32
//    partial rows at 10 TB/s: one sequence of 7692 keys takes 71 us whole and
//    16 in 16 splits, 64 sequences of 300 keys 19 us whole and 32 in two.
TreePlan tree_plan(int batch, int nodes, int group, int kv_heads, int head_dim, int dtype, int max_len, int splits,
                   size_t room) {
  const bool f32 = dtype == SPEECHKV_DTYPE_F32, wide = head_dim == 128;
  const double rows = (double)nodes * group, units = (double)batch * kv_heads, size = head_dim / 128.0;
  const int64_t tiles = ((int64_t)max_len + nodes + kTreeKeys - 1) / kTreeKeys;
  const double row_bytes = head_dim * (f32 ? 4.0 : 2.0);
  const double keys_us = units * tiles * kTreeKeys * 2 * row_bytes / 7.0e6;
  const double rows_us = units * rows * 2 * row_bytes / 7.0e6;
  const double busy_us = f32 ? 3.5 * size : wide ? 0.49 : 0.35;
  static const int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  TreePlan best = {1, splits ? splits : 1};
  double best_us = 1e300;
  for (int groups = 1; groups <= 4 && (groups == 1 || rows > 16 * groups); groups *= 2) {
    const double row_tiles = tree_row_tiles((int64_t)nodes * group, groups);
    const double step_us = f32 ? 4.4 * size : (groups == 1 ? 1.07 : groups == 2 ? 1.23 : 0.95) * (wide ? 1.0 : 0.8);
    const double slots = 256.0 * (f32 && wide ? 1 : !f32 && !wide ? 4 : groups == 4 ? 3 : 2);
    const double read_us = keys_us * (1 + 0.33 * (row_tiles - 1)) + rows_us;
    const double work_us = units * row_tiles * groups * tiles * busy_us / 1024;
    for (int i = 0; i < 10; ++i) {
      const int s = splits ? splits : counts[i];
      if (!splits && (s > tiles || tree_partial_bytes(batch, nodes, group * kv_heads, head_dim, s) > room)) break;
      const double steps = (double)(((tiles + s - 1) / s * groups + 3) / 4);
      const double full = units * row_tiles * s / slots;
      const double rounds = full >= 4 ? full + 0.5 : std::max(1.0, std::ceil(full));
      const double us = std::max({rounds * (1.3 + step_us * steps), 1.3 + read_us, 1.3 + work_us}) +
                        (s > 1 ? 3.2 + units * rows * s * head_dim * 16 / 10.2e6 : 0.0);
      if (us < best_us) {
        best_us = us;
        best = {groups, s};
      }
      if (splits) break;
    }
  }
  return best;
}

}  // namespace

extern "C" {

int speechkv_append_kv(const void* q, int64_t q_stride_b, int64_t q_stride_s, int64_t q_stride_h,
                       int32_t num_q_heads, const void* k, const void* v, int64_t stride_b, int64_t stride_s,
                       int64_t stride_h, int32_t batch, int32_t num_new, const int32_t* new_len,
                       const int32_t* positions, const float* inv_freq, int32_t rot_dim, int32_t rope,
                       const int32_t* cache_len, const speechkv_paged_kv* cache, void* q_out,
                       int32_t* cache_len_out, void* stream) {
  if (!k || !v || !cache_len || (q == nullptr) != (q_out == nullptr)) return SPEECHKV_ERR_INVALID_ARG;
  const int st = check_cache(cache);
  if (st) return st;
  if (batch < 1 || batch > kMaxGrid || num_new < 1 || num_new > kMaxBlocks) return SPEECHKV_ERR_INVALID_ARG;
  if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 16) return SPEECHKV_ERR_INVALID_ARG;
  if (rope != SPEECHKV_ROPE_HALVES && rope != SPEECHKV_ROPE_PAIRS) return SPEECHKV_ERR_INVALID_ARG;
  if (rot_dim && (!positions || !inv_freq)) return SPEECHKV_ERR_INVALID_ARG;
  if (q) {
    if (num_q_heads < 1 || num_q_heads % cache->num_kv_heads) return SPEECHKV_ERR_INVALID_ARG;
    if (group_of(num_q_heads, cache->num_kv_heads) < 0) return SPEECHKV_ERR_UNSUPPORTED;
  }
  const int esz = elt_size(cache->dtype), D = cache->head_dim;
  const int64_t per16 = 16 / esz;
  if (bad_stride(stride_b, per16) || bad_stride(stride_s, per16) || bad_stride(stride_h, per16))
    return SPEECHKV_ERR_INVALID_ARG;
  if (q && (bad_stride(q_stride_b, per16) || bad_stride(q_stride_s, per16) || bad_stride(q_stride_h, per16)))
    return SPEECHKV_ERR_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out)) return SPEECHKV_ERR_INVALID_ARG;
  if (!aligned4(new_len) || !aligned4(positions) || !aligned4(inv_freq) || !aligned4(cache_len) ||
      !aligned4(cache_len_out))
    return SPEECHKV_ERR_INVALID_ARG;
  const int64_t kv_bytes = extent(batch, stride_b, num_new, stride_s, cache->num_kv_heads, stride_h, D, esz);
  const int64_t q_bytes = q ? extent(batch, q_stride_b, num_new, q_stride_s, num_q_heads, q_stride_h, D, esz) : 0;
  const int64_t out_bytes =
      q ? extent(batch, (int64_t)num_new * num_q_heads * D, num_new, (int64_t)num_q_heads * D, num_q_heads, D, D, esz)
        : 0;
  if (kv_bytes < 0 || q_bytes < 0 || out_bytes < 0) return SPEECHKV_ERR_INVALID_ARG;
  // the queries may be rotated in place: a thread reads what it writes (a
  // stride along an axis of length 1 does not matter)
  const bool in_place = q && q == q_out && (num_q_heads == 1 || q_stride_h == D) &&
                        (num_new == 1 || q_stride_s == (int64_t)num_q_heads * D) &&
                        (batch == 1 || q_stride_b == (int64_t)num_new * num_q_heads * D);
  const int64_t pool = page_pool_bytes(cache), lens = (int64_t)batch * 4;
  const Region rd[] = {{in_place ? nullptr : q, q_bytes}, {k, kv_bytes}, {v, kv_bytes}, {new_len, lens},
                       {rot_dim ? positions : nullptr, lens * num_new},
                       {rot_dim ? inv_freq : nullptr, (int64_t)rot_dim * 2}, {cache_len, lens},
                       {cache->block_table, table_bytes(cache, batch)}};
  const Region wr[] = {{cache->k_pages, pool}, {cache->v_pages, pool}, {q_out, out_bytes}, {cache_len_out, lens}};
  if (aliased(wr, 4, rd, 8)) return SPEECHKV_ERR_ALIAS;
  AppendArgs a;
  a.q = q;
  a.q_stride_b = q_stride_b;
  a.q_stride_s = q_stride_s;
  a.q_stride_h = q_stride_h;
  a.num_q_heads = q ? num_q_heads : 0;
  a.k = k;
  a.v = v;
  a.stride_b = stride_b;
  a.stride_s = stride_s;
  a.stride_h = stride_h;
  a.num_new = num_new;
  a.new_len = new_len;
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.rot = rot_dim;
  a.pairs = rope == SPEECHKV_ROPE_PAIRS;
  a.cache_len = cache_len;
  a.k_pages = cache->k_pages;
  a.v_pages = cache->v_pages;
  a.table = cache->block_table;
  a.pv = view_of(cache);
  a.q_out = q_out;
  a.cache_len_out = cache_len_out;
  return status_of(launch_append(a, cache->dtype, D, batch, static_cast<hipStream_t>(stream)));
}

int32_t speechkv_tree_num_splits(int32_t batch, int32_t num_nodes, int32_t num_q_heads, int32_t num_kv_heads,
                                 int32_t head_dim, int32_t dtype, int32_t max_cache_len) {
  if (batch < 1 || num_nodes < 1 || num_nodes > SPEECHKV_MAX_TREE_NODES || num_kv_heads < 1 || max_cache_len < 0 ||
      (head_dim != 64 && head_dim != 128) || (dtype != SPEECHKV_DTYPE_F32 && dtype != SPEECHKV_DTYPE_BF16))
    return -1;
  const int group = group_of(num_q_heads, num_kv_heads);
  if (group < 0) return -1;
  return tree_plan(batch, num_nodes, group, num_kv_heads, head_dim, dtype, max_cache_len, 0, SIZE_MAX).splits;
}

size_t speechkv_tree_workspace_bytes(int32_t batch, int32_t num_nodes, int32_t num_q_heads, int32_t num_kv_heads,
                                     int32_t head_dim, int32_t max_cache_len, int32_t num_splits) {
  if (num_splits < 0) return 0;
  const int32_t f32 = speechkv_tree_num_splits(batch, num_nodes, num_q_heads, num_kv_heads, head_dim,
                                               SPEECHKV_DTYPE_F32, max_cache_len);
  const int32_t bf16 = speechkv_tree_num_splits(batch, num_nodes, num_q_heads, num_kv_heads, head_dim,
                                                SPEECHKV_DTYPE_BF16, max_cache_len);
  if (f32 < 0) return 0;
  return tree_partial_bytes(batch, num_nodes, num_q_heads, head_dim, num_splits ? num_splits : std::max(f32, bf16));
}

int speechkv_tree_attn(const void* q, int32_t batch, int32_t num_nodes, int32_t num_q_heads,
                       const speechkv_paged_kv* cache, const int32_t* cache_len, int32_t max_cache_len,
                       const int32_t* num_nodes_of, const uint32_t* tree_mask, int64_t mask_stride_b, float scale,
                       int32_t num_splits, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !out || !cache_len) return SPEECHKV_ERR_INVALID_ARG;
  const int st = check_cache(cache);
  if (st) return st;
  if (batch < 1 || batch > kMaxGrid || num_nodes < 1 || num_nodes > SPEECHKV_MAX_TREE_NODES || max_cache_len < 0 ||
      num_splits < 0 || num_splits > kMaxGrid)
    return SPEECHKV_ERR_INVALID_ARG;
  if (!(scale > 0.f) || scale > 3.0e38f) return SPEECHKV_ERR_INVALID_ARG;  // finite, > 0
  if ((int64_t)max_cache_len > (int64_t)cache->max_pages_per_seq * cache->page_size) return SPEECHKV_ERR_INVALID_ARG;
  if (num_q_heads < 1 || num_q_heads % cache->num_kv_heads) return SPEECHKV_ERR_INVALID_ARG;
  const int group = group_of(num_q_heads, cache->num_kv_heads);
  if (group < 0 || max_cache_len > kMaxTreeLen) return SPEECHKV_ERR_UNSUPPORTED;
  if (tree_mask && (mask_stride_b < 0 || mask_stride_b > ((int64_t)1 << 40))) return SPEECHKV_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned4(cache_len) || !aligned4(num_nodes_of) || !aligned4(tree_mask))
    return SPEECHKV_ERR_INVALID_ARG;
  const TreePlan plan = tree_plan(batch, num_nodes, group, cache->num_kv_heads, cache->head_dim, cache->dtype,
                                  max_cache_len, num_splits, workspace ? workspace_bytes : 0);
  const int32_t splits = plan.splits;
  const size_t need = tree_partial_bytes(batch, num_nodes, num_q_heads, cache->head_dim, splits);
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return SPEECHKV_ERR_WORKSPACE;
  const int row_tiles = tree_row_tiles((int64_t)num_nodes * group, plan.groups);
  if (((int64_t)batch * cache->num_kv_heads * splits + 7) * row_tiles > kMaxBlocks) return SPEECHKV_ERR_UNSUPPORTED;
  if (splits > 1 && (int64_t)num_nodes * num_q_heads > kMaxBlocks * tree_merge_rows(cache->head_dim))
    return SPEECHKV_ERR_UNSUPPORTED;
  const int64_t tiles = ((int64_t)max_cache_len + num_nodes + kTreeKeys - 1) / kTreeKeys;
  const int64_t tiles_per_split = (tiles + splits - 1) / splits;
  if ((tiles_per_split * splits + kTreeAhead) * kTreeKeys > (int64_t)INT32_MAX + 1) return SPEECHKV_ERR_UNSUPPORTED;
  const int words = (num_nodes + 31) / 32;
  const int64_t qo = (int64_t)batch * num_nodes * num_q_heads * cache->head_dim * elt_size(cache->dtype);
  const int64_t pool = page_pool_bytes(cache), lens = (int64_t)batch * 4;
  const Region rd[] = {{q, qo}, {cache_len, lens}, {num_nodes_of, lens},
                       {tree_mask, ((int64_t)(batch - 1) * mask_stride_b + (int64_t)num_nodes * words) * 4},
                       {cache->block_table, table_bytes(cache, batch)}, {cache->k_pages, pool}, {cache->v_pages, pool}};
  const Region wr[] = {{out, qo}, {need ? workspace : nullptr, (int64_t)need}};
  if (aliased(wr, 2, rd, 7)) return SPEECHKV_ERR_ALIAS;
  TreeArgs a;
  a.q = q;
  a.k_pages = cache->k_pages;
  a.v_pages = cache->v_pages;
  a.table = cache->block_table;
  a.pv = view_of(cache);
  a.cache_len = cache_len;
  a.max_len = max_cache_len;
  a.num_nodes = num_nodes;
  a.nodes_of = num_nodes_of;
  a.mask = tree_mask;
  a.mask_stride = mask_stride_b;
  a.mask_words = words;
  a.num_q_heads = num_q_heads;
  a.group_shift = log2_exact(group);
  a.row_groups = plan.groups;
  a.row_tiles = row_tiles;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.num_splits = splits;
  a.tiles_per_split = (int)tiles_per_split;
  a.out = out;
  a.ws_o = nullptr;
  a.ws_ml = nullptr;
  if (splits > 1) {
    a.ws_o = static_cast<float*>(workspace);
    a.ws_ml = a.ws_o + (size_t)batch * num_nodes * num_q_heads * splits * cache->head_dim;
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = launch_tree(a, cache->dtype, cache->head_dim, batch, s);
  if (e == hipSuccess && splits > 1) e = launch_tree_merge(a, cache->dtype, cache->head_dim, batch, s);
  return status_of(e);
}

int speechkv_tree_commit(const speechkv_layer_cache* layers, int32_t num_layers, int32_t batch, const int32_t* path,
                         int32_t max_path, const int32_t* path_len, int32_t num_nodes, void* stream) {
  if (!layers || !path || !path_len) return SPEECHKV_ERR_INVALID_ARG;
  if (num_layers < 1 || num_layers > SPEECHKV_MAX_COMMIT_LAYERS || batch < 1 || batch > kMaxGrid || num_nodes < 1 ||
      num_nodes > SPEECHKV_MAX_TREE_NODES || max_path < 1 || max_path > num_nodes)
    return SPEECHKV_ERR_INVALID_ARG;
  if (!aligned4(path) || !aligned4(path_len)) return SPEECHKV_ERR_INVALID_ARG;
  const speechkv_paged_kv& first = layers[0].cache;
  const int64_t lens = (int64_t)batch * 4;
  for (int32_t i = 0; i < num_layers; ++i) {
    const speechkv_layer_cache& y = layers[i];
    const int st = check_cache(&y.cache);
    if (st) return st;
    if (!y.cache_len || !aligned4(y.cache_len) || !aligned4(y.cache_len_out)) return SPEECHKV_ERR_INVALID_ARG;
    if (y.cache.num_kv_heads != first.num_kv_heads || y.cache.head_dim != first.head_dim ||
        y.cache.dtype != first.dtype)
      return SPEECHKV_ERR_INVALID_ARG;
  }
  // every layer's written buffers against every layer's read ones and against the
  // other written ones (layers may share pools, so K pools are checked against V
  // pools only)
  auto k_pool = [&](int i) { return Region{layers[i].cache.k_pages, page_pool_bytes(&layers[i].cache)}; };
  auto v_pool = [&](int i) { return Region{layers[i].cache.v_pages, page_pool_bytes(&layers[i].cache)}; };
  auto out = [&](int i) { return Region{layers[i].cache_len_out, lens}; };
  auto len = [&](int i) { return Region{layers[i].cache_len, lens}; };
  auto table = [&](int i) { return Region{layers[i].cache.block_table, table_bytes(&layers[i].cache, batch)}; };
  auto paths = [&](int i) { return i ? Region{path_len, lens} : Region{path, lens * max_path}; };
  const int n = num_layers;
  if (meet(n, k_pool, n, v_pool) || meet(n, k_pool, n, out) || meet(n, v_pool, n, out) || meet(n, k_pool, n, len) ||
      meet(n, v_pool, n, len) || meet(n, out, n, len) || meet(n, k_pool, n, table) || meet(n, v_pool, n, table) ||
      meet(n, out, n, table) || meet(n, k_pool, 2, paths) || meet(n, v_pool, 2, paths) || meet(n, out, 2, paths))
    return SPEECHKV_ERR_ALIAS;
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (out(i).p && out(j).p && overlaps(out(i).p, lens, out(j).p, lens)) return SPEECHKV_ERR_ALIAS;
  CommitArgs a;
  a.path = path;
  a.path_len = path_len;
  a.max_path = max_path;
  a.num_nodes = num_nodes;
  a.kv_heads = first.num_kv_heads;
  for (int32_t at = 0; at < num_layers; at += kCommitLayers) {
    const int32_t some = std::min(num_layers - at, (int32_t)kCommitLayers);
    for (int32_t i = 0; i < some; ++i) {
      const speechkv_layer_cache& y = layers[at + i];
      CommitLayer& c = a.layer[i];
      c.k_pages = y.cache.k_pages;
      c.v_pages = y.cache.v_pages;
      c.table = y.cache.block_table;
      c.cache_len = y.cache_len;
      c.cache_len_out = y.cache_len_out;
      c.num_pages = y.cache.num_pages;
      c.page_shift = log2_exact(y.cache.page_size);
      c.max_pages = y.cache.max_pages_per_seq;
    }
    const hipError_t e = launch_commit(a, first.dtype, first.head_dim, some, batch, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return SPEECHKV_ERR_HIP;
  }
  return SPEECHKV_OK;
}

}  // extern "C"
