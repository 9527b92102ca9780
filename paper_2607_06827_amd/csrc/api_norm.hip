// C-ABI host layer of the per-head norms with rotation (include/speechkv_norm.h):
// argument validation, grid sizing and dispatch.  Every check runs before the
// first HIP call.
#include "../../include/speechkv_norm.h"

#include "head_views.hpp"
#include "kernels_norm.hpp"

namespace {

using namespace skv;

constexpr int kMaxAxes = 16;
constexpr float kLeastEps = 1.17549435e-38f;  // 2^-126

int check_sizes(int32_t batch, int32_t rows, const int32_t* row_len) {
  if (batch < 1 || batch > kMaxGrid || rows < 1 || !aligned4(row_len)) return SPEECHKV_ERR_INVALID_ARG;
  return (int64_t)batch * rows > kMaxBlocks ? SPEECHKV_ERR_UNSUPPORTED : SPEECHKV_OK;
}

int check_elements(int32_t head_dim, int32_t dtype) {
  return (head_dim == 64 || head_dim == 128) && (dtype == SPEECHKV_DTYPE_F32 || dtype == SPEECHKV_DTYPE_BF16)
             ? SPEECHKV_OK
             : SPEECHKV_ERR_UNSUPPORTED;
}

// The norm and the rotation, into a and the read regions from rd[at] on.
constexpr int kPlanRegions = 6;
int check_plan(const speechkv_head_norm* norm, const speechkv_rope* rope, const int32_t* row_len, const Sizes& n,
               NormArgs& a, Region* rd) {
  a.normalise = norm != nullptr;
  a.gamma_q = a.gamma_k = nullptr;
  a.eps = 0.f;
  if (norm) {
    if (!(norm->eps >= kLeastEps) || norm->eps > 3.0e38f) return SPEECHKV_ERR_INVALID_ARG;
    if (!aligned16(norm->gamma_q) || !aligned16(norm->gamma_k)) return SPEECHKV_ERR_INVALID_ARG;
    a.gamma_q = norm->gamma_q;
    a.gamma_k = norm->gamma_k;
    a.eps = norm->eps;
  }
  a.rot = a.pairs = a.num_axes = 0;
  a.positions = nullptr;
  a.inv_freq = nullptr;
  a.axis = nullptr;
  if (rope) {
    if (!rope->positions || !rope->inv_freq || rope->num_axes < 1 || rope->num_axes > kMaxAxes || rope->rot_dim < 16 ||
        rope->rot_dim > n.dim || rope->rot_dim % 16)
      return SPEECHKV_ERR_INVALID_ARG;
    if (rope->layout != SPEECHKV_ROPE_HALVES && rope->layout != SPEECHKV_ROPE_PAIRS) return SPEECHKV_ERR_INVALID_ARG;
    if (!aligned4(rope->positions) || !aligned4(rope->inv_freq) || !aligned4(rope->axis)) return SPEECHKV_ERR_INVALID_ARG;
    a.rot = rope->rot_dim;
    a.pairs = rope->layout == SPEECHKV_ROPE_PAIRS;
    a.num_axes = rope->num_axes;
    a.positions = rope->positions;
    a.inv_freq = rope->inv_freq;
    a.axis = rope->axis;
  }
  a.row_len = row_len;
  a.num_rows = n.rows;
  a.tokens = n.batch * n.rows;
  rd[0] = {row_len, (int64_t)n.batch * 4};
  rd[1] = {a.gamma_q, (int64_t)n.dim * 4};
  rd[2] = {a.gamma_k, (int64_t)n.dim * 4};
  rd[3] = {a.positions, (int64_t)a.num_axes * a.tokens * 4};
  rd[4] = {a.inv_freq, (int64_t)a.rot * 2};
  rd[5] = {a.axis, (int64_t)a.rot * 2};
  return SPEECHKV_OK;
}

}  // namespace

extern "C" {

int speechkv_norm_rope(const speechkv_heads* q, const speechkv_heads* k, int32_t batch, int32_t num_rows,
                       const int32_t* row_len, int32_t head_dim, int32_t dtype, const speechkv_head_norm* norm,
                       const speechkv_rope* rope, const speechkv_heads* q_out, const speechkv_heads* k_out,
                       void* stream) {
  if ((!q && !k) || (q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr))
    return SPEECHKV_ERR_INVALID_ARG;
  int st = check_elements(head_dim, dtype);
  if (st) return st;
  if ((st = check_sizes(batch, num_rows, row_len))) return st;
  const Sizes n = {batch, num_rows, head_dim, elt_size(dtype)};
  View vq, vk, oq, ok;
  if ((st = view_of_heads(q, n, false, vq)) || (st = view_of_heads(k, n, false, vk)) ||
      (st = view_of_heads(q_out, n, true, oq)) || (st = view_of_heads(k_out, n, true, ok)))
    return st;
  if (vq.heads != oq.heads || vk.heads != ok.heads) return SPEECHKV_ERR_INVALID_ARG;
  NormArgs a = {};
  Region rd[kPlanRegions];
  if ((st = check_plan(norm, rope, row_len, n, a, rd))) return st;
  if ((clash(oq, vq, n) && !same(oq, vq, n)) || (clash(ok, vk, n) && !same(ok, vk, n)) || clash(oq, vk, n) ||
      clash(ok, vq, n) || clash(oq, ok, n))
    return SPEECHKV_ERR_ALIAS;
  const Region wq[] = {region(oq)}, wk[] = {region(ok)};
  if (aliased(wq, 1, rd, kPlanRegions) || aliased(wk, 1, rd, kPlanRegions)) return SPEECHKV_ERR_ALIAS;
  a.q = rows_of(vq);
  a.k = rows_of(vk);
  a.q_out = rows_of(oq);
  a.k_out = rows_of(ok);
  a.q_heads = vq.heads;
  a.k_heads = vk.heads;
  return status_of(launch_norm(a, false, dtype, head_dim, static_cast<hipStream_t>(stream)));
}

size_t speechkv_norm_rope_bwd_workspace_bytes(int32_t batch, int32_t num_rows, int32_t num_q_heads,
                                              int32_t num_kv_heads, int32_t head_dim) {
  if (check_sizes(batch, num_rows, nullptr) || (head_dim != 64 && head_dim != 128) || num_q_heads < 0 ||
      num_kv_heads < 0 || num_q_heads > kMaxGrid || num_kv_heads > kMaxGrid || num_q_heads + num_kv_heads == 0)
    return 0;
  return (size_t)norm_bwd_blocks(batch * num_rows, num_q_heads, num_kv_heads, head_dim) * head_dim * sizeof(float);
}

int speechkv_norm_rope_bwd(const speechkv_heads* q, const speechkv_heads* k, const speechkv_heads* dq_out,
                           const speechkv_heads* dk_out, int32_t batch, int32_t num_rows, const int32_t* row_len,
                           int32_t head_dim, int32_t dtype, const speechkv_head_norm* norm, const speechkv_rope* rope,
                           const speechkv_heads* dq, const speechkv_heads* dk, float* dgamma_q, float* dgamma_k,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if ((!q && !k) || (q == nullptr) != (dq_out == nullptr) || (q == nullptr) != (dq == nullptr) ||
      (k == nullptr) != (dk_out == nullptr) || (k == nullptr) != (dk == nullptr))
    return SPEECHKV_ERR_INVALID_ARG;
  if ((dgamma_q && (!q || !norm)) || (dgamma_k && (!k || !norm)) || !aligned4(dgamma_q) || !aligned4(dgamma_k))
    return SPEECHKV_ERR_INVALID_ARG;
  int st = check_elements(head_dim, dtype);
  if (st) return st;
  if ((st = check_sizes(batch, num_rows, row_len))) return st;
  const Sizes n = {batch, num_rows, head_dim, elt_size(dtype)};
  View in[2], grad[2], out[2];
  if ((st = view_of_heads(q, n, false, in[0])) || (st = view_of_heads(k, n, false, in[1])) ||
      (st = view_of_heads(dq_out, n, false, grad[0])) || (st = view_of_heads(dk_out, n, false, grad[1])) ||
      (st = view_of_heads(dq, n, true, out[0])) || (st = view_of_heads(dk, n, true, out[1])))
    return st;
  NormArgs a = {};
  Region rd[kPlanRegions + 4];
  if ((st = check_plan(norm, rope, row_len, n, a, rd))) return st;
  const size_t need = dgamma_q || dgamma_k ? (size_t)norm_bwd_blocks(a.tokens, in[0].heads, in[1].heads, head_dim) *
                                                 head_dim * sizeof(float)
                                           : 0;
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return SPEECHKV_ERR_WORKSPACE;
  for (int x = 0; x < 2; ++x) {
    if (in[x].heads != grad[x].heads || in[x].heads != out[x].heads) return SPEECHKV_ERR_INVALID_ARG;
    if (clash(out[x], in[0], n) || clash(out[x], in[1], n) || clash(out[x], grad[1 - x], n) ||
        (clash(out[x], grad[x], n) && !same(out[x], grad[x], n)))
      return SPEECHKV_ERR_ALIAS;
  }
  if (clash(out[0], out[1], n)) return SPEECHKV_ERR_ALIAS;
  const Region sums[] = {{dgamma_q, (int64_t)head_dim * 4}, {dgamma_k, (int64_t)head_dim * 4},
                         {need ? workspace : nullptr, (int64_t)need}};
  for (int x = 0; x < 2; ++x) {
    const Region w[] = {region(out[x])};
    if (aliased(w, 1, rd, kPlanRegions) || aliased(w, 1, sums, 3)) return SPEECHKV_ERR_ALIAS;
    rd[kPlanRegions + 2 * x] = region(in[x]);
    rd[kPlanRegions + 2 * x + 1] = region(grad[x]);
  }
  if (aliased(sums, 3, rd, kPlanRegions + 4)) return SPEECHKV_ERR_ALIAS;
  a.q = rows_of(in[0]);
  a.k = rows_of(in[1]);
  a.q_out = rows_of(grad[0]);
  a.k_out = rows_of(grad[1]);
  a.dq = rows_of(out[0]);
  a.dk = rows_of(out[1]);
  a.q_heads = in[0].heads;
  a.k_heads = in[1].heads;
  a.partial = need ? static_cast<float*>(workspace) : nullptr;
  a.dgamma_q = dgamma_q;
  a.dgamma_k = dgamma_k;
  return status_of(launch_norm_bwd(a, dtype, head_dim, static_cast<hipStream_t>(stream)));
}

int speechkv_norm_append_kv(const speechkv_heads* q, const speechkv_heads* k, const speechkv_heads* v, int32_t batch,
                            int32_t num_rows, const int32_t* row_len, const speechkv_head_norm* norm,
                            const speechkv_rope* rope, const int32_t* cache_len, const speechkv_paged_kv* cache,
                            const speechkv_heads* q_out, int32_t* cache_len_out, void* stream) {
  if (!k || !v || !cache_len || (q == nullptr) != (q_out == nullptr)) return SPEECHKV_ERR_INVALID_ARG;
  int st = check_cache(cache);
  if (st) return st;
  if ((st = check_sizes(batch, num_rows, row_len))) return st;
  const Sizes n = {batch, num_rows, cache->head_dim, elt_size(cache->dtype)};
  View vq, vk, vv, oq;
  if ((st = view_of_heads(q, n, false, vq)) || (st = view_of_heads(k, n, false, vk)) ||
      (st = view_of_heads(v, n, false, vv)) || (st = view_of_heads(q_out, n, true, oq)))
    return st;
  if (vq.heads != oq.heads || vk.heads != cache->num_kv_heads || vv.heads != cache->num_kv_heads ||
      !aligned4(cache_len) || !aligned4(cache_len_out))
    return SPEECHKV_ERR_INVALID_ARG;
  NormArgs a = {};
  Region rd[kPlanRegions + 5];
  if ((st = check_plan(norm, rope, row_len, n, a, rd))) return st;
  if ((clash(oq, vq, n) && !same(oq, vq, n)) || clash(oq, vk, n) || clash(oq, vv, n)) return SPEECHKV_ERR_ALIAS;
  const int64_t pool = page_pool_bytes(cache), lens = (int64_t)batch * 4;
  rd[kPlanRegions] = {cache_len, lens};
  rd[kPlanRegions + 1] = {cache->block_table, table_bytes(cache, batch)};
  const Region wq[] = {region(oq)};
  if (aliased(wq, 1, rd, kPlanRegions + 2)) return SPEECHKV_ERR_ALIAS;
  rd[kPlanRegions + 2] = region(vk);
  rd[kPlanRegions + 3] = region(vv);
  rd[kPlanRegions + 4] = region(vq);
  const Region wr[] = {{cache->k_pages, pool}, {cache->v_pages, pool}, {cache_len_out, lens}};
  if (aliased(wr, 3, rd, kPlanRegions + 5) || aliased(wr, 3, wq, 1)) return SPEECHKV_ERR_ALIAS;
  a.q = rows_of(vq);
  a.k = rows_of(vk);
  a.v = rows_of(vv);
  a.q_out = rows_of(oq);
  a.q_heads = vq.heads;
  a.k_heads = vk.heads;
  a.cache_len = cache_len;
  a.k_pages = cache->k_pages;
  a.v_pages = cache->v_pages;
  a.table = cache->block_table;
  a.pv = view_of(cache);
  a.cache_len_out = cache_len_out;
  return status_of(launch_norm(a, true, cache->dtype, cache->head_dim, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
