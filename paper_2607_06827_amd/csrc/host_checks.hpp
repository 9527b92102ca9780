// Argument checks shared by the C-ABI host files of libspeechkv.  Host code only;
// nothing here calls HIP.
#pragma once

#include "../../include/speechkv.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace skv {

constexpr int kMaxGrid = 65535;
constexpr int kMaxRows = 2147483647 - SPEECHKV_MAX_WINDOW;  // ceil(T / w) stays in int32

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int elt_size(int dtype) { return dtype == SPEECHKV_DTYPE_BF16 ? 2 : 4; }

inline int log2_exact(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return (1 << s) == x ? s : -1;
}

// Checks shared by every call on the cache description.
inline int check_cache(const speechkv_paged_kv* c) {
  if (!c || !c->k_pages || !c->v_pages || !c->block_table) return SPEECHKV_ERR_INVALID_ARG;
  if (c->num_pages < 1 || c->max_pages_per_seq < 1 || c->num_kv_heads < 1)
    return SPEECHKV_ERR_INVALID_ARG;
  if (c->dtype != SPEECHKV_DTYPE_F32 && c->dtype != SPEECHKV_DTYPE_BF16) return SPEECHKV_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return SPEECHKV_ERR_UNSUPPORTED;
  if (c->page_size < 8 || c->page_size > 256 || log2_exact(c->page_size) < 0)
    return SPEECHKV_ERR_UNSUPPORTED;
  if (c->num_kv_heads > kMaxGrid) return SPEECHKV_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages_per_seq * c->page_size > INT32_MAX) return SPEECHKV_ERR_INVALID_ARG;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return SPEECHKV_ERR_INVALID_ARG;
  return SPEECHKV_OK;
}

inline PagedView view_of(const speechkv_paged_kv* c) {
  PagedView v;
  v.num_pages = c->num_pages;
  v.page_shift = log2_exact(c->page_size);
  v.max_pages = c->max_pages_per_seq;
  v.kv_heads = c->num_kv_heads;
  return v;
}

inline int group_of(int num_q_heads, int num_kv_heads) {
  if (num_q_heads < 1 || num_q_heads % num_kv_heads) return -1;
  const int g = num_q_heads / num_kv_heads;
  return (g == 1 || g == 2 || g == 4 || g == 8) ? g : -1;
}

inline int64_t page_pool_bytes(const speechkv_paged_kv* c) {
  return (int64_t)c->num_pages * c->num_kv_heads * c->page_size * c->head_dim * elt_size(c->dtype);
}

inline bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}

inline int status_of(hipError_t e) { return e == hipSuccess ? SPEECHKV_OK : SPEECHKV_ERR_HIP; }

// A byte range of one argument; a null pointer takes no part in the checks.
struct Region {
  const void* p;
  int64_t n;
};

// True when a written region overlaps a read region or another written one.
inline bool aliased(const Region* wr, int nw, const Region* rd, int nr) {
  for (int i = 0; i < nw; ++i) {
    if (!wr[i].p) continue;
    for (int k = 0; k < nr; ++k)
      if (rd[k].p && overlaps(wr[i].p, wr[i].n, rd[k].p, rd[k].n)) return true;
    for (int k = i + 1; k < nw; ++k)
      if (wr[k].p && overlaps(wr[i].p, wr[i].n, wr[k].p, wr[k].n)) return true;
  }
  return false;
}

}  // namespace skv
