// Argument checks shared by the C-ABI host files of libspeechkv.  Host code only;
// nothing here calls HIP.
#pragma once

#include "../../include/speechkv.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "common.hpp"

namespace skv {

constexpr int kMaxGrid = 65535;
constexpr int kMaxRows = 2147483647 - SPEECHKV_MAX_WINDOW;  // ceil(T / w) stays in int32

// Most blocks of 256 threads along one axis of a launch (its threads are counted
// in 32 bits).
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 1;

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

inline int64_t table_bytes(const speechkv_paged_kv* c, int32_t batch) { return (int64_t)batch * c->max_pages_per_seq * 4; }

// Bytes from the first to past the last element of a strided [batch][rows]
// [heads][dim] tensor, or -1 when they do not fit 2^62 (no tensor is so long).
inline int64_t extent(int64_t batch, int64_t sb, int64_t rows, int64_t ss, int64_t heads, int64_t sh, int64_t dim,
               int64_t elt) {
  const __int128 n = ((__int128)(batch - 1) * sb + (__int128)(rows - 1) * ss + (__int128)(heads - 1) * sh + dim) * elt;
  return n < ((__int128)1 << 62) ? (int64_t)n : -1;
}

inline bool bad_stride(int64_t s, int64_t per16) { return s < 0 || s % per16; }

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

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

}  // namespace skv
