// The strided tensors of a call (speechkv_heads of include/speechkv_norm.h), as the
// host layer checks them.  Host code only; nothing here calls HIP.
#pragma once

#include "../../include/speechkv_norm.h"

#include <algorithm>
#include <utility>

#include "host_checks.hpp"
#include "kernels_norm.hpp"

namespace skv {

// The sizes that the views of a call share.
struct Sizes {
  int32_t batch, rows, dim, esz;
};

// A strided tensor of a call; null data takes no part.
struct View {
  const void* p = nullptr;
  int64_t sb = 0, ss = 0, sh = 0, bytes = 0;
  int32_t heads = 0;
};

// Fills v from h; what a written one's axes overlap is refused.
inline int view_of_heads(const speechkv_heads* h, const Sizes& n, bool written, View& v) {
  if (!h) return SPEECHKV_OK;
  const int64_t per16 = 16 / n.esz;
  if (!h->data || !aligned16(h->data) || h->num_heads < 1 || h->num_heads > kMaxGrid) return SPEECHKV_ERR_INVALID_ARG;
  if (bad_stride(h->stride_b, per16) || bad_stride(h->stride_s, per16) || bad_stride(h->stride_h, per16))
    return SPEECHKV_ERR_INVALID_ARG;
  const int64_t bytes = extent(n.batch, h->stride_b, n.rows, h->stride_s, h->num_heads, h->stride_h, n.dim, n.esz);
  if (bytes < 0) return SPEECHKV_ERR_INVALID_ARG;
  if (written) {
    std::pair<int64_t, int32_t> axis[3] = {
        {h->stride_b, n.batch}, {h->stride_s, n.rows}, {h->stride_h, h->num_heads}};
    std::sort(axis, axis + 3);
    int64_t span = n.dim;  // (fits: it is at most the extent)
    for (const auto& [stride, length] : axis) {
      if (length == 1) continue;
      if (stride < span) return SPEECHKV_ERR_INVALID_ARG;
      span += stride * (length - 1);
    }
  }
  v.p = h->data;
  v.sb = h->stride_b;
  v.ss = h->stride_s;
  v.sh = h->stride_h;
  v.bytes = bytes;
  v.heads = h->num_heads;
  return SPEECHKV_OK;
}

// One tensor with one set of strides (those of axes of length 1 do not matter).
inline bool same(const View& a, const View& b, const Sizes& n) {
  return a.p == b.p && a.heads == b.heads && (n.batch == 1 || a.sb == b.sb) && (n.rows == 1 || a.ss == b.ss) &&
         (a.heads == 1 || a.sh == b.sh);
}

// Views whose byte ranges meet but whose rows do not.  Both go in the same steps along
// some of the outer axes (sequences, rows, or both), and of each such step b's part (the
// axes that are left, and the heads) lies behind a's, before a's next: heads of one
// projection's output in any order of its axes.
inline bool beside(const View& a, const View& b, const Sizes& n) {
  const int64_t off = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  if (off < 0 || off % n.esz) return false;
  const int64_t d = off / n.esz;
  for (const auto& [by_batch, by_rows] : {std::pair(true, true), std::pair(true, false), std::pair(false, true)}) {
    if ((by_batch && n.batch > 1 && a.sb != b.sb) || (by_rows && n.rows > 1 && a.ss != b.ss)) continue;
    auto part = [&](const View& v) {
      return (v.heads - 1) * v.sh + n.dim + (by_batch ? 0 : (n.batch - 1) * v.sb) + (by_rows ? 0 : (n.rows - 1) * v.ss);
    };
    if (d < part(a)) continue;
    // (the steps nested, as those of a written view)
    std::pair<int64_t, int32_t> axis[2] = {{a.sb, by_batch ? n.batch : 1}, {a.ss, by_rows ? n.rows : 1}};
    std::sort(axis, axis + 2);
    int64_t span = d + part(b);  // what a step of both takes
    bool nested = true;
    for (const auto& [stride, length] : axis) {
      if (length == 1) continue;
      nested = nested && stride >= span;
      span += stride * (length - 1);
    }
    if (nested) return true;
  }
  return false;
}

inline bool clash(const View& a, const View& b, const Sizes& n) {
  return a.p && b.p && overlaps(a.p, a.bytes, b.p, b.bytes) && !beside(a, b, n) && !beside(b, a, n);
}

inline Region region(const View& v) { return {v.p, v.bytes}; }

inline HeadRows rows_of(const View& v) { return {const_cast<void*>(v.p), v.sb, v.ss, v.sh}; }

}  // namespace skv
