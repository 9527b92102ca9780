// New keys and values behind a sequence's cache entries, the keys and the
// queries rotated by their positions on the way.
//
// With the angle a_j = position * inv_freq[j], the pair number j of a head
// turns to (x cos a_j - y sin a_j, x sin a_j + y cos a_j).  An angle is a
// number of turns whose whole part drops out: the product and the reduction
// are done in 64 bits, so the fp32 sine and cosine see half a turn at most and
// an error of 2^-25 turns, however far the position.
//
// A block moves one token, a thread two 8-element chunks of a head: the two
// whose elements turn together, or two of the elements that stay.  Each angle's
// sine and cosine are computed once, by a thread of their own, and shared
// through LDS (1024 tokens of 16 + 16 heads 7.1 -> 5.3 us).  Several tokens a
// block, or rows requested before the angles, are no faster.  Bound by HBM:
// 12768 tokens of 16 + 16 heads take 40 us, 209 MB at 5.2 TB/s; a large copy
// reaches 5.1.
#include "kernels_draft.hpp"

namespace skv {

namespace {

constexpr int kThreads = 256;

// Rows are read once.  bf16 rows leave no copy in the caches (4000 tokens of 64
// + 16 heads: 30 us, 34 with ordinary loads); an fp32 chunk takes two loads of
// the same lines, which costs more that way (12768 tokens of 16 + 16 heads: 89,
// 83 with ordinary loads).
__device__ __forceinline__ void load_row(Chunk<bf16_bits>& c, const bf16_bits* p) {
  const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  c.raw = make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void load_row(Chunk<float>& c, const float* p) { c.load(p); }

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  constexpr int kItems = D / 16;  // chunk pairs per head
  __shared__ float2 s_turn[D / 2];  // (cos, sin) of the token's angles
  const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int n = a.new_len ? min(max(a.new_len[b], 0), a.num_new) : a.num_new;
  const int len = max(a.cache_len[b], 0);
  if (i == 0 && tid == 0 && a.cache_len_out)
    a.cache_len_out[b] = (int32_t)min((int64_t)len + n, (int64_t)INT32_MAX);
  if (i >= n) return;

  const int64_t slot = (int64_t)len + i;
  const int64_t index = slot >> a.pv.page_shift;
  int64_t page = -1;
  if (index < a.pv.max_pages) page = a.table[(int64_t)b * a.pv.max_pages + index];
  const bool stored = page >= 0 && page < a.pv.num_pages;

  const int p = tid % kItems;
  const bool turns = p < a.rot / 16;
  int c0, c1;  // the two chunks
  if (turns && !a.pairs) {
    c0 = p;
    c1 = p + a.rot / 16;
  } else {
    c0 = 2 * p;
    c1 = 2 * p + 1;
  }
  if (a.rot) {
    if (tid < a.rot / 2) {
      const double t = (double)a.positions[(int64_t)b * a.num_new + i] * ((double)a.inv_freq[tid] * 0.15915494309189535);
      float s, c;
      sincospif(2.f * (float)(t - __builtin_rint(t)), &s, &c);
      s_turn[tid] = make_float2(c, s);
    }
    __syncthreads();
  }
  float cs[8], sn[8];
  if (turns) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cs[e] = s_turn[8 * p + e].x;
      sn[e] = s_turn[8 * p + e].y;
    }
  }

  const int kv = a.pv.kv_heads, rows = a.num_q_heads + 2 * kv;
  for (int r = tid / kItems; r < rows; r += kThreads / kItems) {
    const T* src;
    T* dst;
    const bool is_q = r < a.num_q_heads, is_v = r >= a.num_q_heads + kv;
    if (is_q) {
      src = static_cast<const T*>(a.q) + b * a.q_stride_b + i * a.q_stride_s + r * a.q_stride_h;
      dst = static_cast<T*>(a.q_out) + (((int64_t)b * a.num_new + i) * a.num_q_heads + r) * D;
    } else {
      const int g = r - a.num_q_heads - (is_v ? kv : 0);
      if (!stored) continue;
      src = static_cast<const T*>(is_v ? a.v : a.k) + b * a.stride_b + i * a.stride_s + g * a.stride_h;
      dst = static_cast<T*>(is_v ? a.v_pages : a.k_pages) +
            page_row<D>(page, g, (int)(slot & ((1 << a.pv.page_shift) - 1)), a.pv);
    }
    Chunk<T> x, y;
    load_row(x, src + 8 * c0);
    load_row(y, src + 8 * c1);
    if (turns && !is_v) {
      float u[8], w[8];
      x.to_float(u);
      y.to_float(w);
      if (a.pairs) {
        float f[16];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = e < 4 ? u[2 * e] : w[2 * e - 8], t = e < 4 ? u[2 * e + 1] : w[2 * e - 7];
          f[2 * e] = s * cs[e] - t * sn[e];
          f[2 * e + 1] = s * sn[e] + t * cs[e];
        }
        x.from_float(f);
        y.from_float(f + 8);
      } else {
        float f[8], h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f[e] = u[e] * cs[e] - w[e] * sn[e];
          h[e] = u[e] * sn[e] + w[e] * cs[e];
        }
        x.from_float(f);
        y.from_float(h);
      }
    }
    x.store(dst + 8 * c0);
    y.store(dst + 8 * c1);
  }
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, int dtype, int head_dim, int batch, hipStream_t s) {
  const dim3 grid(a.num_new, batch), block(kThreads);
  if (dtype == 1) {
    if (head_dim == 128) return launch_struct(append_kernel<bf16_bits, 128>, grid, block, s, a);
    return launch_struct(append_kernel<bf16_bits, 64>, grid, block, s, a);
  }
  if (head_dim == 128) return launch_struct(append_kernel<float, 128>, grid, block, s, a);
  return launch_struct(append_kernel<float, 64>, grid, block, s, a);
}

}  // namespace skv
