// Attention of the nodes of a drafted tree over the cache and over each other.
//
// Node i of a sequence with L cached entries and n nodes sees the slots c < L
// and the slots L + j whose bit j its mask row sets; its output is the softmax
// of scale * q.k over those, times their values.
//
// One wave per (sequence, node, query head): it takes 64 keys at a time, a key
// per lane for the logits, then D / 64 elements per lane for the sum over V.
#include "kernels_draft.hpp"

namespace skv {

namespace {

template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32(bf16_bits x) { return bf16_to_f32(x); }
template <>
__device__ __forceinline__ float to_f32(float x) { return x; }

__device__ __forceinline__ float wave_max(float x) {
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, xor_shuffle(x, d));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
  for (int d = 1; d < 64; d *= 2) x += xor_shuffle(x, d);
  return x;
}

template <typename T, int D>
__global__ __launch_bounds__(64) void tree_kernel(TreeArgs a, int group) {
  __shared__ __attribute__((aligned(16))) T s_q[D];
  __shared__ float s_p[64];
  __shared__ int64_t s_row[64];
  const int split = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
  const int node = blockIdx.x / a.num_q_heads, h = blockIdx.x % a.num_q_heads, g = h / group;
  const int n = a.nodes_of ? min(max(a.nodes_of[b], 0), a.num_nodes) : a.num_nodes;
  if (node >= n) return;
  const int64_t cap = (int64_t)a.pv.max_pages << a.pv.page_shift;
  const int L = (int)min((int64_t)min(max(a.cache_len[b], 0), a.max_len), cap);
  const int keys = (int)min((int64_t)L + n, cap);
  const int64_t row = ((int64_t)b * a.num_nodes + node) * a.num_q_heads + h;
  for (int e = lane; e < D; e += 64) s_q[e] = static_cast<const T*>(a.q)[row * D + e];
  __syncthreads();

  const int per = (keys + a.num_splits - 1) / a.num_splits;
  const int begin = min(split * per, keys), end = min(begin + per, keys);
  const uint32_t* mask = a.mask ? a.mask + b * a.mask_stride + (int64_t)node * a.mask_words : nullptr;
  float m = neg_inf(), l = 0.f, o[D / 64] = {};
  for (int c0 = begin; c0 < end; c0 += 64) {
    const int c = c0 + lane, j = c - L;
    bool see = c < end && (j < 0 || (mask ? (mask[j >> 5] >> (j & 31)) & 1 : j <= node));
    float z = neg_inf();
    if (see) {
      const int64_t page = page_of(a.table, b, c, a.pv);
      see = page >= 0;
      if (see) {
        s_row[lane] = page_row<D>(page, g, c & ((1 << a.pv.page_shift) - 1), a.pv);
        const T* k = static_cast<const T*>(a.k_pages) + s_row[lane];
        z = 0.f;
        for (int e = 0; e < D; e += 8) {
          Chunk<T> kc, qc;
          float kf[8], qf[8];
          kc.load(k + e);
          qc.load(s_q + e);
          kc.to_float(kf);
          qc.to_float(qf);
#pragma unroll
          for (int t = 0; t < 8; ++t) z += kf[t] * qf[t];
        }
        z *= a.scale_log2;
      }
    }
    const float top = wave_max(see ? z : neg_inf());
    if (top > m) {
      const float corr = fast_exp2(m - top);
      l *= corr;
#pragma unroll
      for (int t = 0; t < D / 64; ++t) o[t] *= corr;
      m = top;
    }
    const float p = see ? fast_exp2(z - (m == neg_inf() ? 0.f : m)) : 0.f;
    l += wave_sum(p);
    s_p[lane] = p;
    const uint64_t seen = __builtin_amdgcn_ballot_w64(see);
    __syncthreads();
    for (int k = 0; k < 64; ++k) {
      if (!(seen >> k & 1)) continue;
      const T* v = static_cast<const T*>(a.v_pages) + s_row[k];
#pragma unroll
      for (int t = 0; t < D / 64; ++t) o[t] += s_p[k] * to_f32<T>(v[lane + 64 * t]);
    }
    __syncthreads();
  }

#pragma unroll
  for (int t = 0; t < D / 64; ++t) {
    const int e = lane + 64 * t;
    if (a.num_splits > 1) {
      a.ws_o[(row * a.num_splits + split) * D + e] = o[t];
    } else {
      const float x = l == 0.f ? 0.f : o[t] / l;
      if (sizeof(T) == 2) static_cast<bf16_bits*>(a.out)[row * D + e] = (bf16_bits)f32_to_bf16(x);
      else static_cast<float*>(a.out)[row * D + e] = x;
    }
  }
  if (a.num_splits > 1 && lane == 0) {
    a.ws_ml[(row * a.num_splits + split) * 2] = m;
    a.ws_ml[(row * a.num_splits + split) * 2 + 1] = l;
  }
}

// Log-sum-exp merge of the split partials of one (sequence, node, head).
template <typename T, int D>
__global__ __launch_bounds__(D) void tree_merge_kernel(TreeArgs a) {
  const int b = blockIdx.z, node = blockIdx.y, h = blockIdx.x, e = threadIdx.x;
  const int n = a.nodes_of ? min(a.nodes_of[b], a.num_nodes) : a.num_nodes;
  if (node >= n) return;
  const int S = a.num_splits;
  const int64_t row = ((int64_t)b * a.num_nodes + node) * a.num_q_heads + h;
  const float* ml = a.ws_ml + row * S * 2;
  const float* po = a.ws_o + row * S * D + e;
  float M = neg_inf();
  for (int s = 0; s < S; ++s) M = fmaxf(M, ml[2 * s]);
  float num = 0.f, den = 0.f;
  for (int s = 0; s < S; ++s) {
    const float f = fast_exp2(ml[2 * s] - (M == neg_inf() ? 0.f : M));
    num += f * po[(int64_t)s * D];
    den += f * ml[2 * s + 1];
  }
  const float x = den == 0.f ? 0.f : num / den;
  if (sizeof(T) == 2) static_cast<bf16_bits*>(a.out)[row * D + e] = (bf16_bits)f32_to_bf16(x);
  else static_cast<float*>(a.out)[row * D + e] = x;
}

template <typename T, int D>
hipError_t launch_tree_d(const TreeArgs& a, int group, int batch, hipStream_t s) {
  TreeArgs args = a;
  void* argv[] = {&args, &group};
  return hipLaunchKernel(reinterpret_cast<const void*>(tree_kernel<T, D>),
                         dim3(a.num_nodes * a.num_q_heads, a.num_splits, batch), dim3(64), argv, 0, s);
}

}  // namespace

hipError_t launch_tree(const TreeArgs& a, int dtype, int head_dim, int group, int batch, hipStream_t s) {
  if (dtype == 1) {
    if (head_dim == 128) return launch_tree_d<bf16_bits, 128>(a, group, batch, s);
    return launch_tree_d<bf16_bits, 64>(a, group, batch, s);
  }
  if (head_dim == 128) return launch_tree_d<float, 128>(a, group, batch, s);
  return launch_tree_d<float, 64>(a, group, batch, s);
}

hipError_t launch_tree_merge(const TreeArgs& a, int dtype, int head_dim, int batch, hipStream_t s) {
  const dim3 grid(a.num_q_heads, a.num_nodes, batch), block(head_dim);
  if (dtype == 1) {
    if (head_dim == 128) return launch_struct(tree_merge_kernel<bf16_bits, 128>, grid, block, s, a);
    return launch_struct(tree_merge_kernel<bf16_bits, 64>, grid, block, s, a);
  }
  if (head_dim == 128) return launch_struct(tree_merge_kernel<float, 128>, grid, block, s, a);
  return launch_struct(tree_merge_kernel<float, 64>, grid, block, s, a);
}

}  // namespace skv
