// The accepted nodes of a drafted tree move together behind the cache, in all
// layers at once: slot L + j takes the entry of slot L + path[j].
//
// A path may name any slots, so no entry is written before all are read: a
// block holds its whole share of them in registers (the entries of one
// sequence, layer, KV head and pool, or a part of their columns where the
// path is long), then writes.
#include "kernels_draft.hpp"

namespace skv {

namespace {

constexpr int kThreads = 256;
constexpr int kHeld = 8;  // 16-byte pieces a thread holds

// Column parts that let kThreads * kHeld pieces hold max_path rows of `chunks`
// pieces.
int column_parts(int max_path, int chunks) {
  int parts = 1;
  while (max_path * (chunks / parts) > kThreads * kHeld) parts *= 2;
  return parts;
}

// kChunks: 16-byte pieces of a row.
template <int kChunks>
__global__ __launch_bounds__(kThreads) void commit_kernel(CommitArgs a) {
  const CommitLayer& y = a.layer[blockIdx.z];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int parts = gridDim.x / (2 * a.kv_heads);
  const int part = blockIdx.x % parts, is_v = blockIdx.x / parts & 1, g = blockIdx.x / parts / 2;
  const int cols = kChunks / parts;
  const int len = max(y.cache_len[b], 0);
  const int m = min(max(a.path_len[b], 0), a.max_path);
  if (blockIdx.x == 0 && tid == 0 && y.cache_len_out)
    y.cache_len_out[b] = (int32_t)min((int64_t)len + m, (int64_t)INT32_MAX);
  u32x4_t* const pool = static_cast<u32x4_t*>(is_v ? y.v_pages : y.k_pages) + part * cols;

  // piece number of column 0 of tree node `node`, or -1 where the table has no
  // page for it
  auto row_of = [&](int node) -> int64_t {
    const int64_t slot = (int64_t)len + node;
    const int64_t index = slot >> y.page_shift;
    if (index >= y.max_pages) return -1;
    const int64_t page = y.table[(int64_t)b * y.max_pages + index];
    if (page < 0 || page >= y.num_pages) return -1;
    return (((page * a.kv_heads + g) << y.page_shift) + (slot & ((1 << y.page_shift) - 1))) * kChunks;
  };

  u32x4_t held[kHeld];
  int64_t to[kHeld];
#pragma unroll
  for (int t = 0; t < kHeld; ++t) {
    const int item = tid + t * kThreads, j = item / cols, col = item % cols;
    int64_t from = -1;
    to[t] = -1;
    if (j < m) {
      const int node = a.path[(int64_t)b * a.max_path + j];
      if (node >= 0 && node < a.num_nodes && node != j) {
        from = row_of(node);
        to[t] = from < 0 ? -1 : row_of(j);
      }
    }
    held[t] = u32x4_t{0, 0, 0, 0};
    if (to[t] >= 0) held[t] = pool[from + col];
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < kHeld; ++t)
    if (to[t] >= 0) pool[to[t] + (tid + t * kThreads) % cols] = held[t];
}

}  // namespace

hipError_t launch_commit(const CommitArgs& a, int dtype, int head_dim, int layers, int batch, hipStream_t s) {
  const int chunks = head_dim * (dtype == 1 ? 2 : 4) / 16;
  const dim3 grid(column_parts(a.max_path, chunks) * 2 * a.kv_heads, batch, layers), block(kThreads);
  if (chunks == 8) return launch_struct(commit_kernel<8>, grid, block, s, a);
  if (chunks == 16) return launch_struct(commit_kernel<16>, grid, block, s, a);
  return launch_struct(commit_kernel<32>, grid, block, s, a);
}

}  // namespace skv
