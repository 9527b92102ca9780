// The accepted nodes of a drafted tree move together behind the cache, in all
// layers at once: slot L + j takes the entry of slot L + path[j].
//
// A path may name any slots, so no entry is written before all are read: a
// block holds its whole share in registers, 16 bytes a piece, then writes.  The
// share is the path's entries of one sequence and layer for some of its KV heads
// and pools (K or V), as many as the registers hold, or a part of the columns of
// one where the path is long.  Where each entry is read and written is the same
// for all heads: the block looks it up once, an entry a thread, into LDS.
//
// Bound by the chain of loads (length, path, table entries, rows) where little
// moves (one layer of one user: 2.9 us).  Paths of up to 6 of 64 users through
// 28 layers of 8 KV heads take 10 us, 38 with a block for each KV head and pool;
// with a third of the entries moving (the others stay where they are) that is
// 15 MB read and written, 1.5 TB/s, so not HBM's rate.
#include <algorithm>

#include "kernels_draft.hpp"

namespace skv {

namespace {

constexpr int kThreads = 256;
constexpr int kHeld = 8;  // pieces a thread holds

// kChunks: pieces of a row.
template <int kChunks>
__global__ __launch_bounds__(kThreads) void commit_kernel(CommitArgs a) {
  __shared__ int64_t s_from[kCommitPath], s_to[kCommitPath];  // rows of head 0 in a pool, -1: not moved
  const CommitLayer& y = a.layer[blockIdx.z];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int len = max(y.cache_len[b], 0);
  const int m = min(max(a.path_len[b], 0), a.max_path);
  if (blockIdx.x == 0 && tid == 0 && y.cache_len_out)
    y.cache_len_out[b] = (int32_t)min((int64_t)len + m, (int64_t)INT32_MAX);

  // row of tree node `node` for head 0, or -1 where the table has no page for it
  auto row_of = [&](int node) -> int64_t {
    const int64_t slot = (int64_t)len + node;
    const int64_t index = slot >> y.page_shift;
    if (index >= y.max_pages) return -1;
    const int64_t page = y.table[(int64_t)b * y.max_pages + index];
    if (page < 0 || page >= y.num_pages) return -1;
    return (page * a.kv_heads << y.page_shift) + (slot & ((1 << y.page_shift) - 1));
  };
  for (int j = tid; j < m; j += kThreads) {
    const int node = a.path[(int64_t)b * a.max_path + j];
    int64_t from = -1, to = -1;
    if (node >= 0 && node < a.num_nodes && node != j) {
      from = row_of(node);
      to = row_of(j);
    }
    s_from[j] = from;
    s_to[j] = from < 0 ? -1 : to;
  }
  __syncthreads();

  // piece number `item` of the block: column, then entry of the path, then
  // (KV head, pool)
  const int part = blockIdx.x % a.parts, first = blockIdx.x / a.parts * a.heads;
  const int cols = kChunks / a.parts;
  u32x4_t held[kHeld];
  u32x4_t* at[kHeld];
#pragma unroll
  for (int t = 0; t < kHeld; ++t) {
    const int item = tid + t * kThreads, col = item & (cols - 1);
    int h, j;
    a.by_path.divide(item / cols, h, j);
    const int hv = first + h;
    at[t] = nullptr;
    held[t] = u32x4_t{0, 0, 0, 0};
    if (h < a.heads && hv < 2 * a.kv_heads && j < m && s_to[j] >= 0) {
      u32x4_t* pool = static_cast<u32x4_t*>(hv & 1 ? y.v_pages : y.k_pages) + part * cols + col;
      const int64_t head = (int64_t)(hv >> 1) << y.page_shift;
      held[t] = pool[(s_from[j] + head) * kChunks];
      at[t] = pool + (s_to[j] + head) * kChunks;
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < kHeld; ++t)
    if (at[t]) *at[t] = held[t];
}

}  // namespace

hipError_t launch_commit(const CommitArgs& args, int dtype, int head_dim, int layers, int batch, hipStream_t s) {
  CommitArgs a = args;
  const int chunks = head_dim * (dtype == 1 ? 2 : 4) / 16, pieces = kThreads * kHeld;
  a.by_path = FastDivide(a.max_path);
  a.parts = 1;
  while (a.max_path * (chunks / a.parts) > pieces) a.parts *= 2;
  // (KV head, pool) pairs of a block: what its registers hold, but fewer while
  // the launch has less than two blocks a CU (one sequence, one layer of 8 KV
  // heads: 16 blocks)
  const int64_t pairs = 2 * (int64_t)a.kv_heads;
  const int64_t fill = pairs * layers * batch / 512;
  a.heads = (int)std::max<int64_t>(1, std::min<int64_t>({pieces / (a.max_path * (chunks / a.parts)), fill, pairs}));
  const dim3 grid((uint32_t)((pairs + a.heads - 1) / a.heads * a.parts), batch, layers), block(kThreads);
  if (chunks == 8) return launch_struct(commit_kernel<8>, grid, block, s, a);
  if (chunks == 16) return launch_struct(commit_kernel<16>, grid, block, s, a);
  return launch_struct(commit_kernel<32>, grid, block, s, a);
}

}  // namespace skv
