// The attention weight that cache entries gather from queries: for entry c the sum
// of exp(scale q.k_c - lse) over the rows that see it, added to what it has.
//
// A wave holds 64 keys of a (sequence, KV head) in registers (four tiles of 16,
// operand A) and goes through the rows, query heads of the group and queries, in
// tiles of 16 (operand B): S^T = K Q^T on the 16x16 matrix products, the weights
// straight from it, summed per key in a lane's own registers; the 16 lanes of a
// key add up once, at the end.  Keys and rows go from memory into the operands
// (a lane's 16-byte pieces; four lanes read 64 bytes of a row): K is read once and
// never needed in LDS.  The order of the elements along a row is that of the
// pieces, for both operands alike.
//
// With few row tiles (a decoding step) every wave has keys of its own; with more
// the waves of a block share 64 keys, deal the row tiles out and add up through
// LDS, in order.
#include "attn_mfma.hpp"
#include "kernels_shared.hpp"

namespace skv {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kTiles = kWeightKeys / 16;
constexpr int kSpreadUnits = 32;  // pairs from which an XCD keeps a pair's blocks together

template <typename T>
__device__ __forceinline__ f32x4_t product(u32x4_t k, u32x4_t q, f32x4_t c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q), c,
                                                   0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(q[e]), c, 0, 0, 0);
    return c;
  }
}

// v[j] summed over the 16 lanes of a row, for j = the lane's number in the row.
__device__ __forceinline__ float transposed_sum(float (&v)[16], int lane) {
  auto step = [&](auto half, auto ctrl) __attribute__((always_inline)) {
    constexpr int n = decltype(half)::value;
    const bool up = lane & n;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const float keep = up ? v[k + n] : v[k], send = up ? v[k] : v[k + n];
      v[k] = keep + dpp<decltype(ctrl)::value>(send);
    }
  };
  step(std::integral_constant<int, 8>(), std::integral_constant<int, kDppRowRor8>());
  step(std::integral_constant<int, 4>(), std::integral_constant<int, kDppHalfMirror>());
  step(std::integral_constant<int, 2>(), std::integral_constant<int, kDppQuadXor2>());
  step(std::integral_constant<int, 1>(), std::integral_constant<int, kDppQuadXor1>());
  return v[0];
}

// kDealt: the waves of a block share its keys and deal the row tiles out.
template <typename T, int D, bool kDealt>
__global__ __launch_bounds__(kThreads, 2) void weights_kernel(WeightArgs a) {
  constexpr int kPieces = D * (int)sizeof(T) / 64;  // 16-byte pieces of a row per lane
  constexpr int kElems = 16 / (int)sizeof(T);       // of a piece
  __shared__ float s_part[kWaves][kWeightKeys];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int heads = a.cache.pv.kv_heads, pairs = a.batch * heads;
  int pair, part, b, g;
  if (pairs >= kSpreadUnits) {
    a.by_key_blocks.divide((int)(blockIdx.x >> 3), pair, part);
    pair = pair * 8 + (blockIdx.x & 7);
    if (pair >= pairs) return;
  } else {
    a.by_key_blocks.divide((int)blockIdx.x, pair, part);
  }
  a.by_heads.divide(pair, b, g);
  const PagedView& pv = a.cache.pv;
  const int len = (int)min((int64_t)min(max(a.cache.len[b], 0), a.cache.max_len), (int64_t)pv.max_pages << pv.page_shift);
  const int kb = kDealt ? part * kWeightKeys : (part * kWaves + wave) * kWeightKeys;
  if (kb >= len) return;

  // the keys: lane (col, quarter) has pieces quarter, 4 + quarter, .. of key col of each tile
  u32x4_t k[kTiles][kPieces];
  uint64_t present = 0;  // keys that exist and have a page
  {
    const int32_t* table = a.cache.table + (int64_t)b * pv.max_pages;
    const T* pool = static_cast<const T*>(a.cache.k_pages);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int key = min(kb + 16 * t + col, len - 1);
      const int64_t page = table[key >> pv.page_shift];
      const bool ok = page >= 0 && page < pv.num_pages;
      const T* row = pool + page_row<D>(ok ? page : 0, g, key & ((1 << pv.page_shift) - 1), pv) + quarter * kElems;
      const uint64_t there = __builtin_amdgcn_ballot_w64(ok && kb + 16 * t + col < len);
      present |= (there & 0xffffu) << (16 * t);
#pragma unroll
      for (int p = 0; p < kPieces; ++p) k[t][p] = *reinterpret_cast<const u32x4_t*>(row + 4 * p * kElems);
    }
  }

  float sum[16];  // element 4 t + i: key 16 t + 4 quarter + i, over this lane's rows
#pragma unroll
  for (int j = 0; j < 16; ++j) sum[j] = 0.f;
  const int gmask = (1 << a.group_shift) - 1, rows = a.num_rows << a.group_shift;
  const T* q = static_cast<const T*>(a.q.p) + b * a.q.sb + quarter * kElems;
  const float* lse = a.lse + b * a.lse_b;
  for (int rt = kDealt ? wave : 0; rt < a.row_tiles; rt += kDealt ? kWaves : 1) {
    const int r = rt * 16 + col;
    const int i = min(r, rows - 1) >> a.group_shift, h = (g << a.group_shift) + (r & gmask);
    int seen = a.visible ? a.visible[(int64_t)b * a.num_rows + i] : len - (a.num_rows - 1 - i);
    seen = r < rows ? min(max(seen, 0), len) : 0;
    if (!__builtin_amdgcn_ballot_w64(seen > kb)) continue;
    const float l = lse[h * a.lse_h + i * a.lse_s] * 1.4426950408889634f;
    if (l == neg_inf()) seen = 0;  // (a row that saw nothing)
    const T* row = q + i * a.q.ss + h * a.q.sh;
    u32x4_t x[kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) x[p] = *reinterpret_cast<const u32x4_t*>(row + 4 * p * kElems);
    const bool all = !__builtin_amdgcn_ballot_w64(seen < kb + kWeightKeys);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      f32x4_t st = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < kPieces; ++p) st = product<T>(k[t][p], x[p], st);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float w = fast_exp2(__builtin_fmaf(st[e], a.scale_log2, -l));
        const int key = kb + 16 * t + 4 * quarter + e;
        sum[4 * t + e] += all || key < seen ? w : 0.f;
      }
    }
  }
  float total = transposed_sum(sum, lane);  // of key 16 (col / 4) + 4 quarter + col % 4
  int at = 16 * (col >> 2) + 4 * quarter + (col & 3);
  if constexpr (kDealt) {
    s_part[wave][at] = total;
    __syncthreads();
    if (wave) return;
    at = lane;
    total = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) total += s_part[v][at];
  }
  if (kb + at < len) {
    const int64_t to = (int64_t)pair * a.capacity + kb + at;
    const float had = a.weights ? a.weights[to] : 0.f;
    a.weights_out[to] = present >> at & 1 ? had + total : had;
  }
}

}  // namespace

template <typename T, int D>
hipError_t launch_weights_d(const WeightArgs& args, hipStream_t s) {
  WeightArgs a = args;
  a.by_key_blocks = FastDivide(a.key_blocks);
  a.by_heads = FastDivide(a.cache.pv.kv_heads);
  const int64_t pairs = (int64_t)a.batch * a.cache.pv.kv_heads;
  const dim3 grid((uint32_t)((pairs >= kSpreadUnits ? (pairs + 7) / 8 * 8 : pairs) * a.key_blocks)), block(kThreads);
  return a.row_tiles >= kWeightDealt ? launch_struct(weights_kernel<T, D, true>, grid, block, s, a)
                                     : launch_struct(weights_kernel<T, D, false>, grid, block, s, a);
}

hipError_t launch_weights(const WeightArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? launch_weights_d<bf16_bits, 128>(a, s) : launch_weights_d<bf16_bits, 64>(a, s);
  return head_dim == 128 ? launch_weights_d<float, 128>(a, s) : launch_weights_d<float, 64>(a, s);
}

}  // namespace skv
