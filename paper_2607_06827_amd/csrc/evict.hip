// Caches are shortened to the entries that gathered most attention weight.
//
// Of a (layer, sequence, KV head)'s L entries n stay: the first, the last, and of
// those between them the m heaviest.  A block finds the m-th largest weight digit
// by digit (weights as whole numbers in the order of the numbers; up to four passes of
// 8 bits over the row, a histogram each), which needs no sort; entries above it
// stay, and of those equal to it the lowest slots.  A second pass over the row
// counts who stays before each entry, in order, and writes the kept slots and
// their weights.
//
// Then the rows move, in place and in order: entry j takes slot s_j >= j.  A block
// takes one head of one pool (or a part of its columns) and goes through its
// entries in order: it holds a stretch of them in registers before it writes them,
// and what later stretches read lies behind what it writes.
//
// Bound by HBM: 28 layers of 8 sequences of up to 846 entries, 8 heads, 512 kept, take
// 127 us, 574 MB at 4.5 TB/s (a large copy reaches 5.1).  Rows are read and written
// non-temporally (140 us without), eight pieces a thread (133 with 16: fewer blocks run
// at once).  From 512 rows on one kernel chooses and moves (134 us as two launches, as
// the choice alone, all latency, takes 15); one layer of one sequence has 8 and takes
// 5.7 and 4.9 us as two, whose moves have four times the blocks (6.8 with all four
// passes, though fewer settle it).  A row is one block's however long it is: of one
// sequence with 7532 entries, half of them kept, one layer takes 78 us (31 MB) and 28
// layers 234 (880 MB), chains of turns that nothing requests ahead.
#include <algorithm>

#include "kernels_shared.hpp"

namespace skv {

namespace {

constexpr int kThreads = 256;
constexpr int kFusedRows = 512;  // (layer, sequence, KV head)s from which one kernel does both
constexpr int kHeld = 8;     // pieces a thread of the move holds
constexpr int kKeysHeld = 8;  // weights a thread of the choice holds

// Whole numbers in the order of the weights: 0 and -0 alike, NaN below all.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t x = __float_as_uint(w);
  if ((x & 0x7fffffffu) > 0x7f800000u) return 0u;
  if ((x & 0x7fffffffu) == 0u) return 0x80000000u;
  return x & 0x80000000u ? ~x : x | 0x80000000u;
}

struct Counts {
  int len, keep, first, recent;
};
__device__ __forceinline__ Counts counts_of(const EvictArgs& a, const EvictLayer& y, int b) {
  Counts c;
  c.len = (int)min((int64_t)min(max(y.cache_len[b], 0), a.capacity), (int64_t)y.max_pages << y.page_shift);
  c.keep = min(c.len, min(max(a.keep_len[b], 0), a.max_keep));
  c.first = min(a.num_first, c.keep);
  c.recent = min(a.num_recent, c.keep - c.first);
  return c;
}

struct ChoiceSpace {
  uint32_t count[256];
  int digit, left;
  int stay[2][kThreads / 64], equal[2][kThreads / 64];
};

// The entries of head g of sequence b that stay, into kept and weights_out, by one
// block.
__device__ __forceinline__ void choose(const EvictArgs& a, const EvictLayer& y, int b, int g, const Counts& n,
                                       ChoiceSpace& s) {
  constexpr int kBlock = kThreads, kWaves = kThreads / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (g == 0 && tid == 0 && y.cache_len_out) y.cache_len_out[b] = n.keep;
  const int64_t row = (int64_t)b * a.kv_heads + g;
  const float* w = y.weights + row * a.capacity;
  float* out = y.weights_out + row * a.capacity;
  int32_t* kept = y.kept + row * a.max_keep;
  if (n.keep == n.len) {
    for (int c = tid; c < n.len; c += kBlock) {
      kept[c] = c;
      if (out != w) out[c] = w[c];
    }
    return;
  }
  const int lo = n.first, hi = n.len - n.recent;  // the entries between
  const int m = n.keep - n.first - n.recent;      // of which so many stay
  // the m-th largest: digits from the top, among those that share the ones before
  // (a short row stays in registers between the passes)
  uint32_t least = 0, held[kKeysHeld];
  const bool is_held = hi - lo <= kKeysHeld * kBlock;
  int left = m;
  if (m > 0) {
    if (is_held) {
#pragma unroll
      for (int t = 0; t < kKeysHeld; ++t) {
        const int c = lo + tid + t * kBlock;
        held[t] = c < hi ? order_of(w[c]) : 0u;
      }
    }
    for (int shift = 24; shift >= 0; shift -= 8) {
      s.count[tid] = 0;
      static_assert(kBlock == 256, "a thread a digit");
      __syncthreads();
      auto count = [&](uint32_t x) {
        if (shift == 24 || (x >> (shift + 8)) == (least >> (shift + 8))) atomicAdd(&s.count[x >> shift & 255u], 1u);
      };
      if (is_held) {
#pragma unroll
        for (int t = 0; t < kKeysHeld; ++t)
          if (lo + tid + t * kBlock < hi) count(held[t]);
      } else {
        for (int c = lo + tid; c < hi; c += kBlock) count(order_of(w[c]));
      }
      __syncthreads();
      if (wave == 0) {
        // lane i has the digits 4 i .. 4 i + 3; entries of digits above them
        int mine[4], sum = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += mine[k] = (int)s.count[4 * lane + k];
        int above = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const int x = __shfl_down(above, d, 64);
          if (lane + d < 64) above += x;
        }
        above -= sum;
#pragma unroll
        for (int k = 3; k >= 0; --k) {
          if (above < left && left <= above + mine[k]) {
            s.digit = 4 * lane + k;
            // (all with this digit stay: none of their lower digits matters)
            s.left = mine[k] == left - above ? INT32_MAX : left - above;
          }
          above += mine[k];
        }
      }
      __syncthreads();
      least |= (uint32_t)s.digit << shift;
      left = s.left;
      if (left == INT32_MAX) break;
    }
  }
  // `left` of those equal to `least` stay, the lowest slots first
  int stayed = 0, equals = 0;  // before this stretch
  for (int base = 0, turn = 0; base < n.len; base += kBlock, turn ^= 1) {
    const int c = base + tid;
    const float x = c < n.len ? w[c] : 0.f;
    const uint32_t key = order_of(x);
    const bool between = c >= lo && c < hi;
    const bool equal = between && m > 0 && key == least;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(equal);
    const uint64_t before = ((uint64_t)1 << lane) - 1;
    if (lane == 0) s.equal[turn][wave] = __popcll(eq);
    __syncthreads();
    int rank = equals + __popcll(eq & before);
    for (int v = 0; v < kWaves; ++v) {
      const int k = s.equal[turn][v];
      if (v < wave) rank += k;
      equals += k;
    }
    const bool stay = c < n.len && (between ? m > 0 && (key > least || (equal && rank < left)) : true);
    const uint64_t st = __builtin_amdgcn_ballot_w64(stay);
    if (lane == 0) s.stay[turn][wave] = __popcll(st);
    __syncthreads();  // (every weight of this stretch has been read)
    int to = stayed + __popcll(st & before);
    for (int v = 0; v < kWaves; ++v) {
      const int k = s.stay[turn][v];
      if (v < wave) to += k;
      stayed += k;
    }
    if (stay) {
      kept[to] = c;
      out[to] = x;
    }
  }
  __syncthreads();
  for (int c = n.keep + tid; c < n.len; c += kBlock) out[c] = 0.f;
}

constexpr int kMost = kThreads * kHeld / 4;  // most entries of a stretch (a part has 4 pieces at least)
struct MoveSpace {
  int64_t from[kMost], to[kMost];  // rows in a pool, -1: not moved
};

// The rows of head g of sequence b in pool number v (0: keys, 1: values) move, by one
// block: pieces part * cols .. of the kChunks 16-byte pieces of a row.
template <int kChunks>
__device__ __forceinline__ void move(const EvictArgs& a, const EvictLayer& y, int b, int g, int v, int part, int cols,
                                     const Counts& n, MoveSpace& s) {
  const int tid = threadIdx.x, stretch = kThreads * kHeld / cols;
  const int32_t* kept = y.kept + ((int64_t)b * a.kv_heads + g) * a.max_keep;
  const int32_t* table = y.table + (int64_t)b * y.max_pages;
  u32x4_t* pool = static_cast<u32x4_t*>(v ? y.v_pages : y.k_pages) + part * cols;
  auto row_of = [&](int slot) -> int64_t {
    const int page = table[slot >> y.page_shift];  // (a slot below n.len is inside the table)
    if (page < 0 || page >= y.num_pages) return -1;
    return (((int64_t)page * a.kv_heads + g) << y.page_shift) + (slot & ((1 << y.page_shift) - 1));
  };
  for (int first = 0; first < n.keep; first += stretch) {
    const int some = min(stretch, n.keep - first);
    for (int j = tid; j < some; j += kThreads) {
      const int slot = min(max(kept[first + j], first + j), n.len - 1);
      int64_t from = -1, to = -1;
      if (slot != first + j) {
        from = row_of(slot);
        to = row_of(first + j);
      }
      s.from[j] = from;
      s.to[j] = from < 0 ? -1 : to;
    }
    __syncthreads();
    u32x4_t held[kHeld];
#pragma unroll
    for (int t = 0; t < kHeld; ++t) {
      const int item = tid + t * kThreads, j = item / cols;
      if (j < some && s.to[j] >= 0)
        held[t] = __builtin_nontemporal_load(pool + s.from[j] * kChunks + (item & (cols - 1)));
    }
    __syncthreads();  // (every row of the stretch has been read)
#pragma unroll
    for (int t = 0; t < kHeld; ++t) {
      const int item = tid + t * kThreads, j = item / cols;
      if (j < some && s.to[j] >= 0)
        __builtin_nontemporal_store(held[t], pool + s.to[j] * kChunks + (item & (cols - 1)));
    }
    __syncthreads();  // (the lists have been read)
  }
}

// Few rows: the choice, then the moves as blocks of their own.
__global__ __launch_bounds__(kThreads) void evict_choose_kernel(EvictArgs a) {
  __shared__ ChoiceSpace s;
  const EvictLayer& y = a.layer[blockIdx.z];
  choose(a, y, blockIdx.y, blockIdx.x, counts_of(a, y, blockIdx.y), s);
}

template <int kChunks>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(EvictArgs a) {
  __shared__ MoveSpace s;
  const EvictLayer& y = a.layer[blockIdx.z];
  const Counts n = counts_of(a, y, blockIdx.y);
  if (n.keep == n.len) return;
  const int part = blockIdx.x % a.parts, hv = blockIdx.x / a.parts;
  move<kChunks>(a, y, blockIdx.y, hv >> 1, hv & 1, part, kChunks / a.parts, n, s);
}

// Many rows: a block chooses and moves, so that one block's choice runs beside
// another's moves.
template <int kChunks>
__global__ __launch_bounds__(kThreads) void evict_kernel(EvictArgs a) {
  __shared__ union {
    ChoiceSpace choice;
    MoveSpace moves;
  } s;
  const EvictLayer& y = a.layer[blockIdx.z];
  const int b = blockIdx.y, g = blockIdx.x;
  const Counts n = counts_of(a, y, b);
  choose(a, y, b, g, n, s.choice);
  if (n.keep == n.len) return;
  __syncthreads();  // (the list is complete)
  for (int v = 0; v < 2; ++v) move<kChunks>(a, y, b, g, v, 0, kChunks, n, s.moves);
}

template <int kChunks>
hipError_t launch_evict_d(const EvictArgs& a, int layers, int batch, hipStream_t s) {
  const dim3 rows(a.kv_heads, batch, layers), block(kThreads);
  if ((int64_t)a.kv_heads * batch * layers >= kFusedRows) return launch_struct(evict_kernel<kChunks>, rows, block, s, a);
  const hipError_t e = launch_struct(evict_choose_kernel, rows, block, s, a);
  if (e != hipSuccess) return e;
  return launch_struct(evict_move_kernel<kChunks>, dim3(2 * a.kv_heads * a.parts, batch, layers), block, s, a);
}

}  // namespace

hipError_t launch_evict(const EvictArgs& args, int dtype, int head_dim, int layers, int batch, hipStream_t s) {
  EvictArgs a = args;
  const int chunks = head_dim * (dtype == 1 ? 2 : 4) / 16;
  a.parts = 2;
  if (chunks == 8) return launch_evict_d<8>(a, layers, batch, s);
  if (chunks == 16) return launch_evict_d<16>(a, layers, batch, s);
  return launch_evict_d<32>(a, layers, batch, s);
}

}  // namespace skv
