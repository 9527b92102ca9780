// Attention of the nodes of a drafted tree over the cache and over each other.
//
// Node i of a sequence with L cached entries and n nodes sees the slots c < L
// and the slots L + j whose bit j its mask row sets; its output is the softmax
// of scale * q.k over those, times their values.
//
// All n nodes see the same cache, so the rows of one KV head, n nodes times the
// G query heads of its group, are one matrix: with up to about a hundred rows
// the work is reading each K/V row once (bound by HBM), with more it is the two
// matrix products.  A block of four waves takes 32, 64 or 128 rows (kGroups =
// 1, 2 or 4 row groups of 32, a wave each) and a range of keys in tiles of 32;
// with fewer than four row groups the waves split the tiles between them
// (4 / kGroups streams).  A wave holds its 32 query rows in registers and per
// tile computes
//     S^T = K Q^T      (keys x rows; 32x32 MFMA, A = K tile, B = Q^T)
//     O^T += V^T P^T   (A = V^T tile, B = P^T, straight from S^T's layout)
// with the online softmax between them, one row per lane column.  bf16 takes
// v_mfma_f32_32x32x16_bf16, fp32 takes v_mfma_f32_32x32x2_f32; maxima, weight
// sums and outputs are fp32 in both.
//
// The bf16 product wants the weights in bf16, so they are rounded, as this
// library's decode and prefill do; the weight sum is of those before, so an
// output is off by at most 2^-8 of its weighted |values| and its own rounding.
// Measured against 64 bits: 2.1 to 2.3e-3 (root mean square, relative), 1.7e-3
// of it the output's rounding.  Weights as the sum of two bf16 numbers leave that
// alone, but take the value products twice: 16 sequences of 7692 keys 91 -> 93
// us, one with 64 nodes 17.8 -> 19.8, 301 nodes of 64 heads on 8 43 -> 52.
//
// K/V tiles go from the paged cache straight into LDS (direct loads of 16 bytes
// a lane), rows unpadded and their 16-byte chunks XOR-swizzled so that operand
// reads are spread over the banks.
//
// With one row group every wave streams its own tiles through its own K and V
// buffer, with no barrier: the next K tile is requested as soon as S^T is
// computed, the next V tile as soon as O^T is, so a wave nearly always has a
// tile in flight, and two blocks of 64 KB share a CU.  With two or four row
// groups the waves of a stream load a tile together, one tile ahead, one barrier
// per tile.  (Two tiles ahead are no faster, with or without a third block on a
// CU.)
//
// Tiles below L, or in a chain below the block's first node, need no mask (512
// nodes behind 1000 keys: 53 -> 47 us).  In the others each lane has its row's 32
// bits; a row's weight of a key it does not see is 0, and since 0 times infinity
// is not, values of these tiles that are not finite become 0 and rows that do
// see them get them after the loop, key by key.
//
// Measured (bf16, 128 wide): 16 sequences of 7692 keys, 32 nodes of 16 heads on
// 8: 86 us, 508 MB at 5.9 TB/s (a copy reaches 5.1, reads alone 6.4); 64
// sequences of up to 284 keys, 16 nodes: 16 us, 3.9 TB/s, 5 of them the launch
// and a block's first loads; 8 sequences of up to 447 keys, 301 nodes of 64
// heads on 8: 41 us, 590 TFLOP/s.
//
// Streams merge through LDS at the end, splits through the workspace, both by
// log-sum-exp in a fixed order.
#include "attn_mfma.hpp"
#include "kernels_draft.hpp"

namespace skv {

namespace {

// The running maximum may lag the true one by up to 2^kSlack before the sums are
// rescaled; the division by the weight sum makes the choice exact.
constexpr float kSlack = 8.f;
constexpr int kKeys = kTreeKeys;  // keys per tile
static_assert(kKeys == 32, "a tile's keys are the bits of a word and the rows of a 32x32 product");
constexpr int kWaves = 4;
constexpr int kSpreadUnits = 32;  // units from which an XCD keeps a unit's row tiles together

// Layout of a K or V tile in LDS: rows of kChunks 16-byte chunks, chunk c of
// row r at position c ^ k(r) or c ^ v(r).
template <typename T, int D>
struct Tile {
  static constexpr int kRowBytes = D * (int)sizeof(T);
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kBytes = kKeys * kRowBytes;
  static constexpr int kRowsPerLoad = 64 / kChunks;       // rows a wave-wide direct load fills
  static constexpr int kLoads = kKeys / kRowsPerLoad;     // loads of a tile
  static constexpr int kFrags = kRowBytes / 32;           // 16-byte operand pieces of a row per lane
  static __device__ __forceinline__ int k(int row) { return row & (kChunks - 1); }
  // bf16: the transposed reads take 4 rows x 4 chunks at a time; fp32: rows 4
  // apart at one chunk
  static __device__ __forceinline__ int v(int row) {
    return sizeof(T) == 2 ? (row % (kChunks / 4)) << 2 : ((row >> 2) & 1) << 3;
  }
};

// lds_dma16, without keeping the line in the caches.
__device__ __forceinline__ void lds_dma16_nt(const void* sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
               :
               : "v"(voff), "s"(sbase), "s"(lds)
               : "memory", "m0");
}

template <int kVm>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0)" : : "i"(kVm) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Orders the wave's LDS reads before the direct loads that follow.
__device__ __forceinline__ void wait_lds() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// S^T of one tile: element i is the logit (unscaled) of key 8 (i / 4) + 4 hg +
// i % 4 for this lane's row.
template <typename T, int D>
__device__ __forceinline__ f32x16_t scores(uint32_t sk, const u32x4_t (&q)[Tile<T, D>::kFrags], int lane) {
  typedef Tile<T, D> L;
  typedef __attribute__((address_space(3))) const u32x4_t* lds_ptr;
  const int col = lane & 31, hg = lane >> 5;
  uint32_t a0 = sk + col * L::kRowBytes + ((uint32_t)(hg ^ L::k(col)) << 4);
  asm volatile("" : "+v"(a0));  // one address register, not one per fragment
  f32x16_t st;
#pragma unroll
  for (int i = 0; i < 16; ++i) st[i] = 0.f;
  // fragments are read kAhead ahead of the products
  constexpr int kAhead = 4;
  u32x4_t buf[kAhead];
#pragma unroll
  for (int kc = 0; kc < kAhead; ++kc) buf[kc] = *(lds_ptr)(uintptr_t)(a0 ^ (uint32_t)(32 * kc));
#pragma unroll
  for (int kc = 0; kc < L::kFrags; ++kc) {
    const u32x4_t k = buf[kc % kAhead];
    if (kc + kAhead < L::kFrags) buf[kc % kAhead] = *(lds_ptr)(uintptr_t)(a0 ^ (uint32_t)(32 * (kc + kAhead)));
    if constexpr (sizeof(T) == 2) {
      st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q[kc]),
                                                   st, 0, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        st = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[e]), __uint_as_float(q[kc][e]), st, 0, 0, 0);
    }
  }
  constexpr int kProducts = sizeof(T) == 2 ? 1 : 4;  // MFMAs per fragment
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);  // LDS reads
#pragma unroll
  for (int kc = 0; kc + kAhead < L::kFrags; ++kc) {
    __builtin_amdgcn_sched_group_barrier(0x008, kProducts, 0);  // MFMA
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kAhead * kProducts, 0);
  return st;
}

// O^T += V^T P^T of one tile (weights p in S^T's layout).
template <typename T, int D>
__device__ __forceinline__ void add_values(uint32_t sv, const float (&p)[16], f32x16_t (&o)[D / 32], int lane) {
  typedef Tile<T, D> L;
  if constexpr (sizeof(T) == 2) {
    // through the LDS transpose read, see Mfma<bf16_bits>::load_v
    const int vg = lane >> 4, vj = lane & 15;
    const int vr = 4 * (vg >> 1) + (vj >> 2);
    uint32_t va = sv + vr * L::kRowBytes +
                  (uint32_t)(((L::v(vr) + 2 * (vg & 1) + ((vj & 3) >> 1)) << 4) | ((vj & 1) << 3));
    asm volatile("" : "+v"(va));
    auto vfrag = [&](int idx) __attribute__((always_inline)) {
      const int kk = idx / (D / 32), db = idx % (D / 32);
      const uint32_t al = (va ^ (uint32_t)(64 * db)) + (uint32_t)(kk * 16 * L::kRowBytes);
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)al);
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)(al + 8 * L::kRowBytes));
      const u16x8_t v = {(unsigned short)lo[0], (unsigned short)lo[1], (unsigned short)lo[2], (unsigned short)lo[3],
                         (unsigned short)hi[0], (unsigned short)hi[1], (unsigned short)hi[2], (unsigned short)hi[3]};
      return __builtin_bit_cast(bf16x8_t, v);
    };
    // operands are read kAhead ahead of the products
    constexpr int kProducts = 2 * (D / 32), kAhead = 3;
    bf16x8_t buf[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) buf[i] = vfrag(i);
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
      const bf16x8_t cur = buf[i % kAhead];
      if (i + kAhead < kProducts) buf[i % kAhead] = vfrag(i + kAhead);
      const int db = i % (D / 32);
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cur, Mfma<bf16_bits>::pack_p(p + 8 * (i / (D / 32))), o[db], 0, 0, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 1);  // LDS reads
#pragma unroll
    for (int i = 0; i + kAhead < kProducts; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);  // MFMA
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 1);
  } else {
    typedef __attribute__((address_space(3))) const float* lds_ptr;
    const int col = lane & 31, hg = lane >> 5;
    // key 8 (i / 4) + 4 hg + i % 4: its chunks are flipped by 8 for hg = 1
    uint32_t va = sv + 4 * hg * L::kRowBytes + (uint32_t)((((col >> 2) ^ (hg << 3)) << 4) | ((col & 3) << 2));
    asm volatile("" : "+v"(va));
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const float v = *(lds_ptr)(uintptr_t)((va ^ (uint32_t)(128 * db)) +
                                              (uint32_t)((8 * (i / 4) + i % 4) * L::kRowBytes));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], o[db], 0, 0, 0);
      }
  }
}

// Whether all values of a tile are finite (the same in every lane): 0 times any
// of them is 0 then, else NaN.
template <typename T, int D>
__device__ __forceinline__ bool all_finite(uint32_t sv, int lane) {
  typedef __attribute__((address_space(3))) const u32x4_t* lds_ptr;
  uint32_t zero = 0;
  asm volatile("" : "+v"(zero));  // (no constant: the products are to be made)
  float sum[2] = {0.f, 0.f};
#pragma unroll 2
  for (int i = 0; i < Tile<T, D>::kBytes / 1024; ++i) {
    const u32x4_t x = *(lds_ptr)(uintptr_t)(sv + 1024 * i + 16 * lane);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2)
        sum[e & 1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, (uint32_t)x[e]),
                                                     __builtin_bit_cast(bf16x2_t, zero), sum[e & 1], false);
      else
        sum[e & 1] = __builtin_fmaf(__uint_as_float(x[e]), __uint_as_float(zero), sum[e & 1]);
    }
  }
  return __builtin_amdgcn_ballot_w64(!(sum[0] + sum[1] == 0.f)) == 0;
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Infinities and NaN of a tile become 0.
template <typename T, int D>
__device__ __forceinline__ void clear_non_finite(uint32_t sv, int lane) {
  typedef __attribute__((address_space(3))) u32x4_t* lds_ptr;
#pragma nounroll
  for (int i = 0; i < Tile<T, D>::kBytes / 1024; ++i) {
    const lds_ptr at = (lds_ptr)(uintptr_t)(sv + 1024 * i + 16 * lane);
    u32x4_t x = *at;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) {
        if (!finite(__uint_as_float(x[e] & 0xffff0000u))) x[e] &= 0xffffu;
        if (!finite(__uint_as_float(x[e] << 16))) x[e] &= 0xffff0000u;
      } else {
        if (!finite(__uint_as_float(x[e]))) x[e] = 0;
      }
    }
    *at = x;
  }
}

// kGroups: row groups of a block; kOnce: no other block reads its keys.
template <typename T, int D, int kGroups, bool kOnce>
__global__ __launch_bounds__(kWaves * 64, (sizeof(T) == 2 ? 2 : 1) + (kGroups == 4)) void tree_kernel(TreeArgs a) {
  typedef Tile<T, D> L;
  static_assert(kGroups == 1 || kGroups == 2 || kGroups == 4, "row groups of a block");
  constexpr int kStreams = kWaves / kGroups, kRows = 32 * kGroups;
  constexpr int kLoadsPerWave = L::kLoads / kGroups;
  constexpr int kVm = 2 * kLoadsPerWave;  // direct loads of a wave per tile
  static_assert(L::kLoads % kGroups == 0 && kVm < 63, "vector-memory counter");

  // (K, V) buffers: one a stream with one row group, else two
  __shared__ __attribute__((aligned(1024))) unsigned char s_tile[(kGroups == 1 ? 1 : 2) * kStreams * 2 * L::kBytes];
  __shared__ float s_m[kWaves][32], s_l[kWaves][32];
  __shared__ uint32_t s_mask[kRows * kMaskWords];  // the mask rows of the block's nodes
  __shared__ int s_far[kStreams];                  // values left out of the stream's sums (see keep_finite)

  // A unit is a (sequence, KV head) and a split; its row tiles read the same
  // keys, so they follow each other on one XCD (block index mod 8) and its L2.
  // Units go round the XCDs, so that long sequences spread.  With few units
  // the row tiles go round the XCDs instead.
  const int bid = blockIdx.x, units = a.num_units;
  int unit, row_tile, pair, split, b, g;
  if (units >= kSpreadUnits) {
    a.by_row_tiles.divide(bid >> 3, unit, row_tile);
    unit = unit * 8 + (bid & 7);
    if (unit >= units) return;
  } else {
    a.by_row_tiles.divide(bid, unit, row_tile);
  }
  row_tile = a.row_tiles - 1 - row_tile;  // (a chain's last rows see most keys)
  a.by_splits.divide(unit, pair, split);
  a.by_heads.divide(pair, b, g);
  const int heads = a.pv.kv_heads;

  // lengths by scalar loads (no kernel writes them while this one runs)
  typedef __attribute__((address_space(4))) const int32_t* const_ptr;
  const int n_alloc = a.num_nodes;
  const int len_given = ((const_ptr)a.cache_len)[b];
  const int nodes_given = a.nodes_of ? ((const_ptr)a.nodes_of)[b] : n_alloc;

  // Blocks behind a sequence's last node give up their place before they load
  // anything (8 sequences of 109 to 301 nodes, 64 heads on 8: 47 -> 45 us); with
  // one row tile there are none, and nothing waits for the count.
  if (a.nodes_of && a.row_tiles > 1 && (row_tile * kRows) >> a.group_shift >= nodes_given) return;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % kGroups, stream = wave / kGroups;
  const int col = lane & 31, hg = lane >> 5;
  const int gshift = a.group_shift;
  const int r = row_tile * kRows + rg * 32 + col;  // this lane's row
  const int node = r >> gshift;

  // this split's tiles, cut from the host's bound; step s of a stream is tile
  // t_first + s * kStreams
  const int t_first = split * a.tiles_per_split + stream;
  const int shift = a.pv.page_shift, slot_mask = (1 << shift) - 1;

  // What depends on no length goes out first: the queries, the block's mask
  // rows, and the table entries of the stream's next 16 tiles (pages hold at
  // least 8 rows, so a tile has four: lane 4 s + i has that of rows 8 i .. of
  // step s).
  u32x4_t q[L::kFrags];
  {
    const int h = (g << gshift) + (r & ((1 << gshift) - 1));
    const char* row = static_cast<const char*>(a.q) +
                      (((int64_t)b * n_alloc + min(node, n_alloc - 1)) * a.num_q_heads + h) * L::kRowBytes + 16 * hg;
#pragma unroll
    for (int i = 0; i < L::kFrags; ++i) q[i] = *reinterpret_cast<const u32x4_t*>(row + 32 * i);
  }
  const int32_t* table = a.table + (int64_t)b * a.pv.max_pages;
  auto table_of = [&](int step, int at) __attribute__((always_inline)) {  // at: the lane
    const uint32_t key = (uint32_t)(t_first + (step + (at >> 2)) * kStreams) * kKeys + 8 * (at & 3);
    return table[min(key >> shift, (uint32_t)a.pv.max_pages - 1)];
  };
  int tbl = table_of(0, lane);
  // (asked for by now, all of them: each would wait for the one before it if
  // they were loaded where they are used)
  asm volatile("" : : "s"(len_given), "s"(nodes_given), "s"(a.mask), "s"(a.mask_stride), "s"(a.mask_words),
               "s"(a.max_len), "s"(a.k_pages), "s"(a.v_pages), "s"(a.pv.num_pages), "s"(a.tiles_per_split));
  const int node0 = (row_tile * kRows) >> gshift;
  if (a.mask) {
    const uint32_t* from = a.mask + b * a.mask_stride + (int64_t)node0 * a.mask_words;
    const int words = min(kRows >> gshift, n_alloc - node0) * a.mask_words;
    for (int i = tid; i < words; i += kWaves * 64) s_mask[i] = from[i];
  }
  if (tid < kStreams) s_far[tid] = 0;

  const int64_t cap = (int64_t)a.pv.max_pages << shift;
  const int nn = min(max(nodes_given, 0), n_alloc);
  const int len = (int)min((int64_t)min(max(len_given, 0), a.max_len), cap);
  if (node0 >= nn) return;  // no node in this block
  // keys any row of the block sees: in a chain none behind its last node
  const int node_end = a.mask ? nn : min(nn, ((row_tile * kRows + kRows - 1) >> gshift) + 1);
  const int keys = (int)min((int64_t)len + node_end, cap);
  const int last = keys - 1;
  const int tiles = (keys + kKeys - 1) / kKeys;
  const int t_end = min((split + 1) * a.tiles_per_split, tiles);

  // All of it has arrived before the first direct load, which the compiler
  // does not count: later waits are for the direct loads alone.  A row that is
  // no node gets zero queries: finite logits that nothing reads.
  __syncthreads();
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
#pragma unroll
  for (int i = 0; i < L::kFrags; ++i) {
    if (node >= nn) q[i] = u32x4_t{0, 0, 0, 0};
    asm volatile("" : "+v"(q[i]));
  }
  asm volatile("" : "+v"(tbl));
  __builtin_amdgcn_sched_barrier(0);

  const uint32_t npages = (uint32_t)a.pv.num_pages;
  const uint64_t head_bytes = (uint64_t)L::kRowBytes << shift, page_bytes = head_bytes * heads;
  const uintptr_t kpool = (uintptr_t)a.k_pages + g * head_bytes;
  const uintptr_t v_minus_k = (uintptr_t)a.v_pages - (uintptr_t)a.k_pages;
  const uint32_t lds0 = lds_addr(s_tile);
  const int lrow = lane / L::kChunks, lpos = lane % L::kChunks;  // row within a load, LDS chunk position

  // A run is 8 rows of a tile, all in one page.  Sixteen steps at a time, lane
  // 4 s + i works out where run i of step s starts in the K pool (run_at) and
  // whether its page is in range (run_ok).  Runs past the last key take its run's
  // place, runs without a page that of page 0: rows that exist, of keys that
  // count as not seen.
  constexpr int kShare = kKeys / kGroups;  // rows of a tile that a wave loads, from rg * kShare on
  constexpr int kRuns = kShare / 8;
  uint32_t run_lo = 0, run_hi = 0;
  uint64_t run_ok = 0;
  auto place_runs = [&](int step, int entry, int at) __attribute__((always_inline)) {
    const int kb = (t_first + (step + (at >> 2)) * kStreams) * kKeys;
    const int run = min(at & 3, max((last - kb) >> 3, 0));
    const uint32_t e = (uint32_t)__shfl(entry, (at & ~3) + run, 64);
    const uint64_t start = kpool + (uint64_t)(e < npages ? e : 0u) * page_bytes +
                           (uint32_t)((kb + 8 * run) & slot_mask) * L::kRowBytes;
    run_lo = (uint32_t)start;
    run_hi = (uint32_t)(start >> 32);
    run_ok = __builtin_amdgcn_ballot_w64(e < npages);
  };
  place_runs(0, tbl, lane);
  struct Entries {
    uint64_t at[kRuns];  // where the runs that this wave loads start in the K pool
    uint32_t present;    // the tile's keys whose page is in range, as bits
  };
  auto entries = [&](int step) __attribute__((always_inline)) {
    const int lane0 = 4 * (step & 15);
    if (lane0 == 0 && step) {
      int at = lane;
      asm volatile("" : "+v"(at));  // (nothing of this is kept in registers meanwhile)
      const int entry = table_of(step, at);
      __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);  // (here, not at every use)
      place_runs(step, entry, at);
      asm volatile("" : "+v"(run_lo), "+v"(run_hi));
    }
    Entries x;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int from = lane0 + rg * kRuns + i;
      x.at[i] = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(run_hi, from) << 32 |
                (uint32_t)__builtin_amdgcn_readlane(run_lo, from);
    }
    const uint32_t ok = (uint32_t)(run_ok >> lane0) & 15u;
    x.present = ((ok * 0x00204081u) & 0x01010101u) * 0xffu;  // each bit to a byte
    return x;
  };
  // This wave's share of tile t into LDS at dst (K or V).  The lane offset of a
  // load within its run is the same for every tile.  In the last tile, rows past
  // the last key read that key's row.
  const uint32_t lane_k = lrow * L::kRowBytes + ((lpos ^ L::k(lrow) ^ L::k(rg * kShare)) << 4);
  const uint32_t lane_v = lrow * L::kRowBytes + ((lpos ^ L::v(lrow)) << 4);
  auto load = [&](int t, const Entries& x, uint32_t dst, bool is_v) __attribute__((always_inline)) {
    auto move = [&](uint64_t at, uint32_t off, int in) __attribute__((always_inline)) {
      if (is_v) at += v_minus_k;
      // (the same in every lane, which the compiler does not always see)
      const uint32_t to = __builtin_amdgcn_readfirstlane(dst + (rg * kShare + in) * L::kRowBytes);
      if constexpr (kOnce) lds_dma16_nt((const void*)at, off, to);
      else lds_dma16((const void*)at, off, to);
    };
    if (t * kKeys + kKeys <= keys) {
#pragma unroll
      for (int i = 0; i < kLoadsPerWave; ++i) {
        const int in = i * L::kRowsPerLoad;  // (a constant)
        const uint32_t swz = (is_v ? L::v(in) : L::k(in)) << 4;
        move(x.at[in / 8], ((is_v ? lane_v : lane_k) ^ swz) + (in & 7) * L::kRowBytes, in);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoadsPerWave; ++i) {
        const int in = i * L::kRowsPerLoad, row = rg * kShare + in + lrow;
        const int swz = is_v ? L::v(row) : L::k(row);
        const int to = t * kKeys + (row | 7) > last ? min((in & 7) + lrow, last & 7) : (in & 7) + lrow;
        move(x.at[in / 8], to * L::kRowBytes + ((lpos ^ swz) << 4), in);
      }
    }
  };

  f32x16_t o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m_run = neg_inf(), l_run = 0.f;

  // the 32 keys from kb on that this lane's row sees
  auto tile_bits = [&](int kb, uint32_t present) __attribute__((always_inline)) -> uint32_t {
    uint32_t bits = ~0u;
    int lim = keys - kb;
    if (a.mask) {
      const int j0 = kb - len, w = j0 >> 5;  // node of the first key (below 0: cached keys)
      const uint32_t* row = s_mask + (node - node0) * a.mask_words;
      const uint32_t lo = row[min(max(w, 0), a.mask_words - 1)], hi = row[min(max(w + 1, 0), a.mask_words - 1)];
      if (w >= -1) bits = (uint32_t)((((uint64_t)hi << 32) | (w >= 0 ? lo : ~0u)) >> (j0 & 31));
      // (words past the last are of nodes past the last: cut by lim)
    } else {
      lim = min(lim, len + node + 1 - kb);
    }
    if (lim < 32) bits &= lim > 0 ? (1u << lim) - 1 : 0u;
    return node < nn ? bits & present : 0u;
  };

  // softmax of a tile's logits: st becomes the weights
  auto softmax = [&](const f32x16_t& st, bool masked, uint32_t bits, float (&p)[16]) __attribute__((always_inline)) {
    float mt = neg_inf();
    if (masked) {
      const uint32_t mine = bits >> (4 * hg);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = (mine >> (8 * (i / 4) + i % 4)) & 1 ? st[i] : neg_inf();
        mt = fmaxf(mt, p[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = st[i];
        mt = fmaxf(mt, p[i]);
      }
    }
    mt = partner_max(mt) * a.scale_log2;  // the scale is > 0
    // (one branch for the wave: the sums of rows that stay are multiplied by 1)
    const bool grow = mt > m_run + kSlack;
    if (__builtin_amdgcn_ballot_w64(grow)) {
      const float corr = grow ? fast_exp2(m_run - mt) : 1.f;
      l_run *= corr;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= corr;
      m_run = grow ? mt : m_run;
    }
    const float m_use = m_run == neg_inf() ? 0.f : m_run;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = fast_exp2(__builtin_fmaf(p[i], a.scale_log2, -m_use));
      sum += p[i];
    }
    l_run += sum;
  };

  // Before the values of a tile with bits are added: those that are not finite
  // become 0 (a row that does not see them would get 0 times infinity) and
  // s_far says that rows that do see them are owed them.  (The flag goes up
  // before the first value changes, so a wave that shares the tile finds the
  // one or the other.)
  auto keep_finite = [&](uint32_t sv) __attribute__((always_inline)) {
    if (!all_finite<T, D>(sv, lane)) {
      s_far[stream] = 1;
      clear_non_finite<T, D>(sv, lane);
      wait_lds();
    }
  };

  // A tile needs its bits where it reaches past the keys that every row of the
  // block sees (in a chain those up to its first node's) or lacks a page.
  const int seen = a.mask ? len : min(len + node0 + 1, keys);
  auto needs_bits = [&](int t, uint32_t present) { return t * kKeys + kKeys > seen || present != ~0u; };

  if constexpr (kGroups == 1) {
    // every wave its own stream: K and V buffer of its own, no barrier
    const uint32_t sk = lds0 + wave * 2 * L::kBytes, sv = sk + L::kBytes;
    if (t_first < t_end) {
      int t = t_first, step = 0;
      Entries x = entries(0);
      load(t, x, sk, false);
      load(t, x, sv, true);
      wait_vm<kVm / 2>();
      while (true) {
        const bool more = t + kStreams < t_end, masked = needs_bits(t, x.present);
        const uint32_t bits = masked ? tile_bits(t * kKeys, x.present) : ~0u;
        const f32x16_t st = scores<T, D>(sk, q, lane);
        wait_lds();
        ++step;
        if (more) {
          x = entries(step);
          load(t + kStreams, x, sk, false);
        }
        float p[16];
        softmax(st, masked, bits, p);
        if (more) wait_vm<kVm / 2>();
        else wait_vm<0>();
        if (masked) keep_finite(sv);
        add_values<T, D>(sv, p, o, lane);
        if (!more) break;
        wait_lds();
        t += kStreams;
        load(t, x, sv, true);
        wait_vm<kVm / 2>();
      }
    }
  } else {
    // two buffers a stream: a step's tile is computed while the next arrives
    const uint32_t base = lds0 + stream * 4 * L::kBytes;
    const int t_block = split * a.tiles_per_split;  // (a split behind the last key has no step)
    const int steps = t_block < t_end ? (t_end - t_block + kStreams - 1) / kStreams : 0;
    Entries x;
    x.present = 0;
    auto request = [&](int step) __attribute__((always_inline)) {
      const int t = t_first + step * kStreams;
      if (t >= t_end) return;
      const uint32_t dst = base + (uint32_t)(step & 1) * 2 * L::kBytes;
      x = entries(step);
      load(t, x, dst, false);
      load(t, x, dst + L::kBytes, true);
    };
    if (steps > 0) request(0);
    for (int step = 0; step < steps; ++step) {
      bare_barrier<0>();  // this step's tile has landed in every wave's part
      const int t = t_first + step * kStreams;
      const uint32_t present = x.present;
      request(step + 1);
      if (t < t_end) {
        const uint32_t sk = base + (uint32_t)(step & 1) * 2 * L::kBytes, sv = sk + L::kBytes;
        const bool masked = needs_bits(t, present);
        const uint32_t bits = masked ? tile_bits(t * kKeys, present) : ~0u;
        const f32x16_t st = scores<T, D>(sk, q, lane);
        float p[16];
        softmax(st, masked, bits, p);
        if (masked) keep_finite(sv);
        add_values<T, D>(sv, p, o, lane);
      }
    }
  }
  __syncthreads();  // every wave is done with the tiles, and no load is in flight

  // What keep_finite left out, key by key from the cache (rare: a model that
  // has gone wrong).
  if (s_far[stream]) {
    const float m_use = m_run == neg_inf() ? 0.f : m_run;
#pragma nounroll
    for (int key = t_first * kKeys; key < min(t_end * kKeys, keys); ++key) {
      const int t = key / kKeys;
      if ((t - t_first) % kStreams) continue;
      uint32_t present = 0;
      for (int i = 0; i < 4; ++i)
        present |= (uint32_t)table[min(t * kKeys + 8 * i, last) >> shift] < npages ? 0xffu << (8 * i) : 0u;
      if (!needs_bits(t, present) || !(present >> (key % kKeys) & 1)) continue;
      const bool see = tile_bits(t * kKeys, present) >> (key % kKeys) & 1;
      const uint64_t at = (uint64_t)(uint32_t)table[key >> shift] * page_bytes + (uint64_t)(key & slot_mask) * L::kRowBytes;
      const T* k = reinterpret_cast<const T*>(kpool + at);
      const T* v = reinterpret_cast<const T*>(kpool + v_minus_k + at);
      constexpr int kElems = 16 / (int)sizeof(T);  // of a chunk; this lane's are 2 i + hg
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < L::kFrags; ++i) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(k + (2 * i + hg) * kElems);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 2)
            z = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, (uint32_t)x[e]),
                                                __builtin_bit_cast(bf16x2_t, (uint32_t)q[i][e]), z, false);
          else
            z = __builtin_fmaf(__uint_as_float(x[e]), __uint_as_float(q[i][e]), z);
        }
      }
      z = partner_sum(z);
      const float w = fast_exp2(__builtin_fmaf(z, a.scale_log2, -m_use));
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const T x = v[32 * db + 8 * (i / 4) + 4 * hg + i % 4];
          float f;
          if constexpr (sizeof(T) == 2) f = bf16_to_f32(x);
          else f = x;
          if (see && !finite(f)) o[db][i] += w * f;
        }
    }
  }

  const float l_tot = partner_sum(l_run);
  if constexpr (kStreams == 1) {
    // every wave has its rows whole: four values of a row at a time
    int at = lane;
    asm volatile("" : "+v"(at));  // (the row's number is worked out again, not kept through the loop)
    const int mine = row_tile * kRows + rg * 32 + (at & 31), half = at >> 5;
    if ((mine >> gshift) >= nn) return;
    const int64_t row = ((int64_t)b * n_alloc + (mine >> gshift)) * a.num_q_heads + (g << gshift) +
                        (mine & ((1 << gshift) - 1));
    const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;  // (nothing seen: 0)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int ig = 0; ig < 4; ++ig) {
        const int e = 32 * db + 8 * ig + 4 * half;
        const f32x16_t& x = o[db];
        if (a.num_splits == 1)
          Mfma<T>::store4(static_cast<T*>(a.out) + row * D + e, x[4 * ig] * inv, x[4 * ig + 1] * inv,
                          x[4 * ig + 2] * inv, x[4 * ig + 3] * inv);
        else
          Mfma<float>::store4(a.ws_o + (row * a.num_splits + split) * D + e, x[4 * ig], x[4 * ig + 1], x[4 * ig + 2],
                              x[4 * ig + 3]);
      }
    if (a.num_splits > 1 && half == 0) {
      a.ws_ml[(row * a.num_splits + split) * 2] = m_run;
      a.ws_ml[(row * a.num_splits + split) * 2 + 1] = l_tot;
    }
    return;
  }

  // the waves' rows through LDS: wave w's 32 x D sums at s_o + 32 w D, 16-byte
  // chunks swizzled by the row
  float* const s_o = reinterpret_cast<float*>(s_tile);
  constexpr int kO = D / 4;  // chunks of an output row
  {
    if (hg == 0) {
      s_m[wave][col] = m_run;
      s_l[wave][col] = l_tot;
    }
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int ig = 0; ig < 4; ++ig)
        *reinterpret_cast<f32x4_t*>(s_o + (wave * 32 + col) * D + (((8 * db + 2 * ig + hg) ^ (col & (kO - 1))) << 2)) =
            f32x4_t{o[db][4 * ig], o[db][4 * ig + 1], o[db][4 * ig + 2], o[db][4 * ig + 3]};
  }
  __syncthreads();
  for (int it = tid; it < kRows * (D / 8); it += kWaves * 64) {
    const int row = it / (D / 8), ch = it % (D / 8), rr = row & 31, rw = row >> 5;
    const int gr = row_tile * kRows + row, out_node = gr >> gshift;
    if (out_node >= nn) continue;
    float M = neg_inf();
#pragma unroll
    for (int s = 0; s < kStreams; ++s) M = fmaxf(M, s_m[s * kGroups + rw][rr]);
    float num[8] = {}, den = 0.f;
#pragma unroll
    for (int s = 0; s < kStreams; ++s) {
      const int w = s * kGroups + rw;
      const float ms = s_m[w][rr];
      const float f = ms == neg_inf() ? 0.f : fast_exp2(ms - M);
      den += f * s_l[w][rr];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const f32x4_t x =
            *reinterpret_cast<const f32x4_t*>(s_o + (w * 32 + rr) * D + (((2 * ch + c) ^ (rr & (kO - 1))) << 2));
#pragma unroll
        for (int e = 0; e < 4; ++e) num[4 * c + e] += f * x[e];
      }
    }
    const int64_t out_row = ((int64_t)b * n_alloc + out_node) * a.num_q_heads + (g << gshift) + (gr & ((1 << gshift) - 1));
    if (a.num_splits == 1) {
      const float inv = den == 0.f ? 0.f : 1.f / den;  // (nothing seen: 0)
#pragma unroll
      for (int e = 0; e < 8; ++e) num[e] *= inv;
      Chunk<T> x;
      x.from_float(num);
      x.store(static_cast<T*>(a.out) + out_row * D + 8 * ch);
    } else {
      Chunk<float> x;
      x.from_float(num);
      x.store(a.ws_o + (out_row * a.num_splits + split) * D + 8 * ch);
      if (ch == 0) {
        a.ws_ml[(out_row * a.num_splits + split) * 2] = M;
        a.ws_ml[(out_row * a.num_splits + split) * 2 + 1] = den;
      }
    }
  }
}

// Log-sum-exp merge of the split partials of a (sequence, node, head) row, in
// split order: D / 4 lanes a row, four elements a lane.
template <typename T, int D>
__global__ __launch_bounds__(kMergeThreads) void tree_merge_kernel(TreeArgs a) {
  constexpr int kLanes = D / 4, kRows = tree_merge_rows(D);
  const int b = blockIdx.y, e = threadIdx.x % kLanes;
  const int in = blockIdx.x * kRows + threadIdx.x / kLanes;  // (node, head) of the sequence
  const int n = a.nodes_of ? min(a.nodes_of[b], a.num_nodes) : a.num_nodes;
  if (in >= (int64_t)n * a.num_q_heads) return;
  const int S = a.num_splits;
  const int64_t row = (int64_t)b * a.num_nodes * a.num_q_heads + in;
  const float2* ml = reinterpret_cast<const float2*>(a.ws_ml) + row * S;
  const f32x4_t* po = reinterpret_cast<const f32x4_t*>(a.ws_o + row * S * D) + e;
  // kAtOnce splits at a time, all of their loads under way together
  constexpr int kAtOnce = 8;
  float M = neg_inf(), den = 0.f;
  f32x4_t num = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < S; s0 += kAtOnce) {
    float2 x[kAtOnce];
    f32x4_t v[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      x[k] = make_float2(neg_inf(), 0.f);
      v[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (s0 + k < S) {
        x[k] = ml[s0 + k];
        v[k] = po[(s0 + k) * kLanes];
      }
    }
    float top = M;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, x[k].x);
    const float ref = top == neg_inf() ? 0.f : top;
    const float back = fast_exp2(M - ref);
    den *= back;
#pragma unroll
    for (int i = 0; i < 4; ++i) num[i] *= back;
    M = top;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float f = fast_exp2(x[k].x - ref);
      den += f * x[k].y;
#pragma unroll
      for (int i = 0; i < 4; ++i) num[i] += f * v[k][i];
    }
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;  // (nothing seen: 0)
  if constexpr (sizeof(T) == 2) {
    uint2 x = make_uint2(pack_bf16x2(num[0] * inv, num[1] * inv), pack_bf16x2(num[2] * inv, num[3] * inv));
    *reinterpret_cast<uint2*>(static_cast<bf16_bits*>(a.out) + row * D + 4 * e) = x;
  } else {
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + row * D + 4 * e) =
        f32x4_t{num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv};
  }
}

template <typename T, int D>
hipError_t launch_tree_d(const TreeArgs& a, int batch, hipStream_t s) {
  TreeArgs x = a;
  const int groups = a.row_groups;
  x.by_row_tiles = FastDivide(a.row_tiles);
  x.by_splits = FastDivide(a.num_splits);
  x.by_heads = FastDivide(a.pv.kv_heads);
  x.num_units = batch * a.pv.kv_heads * a.num_splits;
  const int64_t units = x.num_units >= kSpreadUnits ? ((int64_t)x.num_units + 7) / 8 * 8 : x.num_units;
  const dim3 grid((uint32_t)(units * a.row_tiles)), block(kWaves * 64);
  // one row tile: the keys are read once, past the caches (64 sequences of 862
  // keys 47.8 -> 41.7 us, 16 of 7724 keys 103 -> 92); more tiles share them in
  // L2 (301 nodes of 8 heads a group: 61 us, 64 without)
  const bool once = a.row_tiles == 1;
  if (groups == 1 && once) return launch_struct(tree_kernel<T, D, 1, true>, grid, block, s, x);
  if (groups == 1) return launch_struct(tree_kernel<T, D, 1, false>, grid, block, s, x);
  if (groups == 2 && once) return launch_struct(tree_kernel<T, D, 2, true>, grid, block, s, x);
  if (groups == 2) return launch_struct(tree_kernel<T, D, 2, false>, grid, block, s, x);
  if (once) return launch_struct(tree_kernel<T, D, 4, true>, grid, block, s, x);
  return launch_struct(tree_kernel<T, D, 4, false>, grid, block, s, x);
}

}  // namespace

hipError_t launch_tree(const TreeArgs& a, int dtype, int head_dim, int batch, hipStream_t s) {
  if (dtype == 1) {
    if (head_dim == 128) return launch_tree_d<bf16_bits, 128>(a, batch, s);
    return launch_tree_d<bf16_bits, 64>(a, batch, s);
  }
  if (head_dim == 128) return launch_tree_d<float, 128>(a, batch, s);
  return launch_tree_d<float, 64>(a, batch, s);
}

template <typename T, int D>
hipError_t launch_merge_d(const TreeArgs& a, int batch, hipStream_t s) {
  const int per = tree_merge_rows(D);
  const dim3 grid((uint32_t)(((int64_t)a.num_nodes * a.num_q_heads + per - 1) / per), batch), block(kMergeThreads);
  return launch_struct(tree_merge_kernel<T, D>, grid, block, s, a);
}

hipError_t launch_tree_merge(const TreeArgs& a, int dtype, int head_dim, int batch, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? launch_merge_d<bf16_bits, 128>(a, batch, s) : launch_merge_d<bf16_bits, 64>(a, batch, s);
  return head_dim == 128 ? launch_merge_d<float, 128>(a, batch, s) : launch_merge_d<float, 64>(a, batch, s);
}

}  // namespace skv
