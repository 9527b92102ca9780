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
// v_mfma_f32_32x32x16_bf16 with the weights rounded to bf16 and fp32 sums,
// fp32 takes v_mfma_f32_32x32x2_f32.
//
// K/V tiles go from the paged cache straight into LDS (direct loads of 16 bytes
// a lane), rows unpadded and their 16-byte chunks XOR-swizzled so that operand
// reads are spread over the banks.
//
// With one row group every wave streams its own tiles through its own K and V
// buffer, with no barrier: the next K tile is requested as soon as S^T is
// computed, the next V tile as soon as O^T is, so a wave nearly always has a
// tile in flight, and two blocks of 64 KB share a CU.  With two or four row
// groups the waves of a stream load a tile together, one barrier per tile, one
// (kGroups = 2) or three tiles ahead.
//
// Tiles below L need no mask.  In the others each lane has its row's 32 bits; a
// row's weight of a key it does not see is 0, and since 0 times infinity is
// not, a tile of these whose values are not all finite takes its products one
// key at a time instead.
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
constexpr int kKeys = 32;   // keys per tile
constexpr int kWaves = 4;

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

// Whether all values of a tile are finite (the same in every lane).
template <typename T, int D>
__device__ __forceinline__ bool all_finite(uint32_t sv, int lane) {
  typedef __attribute__((address_space(3))) const u32x4_t* lds_ptr;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < Tile<T, D>::kBytes / 1024; ++i) {
    const u32x4_t x = *(lds_ptr)(uintptr_t)(sv + 1024 * i + 16 * lane);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bad = bad || (x[e] & 0x7f800000u) == 0x7f800000u;
      if (sizeof(T) == 2) bad = bad || (x[e] & 0x7f80u) == 0x7f80u;
    }
  }
  return __builtin_amdgcn_ballot_w64(bad) == 0;
}

// add_values for a tile with infinities or NaN among its values, key by key: a
// row takes the keys of its bits only.
template <typename T, int D>
__device__ __forceinline__ void add_values_by_key(uint32_t sv, const float (&p)[16], uint32_t bits,
                                                  f32x16_t (&o)[D / 32], int lane) {
  typedef Tile<T, D> L;
  const int col = lane & 31, hg = lane >> 5;
#pragma nounroll
  for (int key = 0; key < kKeys; ++key) {
    const int at = 4 * (key >> 3) + (key & 3);  // its element, in the lanes of half (key / 4) % 2
    float w = p[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) w = i == at ? p[i] : w;
    w = __shfl(w, col + 32 * ((key >> 2) & 1), 64);
    const bool see = (bits >> key) & 1;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int ig = 0; ig < 4; ++ig) {
        float v[4];
        if constexpr (sizeof(T) == 2) {
          typedef __attribute__((address_space(3))) const uint64_t* lds_ptr;
          const uint64_t x = *(lds_ptr)(uintptr_t)(sv + key * L::kRowBytes + ((4 * db + ig) ^ L::v(key)) * 16 + 8 * hg);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = bf16_to_f32((uint32_t)(x >> (16 * e)) & 0xffffu);
        } else {
          typedef __attribute__((address_space(3))) const f32x4_t* lds_ptr;
          const f32x4_t x = *(lds_ptr)(uintptr_t)(sv + key * L::kRowBytes + ((8 * db + 2 * ig + hg) ^ L::v(key)) * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = x[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[db][4 * ig + e] += see ? w * v[e] : 0.f;
      }
  }
}

// kGroups: row groups of a block (1, 2 or 4).
template <typename T, int D, int kGroups>
struct TreeShape {
  static constexpr int kStreams = kWaves / kGroups;
  static constexpr int kBuffers = kGroups;  // tile buffers of a stream
  static constexpr int kRows = 32 * kGroups;
  static constexpr int kTiles = kStreams * kBuffers;  // (always four)
};

template <typename T, int D, int kGroups>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) == 2 ? 2 : 1) void tree_kernel(TreeArgs a) {
  typedef Tile<T, D> L;
  typedef TreeShape<T, D, kGroups> S;
  constexpr int kStreams = S::kStreams, kBuffers = S::kBuffers;
  constexpr int kLoadsPerWave = L::kLoads / kGroups;
  constexpr int kVm = 2 * kLoadsPerWave;  // direct loads of a wave per tile
  static_assert(L::kLoads % kGroups == 0 && kVm * (kBuffers > 1 ? kBuffers - 1 : 1) < 63, "vector-memory counter");

  // K and V tile i at s_tile + 2 i and 2 i + 1 tiles
  __shared__ __attribute__((aligned(1024))) unsigned char s_tile[2 * S::kTiles * L::kBytes];
  __shared__ float s_m[kWaves][32], s_l[kWaves][32];

  // XCD x takes a contiguous range of items, (pair, split) with their row
  // tiles innermost: the tiles that read the same keys run side by side on one
  // L2.
  const int nblk = gridDim.x, per_xcd = nblk >> 3, rem = nblk & 7, xcd = blockIdx.x & 7;
  const int item = xcd * per_xcd + min(xcd, rem) + (blockIdx.x >> 3);
  const int row_tile = item % a.row_tiles, rest = item / a.row_tiles;
  const int split = rest % a.num_splits, pair = rest / a.num_splits;
  const int heads = a.pv.kv_heads, b = pair / heads, g = pair % heads;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % kGroups, stream = wave / kGroups;
  const int col = lane & 31, hg = lane >> 5;
  const int gshift = a.group_shift;
  const int r = row_tile * S::kRows + rg * 32 + col;  // this lane's row
  const int node = r >> gshift;
  const int n_alloc = a.num_nodes;

  // the queries first: they depend on no length
  u32x4_t q[L::kFrags];
  {
    const int h = (g << gshift) + (r & ((1 << gshift) - 1));
    const char* row = static_cast<const char*>(a.q) +
                      (((int64_t)b * n_alloc + min(node, n_alloc - 1)) * a.num_q_heads + h) * L::kRowBytes + 16 * hg;
#pragma unroll
    for (int i = 0; i < L::kFrags; ++i) q[i] = *reinterpret_cast<const u32x4_t*>(row + 32 * i);
  }

  // lengths and the first table entries come by scalar loads (no kernel writes
  // them while this one runs)
  typedef __attribute__((address_space(4))) const int32_t* const_ptr;
  const int shift = a.pv.page_shift, slot_mask = (1 << shift) - 1;
  const int64_t cap = (int64_t)a.pv.max_pages << shift;
  const int nn = a.nodes_of ? min(max(((const_ptr)a.nodes_of)[b], 0), n_alloc) : n_alloc;
  const int len = (int)min((int64_t)min(max(((const_ptr)a.cache_len)[b], 0), a.max_len), cap);
  const int node0 = (row_tile * S::kRows) >> gshift;
  // keys any row of the block sees: in a chain none behind its last node
  const int node_end = a.mask ? nn : min(nn, ((row_tile * S::kRows + S::kRows - 1) >> gshift) + 1);
  const int keys = (int)min((int64_t)len + node_end, cap);
  const int last = keys - 1;
  const int tiles = (keys + kKeys - 1) / kKeys;
  // this split's tiles, cut from the host's bound
  const int t_begin = min(split * a.tiles_per_split, tiles), t_end = min(t_begin + a.tiles_per_split, tiles);
  const int steps = (t_end - t_begin + kStreams - 1) / kStreams;

  const const_ptr table = (const_ptr)(a.table + (int64_t)b * a.pv.max_pages);
  const uint32_t npages = (uint32_t)a.pv.num_pages;
  const uint64_t head_bytes = (uint64_t)L::kRowBytes << shift, page_bytes = head_bytes * heads;
  const uintptr_t kpool = (uintptr_t)a.k_pages + g * head_bytes;
  const uintptr_t v_minus_k = (uintptr_t)a.v_pages - (uintptr_t)a.k_pages;
  const uint32_t lds0 = lds_addr(s_tile);
  const int lrow = lane / L::kChunks, lpos = lane % L::kChunks;  // row within a load, LDS chunk position

  // Pages hold at least 8 rows: a tile has four table entries, and a load's
  // rows lie in one page.  Keys past the last one read the last one.
  struct Entries {
    int e[4];
  };
  auto entries = [&](int t) __attribute__((always_inline)) {
    Entries x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.e[i] = table[min(t * kKeys + 8 * i, last) >> shift];
    return x;
  };
  // keys of a tile whose page is in range, as bits
  auto present = [&](const Entries& x) __attribute__((always_inline)) {
    uint32_t ok = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) ok |= (uint32_t)x.e[i] < npages ? 0xffu << (8 * i) : 0u;
    return ok;
  };
  // this wave's share of tile t, its rows from rg * kShare on (table entries
  // own[i] for rows 8 i.. of it), into LDS at dst (K or V)
  constexpr int kShare = kKeys / kGroups;
  auto load = [&](int t, const Entries& own, uint32_t dst, bool is_v) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kLoadsPerWave; ++i) {
      const int in = i * L::kRowsPerLoad;  // (a constant)
      const int e = own.e[in / 8];
      const uint32_t page = (uint32_t)e < npages ? (uint32_t)e : 0u;  // a bad entry reads an in-range page
      const uintptr_t base = kpool + (uint64_t)page * page_bytes + (is_v ? v_minus_k : 0);
      const int row0 = rg * kShare + in, row = row0 + lrow;
      const int key = min(t * kKeys + row, last);
      const int swz = is_v ? L::v(row) : L::k(row);
      lds_dma16((const void*)base, (uint32_t)((key & slot_mask) * L::kRowBytes + ((lpos ^ swz) << 4)),
                dst + row0 * L::kRowBytes);
    }
  };

  f32x16_t o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m_run = neg_inf(), l_run = 0.f;

  // the 32 keys from kb on that this lane's row sees
  const uint32_t* mask_row =
      a.mask ? a.mask + b * a.mask_stride + (int64_t)min(node, n_alloc - 1) * a.mask_words : nullptr;
  auto tile_bits = [&](int kb, uint32_t ok) __attribute__((always_inline)) -> uint32_t {
    uint32_t bits;
    int lim = keys - kb;
    if (a.mask) {
      const int j0 = kb - len, w = j0 >> 5;  // (w >= -1: the tile reaches past len)
      const uint32_t lo = w >= 0 ? (w < a.mask_words ? mask_row[w] : 0u) : ~0u;
      const uint32_t hi = w + 1 < a.mask_words && w + 1 >= 0 ? mask_row[w + 1] : 0u;
      bits = w < -1 ? ~0u : (uint32_t)((((uint64_t)hi << 32) | lo) >> (j0 & 31));
    } else {
      bits = ~0u;
      lim = min(lim, len + node + 1 - kb);
    }
    if (lim < 32) bits &= lim > 0 ? (1u << lim) - 1 : 0u;
    return node < nn ? bits & ok : 0u;
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
    if (mt > m_run + kSlack) {
      if (m_run != neg_inf()) {  // (before the first visible key o and l are still 0)
        const float corr = fast_exp2(m_run - mt);
        l_run *= corr;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= corr;
      }
      m_run = mt;
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

  // A tile needs its bits where it reaches past len or lacks a page.
  auto needs_bits = [&](int t, uint32_t ok) { return t * kKeys + kKeys > len || ok != ~0u; };
  if (node0 >= nn) return;  // no node in this block

  // The queries have arrived, by and large, when the first table entries have.
  // Waiting for them here, before the first direct load (which the compiler
  // does not count), keeps later waits on the direct loads alone.  A row that
  // is no node gets zero queries: finite logits that nothing reads.
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
#pragma unroll
  for (int i = 0; i < L::kFrags; ++i) {
    if (node >= nn) q[i] = u32x4_t{0, 0, 0, 0};
    asm volatile("" : "+v"(q[i]));
  }
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (kGroups == 1) {
    // every wave its own stream: K and V buffer of its own, no barrier
    const uint32_t sk = lds0 + wave * 2 * L::kBytes, sv = sk + L::kBytes;
    int t = t_begin + wave;
    if (t < t_end) {
      Entries x = entries(t);
      uint32_t ok = present(x);
      load(t, x, sk, false);
      load(t, x, sv, true);
      if (t + kWaves < t_end) x = entries(t + kWaves);
      wait_vm<kVm / 2>();
      while (true) {
        const bool more = t + kWaves < t_end, masked = needs_bits(t, ok);
        uint32_t bits = masked ? tile_bits(t * kKeys, ok) : ~0u;
        asm volatile("" : "+v"(bits));  // (loaded before the next K tile is requested)
        const f32x16_t st = scores<T, D>(sk, q, lane);
        wait_lds();
        if (more) load(t + kWaves, x, sk, false);
        float p[16];
        softmax(st, masked, bits, p);
        if (more) wait_vm<kVm / 2>();
        else wait_vm<0>();
        if (masked && !all_finite<T, D>(sv, lane)) add_values_by_key<T, D>(sv, p, bits, o, lane);
        else add_values<T, D>(sv, p, o, lane);
        if (!more) break;
        wait_lds();
        load(t + kWaves, x, sv, true);
        ok = present(x);
        t += kWaves;
        if (t + kWaves < t_end) x = entries(t + kWaves);
        wait_vm<kVm / 2>();
      }
    }
  } else {
    // tile `step` of the stream, kBuffers - 1 tiles ahead
    const uint32_t base = lds0 + stream * kBuffers * 2 * L::kBytes;
    auto buffer = [&](int step) { return base + (uint32_t)(step % kBuffers) * 2 * L::kBytes; };
    auto tile_of = [&](int step) { return t_begin + step * kStreams + stream; };
    uint32_t oks[kBuffers];  // of the tiles in flight, the next one first
    auto request = [&](int step) __attribute__((always_inline)) -> uint32_t {
      const int t = tile_of(step);
      if (t >= t_end) return 0;
      Entries own;
#pragma unroll
      for (int i = 0; i < 4; ++i) own.e[i] = table[min(t * kKeys + rg * kShare + 8 * (i % (kShare / 8)), last) >> shift];
      const Entries x = entries(t);
      load(t, own, buffer(step), false);
      load(t, own, buffer(step) + L::kBytes, true);
      return present(x);
    };
#pragma unroll
    for (int i = 0; i < kBuffers - 1; ++i) oks[i] = i < steps ? request(i) : 0;
    for (int step = 0; step < steps; ++step) {
      // tile `step` has landed when only the tiles behind it are in flight
      if (kBuffers > 2 && tile_of(step + kBuffers - 2) < t_end) bare_barrier<kVm * (kBuffers - 2)>();
      else bare_barrier<0>();
      oks[kBuffers - 1] = step + kBuffers - 1 < steps ? request(step + kBuffers - 1) : 0;
      const int t = tile_of(step);
      const uint32_t ok = oks[0];
      if (t < t_end) {
        const uint32_t sk = buffer(step), sv = sk + L::kBytes;
        const bool masked = needs_bits(t, ok);
        const uint32_t bits = masked ? tile_bits(t * kKeys, ok) : ~0u;
        const f32x16_t st = scores<T, D>(sk, q, lane);
        float p[16];
        softmax(st, masked, bits, p);
        if (masked && !all_finite<T, D>(sv, lane)) add_values_by_key<T, D>(sv, p, bits, o, lane);
        else add_values<T, D>(sv, p, o, lane);
      }
#pragma unroll
      for (int i = 0; i + 1 < kBuffers; ++i) oks[i] = oks[i + 1];
    }
  }
  __syncthreads();  // every wave is done with the tiles, and no load is in flight

  // the waves' rows through LDS: wave w's 32 x D sums at s_o + 32 w D, 16-byte
  // chunks swizzled by the row
  float* const s_o = reinterpret_cast<float*>(s_tile);
  constexpr int kO = D / 4;  // chunks of an output row
  {
    const float l_tot = partner_sum(l_run);
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
  for (int it = tid; it < S::kRows * (D / 8); it += kWaves * 64) {
    const int row = it / (D / 8), ch = it % (D / 8), rr = row & 31, rw = row >> 5;
    const int gr = row_tile * S::kRows + row, out_node = gr >> gshift;
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
hipError_t launch_tree_d(const TreeArgs& a, int batch, hipStream_t s) {
  TreeArgs x = a;
  const int groups = tree_row_groups((int64_t)a.num_nodes << a.group_shift);
  const dim3 grid((uint32_t)((int64_t)batch * a.pv.kv_heads * a.num_splits * a.row_tiles)), block(kWaves * 64);
  if (groups == 1) return launch_struct(tree_kernel<T, D, 1>, grid, block, s, x);
  if (groups == 2) return launch_struct(tree_kernel<T, D, 2>, grid, block, s, x);
  return launch_struct(tree_kernel<T, D, 4>, grid, block, s, x);
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
