// One decoding step of attention for groups of sequences that share long prefixes.
//
// A member's output is the softmax over its group's prefix and its own entries.
// Every member sees the whole prefix, so the rows of one KV head, members times the
// G query heads of its group, are one matrix and the prefix is read once for all
// of them; what they have of their own is read once each, with G rows.  Both are
// partial results of the same softmax: blocks of one launch compute them (prefix
// blocks: a group, KV head, range of its keys and 32 rows; the waves of own blocks: a
// sequence, KV head and range of its keys each), and a second launch merges a row's
// partials by log-sum-exp, in a fixed order.
//
// A block of four waves takes 32 rows and a range of keys in tiles of 32, which the
// waves deal out (of its own entries a wave has a whole range); each holds the query
// rows in registers and per tile computes S^T = K Q^T and O^T += V^T P^T on the 32x32
// matrix products (tile_attn.hpp) with the online softmax between them.  Tiles go
// from the paged cache straight into LDS, into a K and a V buffer of the wave's own,
// the next K requested as soon as S^T is there, the next V as soon as O^T is: no
// barrier.  More than 32 rows are more blocks that read the same keys, side by side
// on one XCD and out of its L2 (on different XCDs HBM gives the keys to each: 64
// questions about 7532 entries 24 us, 21 so).  There the kernel takes 17 us and the
// merge 4: a CU reads about 57 GB/s whatever is on its way, and four row tiles bring
// 123 MB into LDS; more splits or fewer rows a block cost partial rows or reads.  Six
// recordings of 1532 entries with 40 questions of up to 301 own ones take 17.6 and 4
// us, 59 MB.  Blocks of 64 or 128 rows, whose waves
// share a tile and a barrier, are slower (23 and 25 us), also with four tiles on their
// way, and so are blocks of eight waves, and waves with 64 rows each (one block a CU
// for their 297 registers: 24 us).
//
// Every row of a block sees the same keys, so keys that are not there (past the
// last, or without a page) are masked for all: their logits become -inf and their
// values 0 in LDS.
//
// With bf16 the weights are rounded to bf16 before the product with V, as in this
// library's other attention (at most 2^-8 of each; the sum is of those before): the
// matrix products take both operands in one type.  It takes the outputs' error against
// 64 bits from 0.0017 of their size, the outputs' own rounding, to 0.0020 .. 0.0023.
#include "kernels_shared.hpp"
#include "tile_attn.hpp"

namespace skv {

namespace {

constexpr int kWaves = 4;
static_assert(kSharedKeys == kKeys, "the tile that the host cuts splits by");

// What a block, or a wave, attends: rows (`rows` of them, of which it has 32 from
// `row0` on) and keys.
struct Job {
  const KeySource* src;
  int entry;           // row of the block table
  int g;               // KV head
  int first_b, rows;   // sequence of the first row, rows (sequence, head of the group)
  int row0;
  int keys;            // of the source
  int tile0, tile1;    // key tiles of this split
  int part;            // which partial result it is
};

// kOnce: no other block reads its keys.  kAlone: every wave has a job of its own and
// meets no barrier.
template <typename T, int D, bool kOnce, bool kAlone>
__device__ __forceinline__ void attend(const SharedArgs& a, const Job& job, unsigned char* s_tile, float (*s_m)[32],
                                       float (*s_l)[32]) {
  typedef Tile<T, D> L;
  constexpr int kStreams = kAlone ? 1 : kWaves;  // waves that the tiles are dealt to
  constexpr int kRuns = kKeys / 8;               // runs of 8 rows of a tile
  static_assert(L::kLoads < 63, "vector-memory counter");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int stream = kAlone ? 0 : wave;
  const int col = lane & 31, hg = lane >> 5;
  const int parts = a.prefix_splits + a.own_splits, gshift = a.group_shift, gmask = (1 << gshift) - 1;
  const KeySource& src = *job.src;
  const int shift = src.pv.page_shift, slot_mask = (1 << shift) - 1, heads = src.pv.kv_heads;

  // output row of row r of the job
  auto out_row = [&](int r) {
    return ((int64_t)job.first_b + (r >> gshift)) * a.num_q_heads + (job.g << gshift) + (r & gmask);
  };
  const int t_end = min(job.tile1, (job.keys + kKeys - 1) / kKeys), last = job.keys - 1;
  if (job.tile0 >= t_end) {  // nothing here: the merge passes over it
    const int r = job.row0 + (kAlone ? lane : tid);
    if (r < min(job.rows, job.row0 + 32)) {
      const int64_t at = out_row(r) * parts + job.part;
      a.ws_ml[2 * at] = neg_inf();
      a.ws_ml[2 * at + 1] = 0.f;
    }
    return;
  }

  const int r = job.row0 + col;  // this lane's row
  u32x4_t q[L::kFrags];
  {
    const char* row = static_cast<const char*>(a.q) + out_row(min(r, job.rows - 1)) * L::kRowBytes + 16 * hg;
#pragma unroll
    for (int i = 0; i < L::kFrags; ++i) q[i] = *reinterpret_cast<const u32x4_t*>(row + 32 * i);
  }
  const int t_first = job.tile0 + stream;
  // table entries of the stream's next 16 tiles: lane 4 s + i has that of rows 8 i
  // .. of step s
  const int32_t* table = src.table + (int64_t)job.entry * src.pv.max_pages;
  auto table_of = [&](int step, int at) __attribute__((always_inline)) {
    const uint32_t key = (uint32_t)(t_first + (step + (at >> 2)) * kStreams) * kKeys + 8 * (at & 3);
    return table[min(key >> shift, (uint32_t)src.pv.max_pages - 1)];
  };
  int tbl = table_of(0, lane);
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);  // (the direct loads that follow are counted alone)
#pragma unroll
  for (int i = 0; i < L::kFrags; ++i) {
    if (r >= job.rows) q[i] = u32x4_t{0, 0, 0, 0};
    asm volatile("" : "+v"(q[i]));
  }
  asm volatile("" : "+v"(tbl));
  __builtin_amdgcn_sched_barrier(0);

  const uint32_t npages = (uint32_t)src.pv.num_pages;
  const uint64_t head_bytes = (uint64_t)L::kRowBytes << shift, page_bytes = head_bytes * heads;
  const uintptr_t kpool = (uintptr_t)src.k_pages + job.g * head_bytes;
  const uintptr_t v_minus_k = (uintptr_t)src.v_pages - (uintptr_t)src.k_pages;
  const uint32_t lds0 = lds_addr(s_tile);
  const int lrow = lane / L::kChunks, lpos = lane % L::kChunks;  // row within a load, LDS chunk position

  // A run is 8 rows of a tile, all in one page.  Sixteen steps at a time, lane
  // 4 s + i works out where run i of step s starts in the K pool and whether its
  // page is in range.  Runs past the last key take its run's place, runs without a
  // page that of page 0: rows that exist, of keys that count as not there.
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
      asm volatile("" : "+v"(at));
      const int entry = table_of(step, at);
      __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
      place_runs(step, entry, at);
      asm volatile("" : "+v"(run_lo), "+v"(run_hi));
    }
    Entries x;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int from = lane0 + i;
      x.at[i] = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(run_hi, from) << 32 |
                (uint32_t)__builtin_amdgcn_readlane(run_lo, from);
    }
    const uint32_t ok = (uint32_t)(run_ok >> lane0) & 15u;
    x.present = ((ok * 0x00204081u) & 0x01010101u) * 0xffu;  // each bit to a byte
    return x;
  };
  const uint32_t lane_k = lrow * L::kRowBytes + ((lpos ^ L::k(lrow)) << 4);
  const uint32_t lane_v = lrow * L::kRowBytes + ((lpos ^ L::v(lrow)) << 4);
  // Tile t into LDS at dst (K or V).  In the last tile, rows
  // past the last key read that key's row.
  auto load = [&](int t, const Entries& x, uint32_t dst, bool is_v) __attribute__((always_inline)) {
    auto move = [&](uint64_t at, uint32_t off, int in) __attribute__((always_inline)) {
      if (is_v) at += v_minus_k;
      const uint32_t to = __builtin_amdgcn_readfirstlane(dst + in * L::kRowBytes);
      if constexpr (kOnce) lds_dma16_nt((const void*)at, off, to);
      else lds_dma16((const void*)at, off, to);
    };
    if (t * kKeys + kKeys <= job.keys) {
#pragma unroll
      for (int i = 0; i < L::kLoads; ++i) {
        const int in = i * L::kRowsPerLoad;  // (a constant)
        const uint32_t swz = (is_v ? L::v(in) : L::k(in)) << 4;
        move(x.at[in / 8], ((is_v ? lane_v : lane_k) ^ swz) + (in & 7) * L::kRowBytes, in);
      }
    } else {
#pragma unroll
      for (int i = 0; i < L::kLoads; ++i) {
        const int in = i * L::kRowsPerLoad, row = in + lrow;
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

  // the keys of tile t that are there, as bits
  auto bits_of = [&](int t, uint32_t present) {
    const int lim = job.keys - t * kKeys;
    return lim < 32 ? present & ((1u << lim) - 1) : present;
  };
  // softmax of a tile's logits: st becomes the weights
  auto softmax = [&](const f32x16_t& st, uint32_t bits, float (&p)[16]) __attribute__((always_inline)) {
    float mt = neg_inf();
    if (bits != ~0u) {
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
    const bool grow = mt > m_run + kSlack;
    if (__builtin_amdgcn_ballot_w64(grow)) {  // (one branch for the wave)
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
  // Values of keys that are not there become 0 in LDS: 0 times what lies there may
  // be NaN.
  auto clear_missing = [&](uint32_t sv, uint32_t bits) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) u32x4_t* lds_ptr;
#pragma nounroll
    for (int i = 0; i < L::kLoads; ++i)
      if (!(bits >> (i * L::kRowsPerLoad + lrow) & 1)) *(lds_ptr)(uintptr_t)(sv + 1024 * i + 16 * lane) = u32x4_t{0, 0, 0, 0};
    wait_lds();
  };

  const uint32_t sk = lds0 + wave * 2 * L::kBytes, sv = sk + L::kBytes;
  if (t_first < t_end) {
    int t = t_first, step = 0;
    Entries x = entries(0);
    load(t, x, sk, false);
    load(t, x, sv, true);
    wait_vm<L::kLoads>();
    while (true) {
      const bool more = t + kStreams < t_end;
      const uint32_t bits = bits_of(t, x.present);
      const f32x16_t st = scores<T, D>(sk, q, lane);
      wait_lds();
      ++step;
      if (more) {
        x = entries(step);
        load(t + kStreams, x, sk, false);
      }
      float p[16];
      softmax(st, bits, p);
      if (more) wait_vm<L::kLoads>();
      else wait_vm<0>();
      if (bits != ~0u) clear_missing(sv, bits);
      add_values<T, D>(sv, p, o, lane);
      if (!more) break;
      wait_lds();
      t += kStreams;
      load(t, x, sv, true);
      wait_vm<L::kLoads>();
    }
  }
  if constexpr (!kAlone) __syncthreads();  // every wave is done with the tiles, and no load is in flight

  const float l_tot = partner_sum(l_run);
  if constexpr (kAlone) {
    if (r >= job.rows) return;
    const int64_t at = out_row(r) * parts + job.part;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int ig = 0; ig < 4; ++ig)
        *reinterpret_cast<f32x4_t*>(a.ws_o + at * D + 32 * db + 8 * ig + 4 * hg) =
            f32x4_t{o[db][4 * ig], o[db][4 * ig + 1], o[db][4 * ig + 2], o[db][4 * ig + 3]};
    if (hg == 0) {
      a.ws_ml[2 * at] = m_run;
      a.ws_ml[2 * at + 1] = l_tot;
    }
  } else {
    // the waves' rows through LDS: wave w's 32 x D sums at s_o + 32 w D, 16-byte
    // chunks swizzled by the row
    float* const s_o = reinterpret_cast<float*>(s_tile);
    constexpr int kO = D / 4;  // chunks of an output row
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
    __syncthreads();
    for (int it = tid; it < 32 * kO; it += kWaves * 64) {
      const int row = it / kO, ch = it % kO;
      if (job.row0 + row >= job.rows) continue;
      float M = neg_inf();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][row]);
      f32x4_t num = {0.f, 0.f, 0.f, 0.f};
      float den = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float ms = s_m[w][row];
        const float f = ms == neg_inf() ? 0.f : fast_exp2(ms - M);
        den += f * s_l[w][row];
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(s_o + (w * 32 + row) * D + ((ch ^ (row & (kO - 1))) << 2));
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] += f * x[e];
      }
      const int64_t at = out_row(job.row0 + row) * parts + job.part;
      *reinterpret_cast<f32x4_t*>(a.ws_o + at * D + 4 * ch) = num;
      if (ch == 0) {
        a.ws_ml[2 * at] = M;
        a.ws_ml[2 * at + 1] = den;
      }
    }
  }
}

// Members of group j: sequences [first, first + count).
__device__ __forceinline__ void members(const SharedArgs& a, int j, int& first, int& count) {
  first = min(max(a.group_start[j], 0), a.batch);
  count = min(max(min(a.group_start[j + 1], a.batch) - first, 0), a.max_group);
}

__device__ __forceinline__ int keys_of(const KeySource& src, int entry) {
  return (int)min((int64_t)min(max(src.len[entry], 0), src.max_len), (int64_t)src.pv.max_pages << src.pv.page_shift);
}

template <typename T, int D, bool kOnce>
__global__ __launch_bounds__(kWaves * 64, (sizeof(T) == 2 || D == 64 ? 2 : 1)) void shared_kernel(SharedArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char s_tile[kWaves * 2 * Tile<T, D>::kBytes];
  __shared__ float s_m[kWaves][32], s_l[kWaves][32];
  static_assert(sizeof(s_tile) >= kWaves * 32 * D * 4, "the waves' sums");
  Job job;
  if ((int)blockIdx.x < a.prefix_blocks) {
    int unit, row_tile, pair, split, j, first, count;
    // the row tiles of a unit read the same keys: they follow each other on one XCD
    // (block index mod 8) and its L2
    a.by_row_tiles.divide((int)(blockIdx.x >> 3), unit, row_tile);
    unit = unit * 8 + (int)(blockIdx.x & 7);
    if (unit >= a.prefix_units) return;
    a.by_prefix_splits.divide(unit, pair, split);
    a.by_heads.divide(pair, j, job.g);
    members(a, j, first, count);
    job.src = &a.prefix;
    job.entry = j;
    job.first_b = first;
    job.rows = count << a.group_shift;
    job.row0 = row_tile * kSharedRows;
    if (job.row0 >= job.rows) return;
    job.keys = keys_of(a.prefix, j);
    job.tile0 = split * a.prefix_tiles;
    job.tile1 = job.tile0 + a.prefix_tiles;
    job.part = split;
    attend<T, D, kOnce, false>(a, job, s_tile, s_m, s_l);
  } else {
    // a (sequence, KV head) and split a wave
    int pair, split, b;
    const int unit = ((int)blockIdx.x - a.prefix_blocks) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    a.by_own_splits.divide(unit, pair, split);
    a.by_heads.divide(pair, b, job.g);
    if (b >= a.batch) return;
    job.src = &a.own;
    job.entry = job.first_b = b;
    job.rows = 1 << a.group_shift;
    job.row0 = 0;
    job.keys = keys_of(a.own, b);
    job.tile0 = split * a.own_tiles;
    job.tile1 = job.tile0 + a.own_tiles;
    job.part = a.prefix_splits + split;
    attend<T, D, true, true>(a, job, s_tile, s_m, s_l);
  }
}

// Log-sum-exp merge of a row's partial results, the prefix's splits before the own
// ones: D / 4 lanes a row, four elements a lane.
constexpr int kMergeRows = 256;  // threads of a block
template <typename T, int D>
__global__ __launch_bounds__(kMergeRows) void shared_merge_kernel(SharedArgs a) {
  constexpr int kLanes = D / 4;
  const int e = threadIdx.x % kLanes;
  const int64_t row = (int64_t)blockIdx.x * (kMergeRows / kLanes) + threadIdx.x / kLanes;
  if (row >= (int64_t)a.batch * a.num_q_heads) return;
  const int b = (int)(row / a.num_q_heads), parts = a.prefix_splits + a.own_splits;
  // the last group that begins at b or before it, if b is one of its members
  int lo = 0, hi = a.groups;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.group_start[mid] <= b) lo = mid + 1;
    else hi = mid;
  }
  int first = 0, count = 0;
  if (lo > 0) members(a, lo - 1, first, count);
  const bool in_group = b >= first && b < first + count;

  const float2* ml = reinterpret_cast<const float2*>(a.ws_ml) + row * parts;
  const f32x4_t* po = reinterpret_cast<const f32x4_t*>(a.ws_o + row * parts * D) + e;
  constexpr int kAtOnce = 8;  // partial results whose loads are under way together
  float M = neg_inf(), den = 0.f;
  f32x4_t num = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = in_group ? 0 : a.prefix_splits; s0 < parts; s0 += kAtOnce) {
    float2 x[kAtOnce];
    f32x4_t v[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      x[k] = make_float2(neg_inf(), 0.f);
      if (s0 + k < parts) x[k] = ml[s0 + k];
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      v[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (x[k].x != neg_inf()) v[k] = po[(s0 + k) * kLanes];  // (nothing is written there else)
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
  // (the sum is 0 where nothing was seen: its logarithm is -inf)
  if (a.lse && e == 0) a.lse[row] = den == 0.f ? neg_inf() : M * 0.6931471805599453f + logf(den);
}

}  // namespace

template <typename T, int D>
hipError_t launch_shared_d(const SharedArgs& args, hipStream_t s) {
  SharedArgs a = args;
  const int heads = a.own.pv.kv_heads;
  a.by_row_tiles = FastDivide(a.row_tiles);
  a.by_prefix_splits = FastDivide(a.prefix_splits);
  a.by_own_splits = FastDivide(a.own_splits);
  a.by_heads = FastDivide(heads);
  a.prefix_units = a.groups * heads * a.prefix_splits;
  a.prefix_blocks = (a.prefix_units + 7) / 8 * 8 * a.row_tiles;
  const int64_t own_units = (int64_t)a.batch * heads * a.own_splits;
  const dim3 grid((uint32_t)(a.prefix_blocks + (own_units + kWaves - 1) / kWaves)), block(kWaves * 64);
  return a.row_tiles == 1 ? launch_struct(shared_kernel<T, D, true>, grid, block, s, a)
                          : launch_struct(shared_kernel<T, D, false>, grid, block, s, a);
}

hipError_t launch_shared(const SharedArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? launch_shared_d<bf16_bits, 128>(a, s) : launch_shared_d<bf16_bits, 64>(a, s);
  return head_dim == 128 ? launch_shared_d<float, 128>(a, s) : launch_shared_d<float, 64>(a, s);
}

template <typename T, int D>
hipError_t launch_merge_d(const SharedArgs& a, hipStream_t s) {
  const int per = kMergeRows / (D / 4);
  const dim3 grid((uint32_t)(((int64_t)a.batch * a.num_q_heads + per - 1) / per)), block(kMergeRows);
  return launch_struct(shared_merge_kernel<T, D>, grid, block, s, a);
}

hipError_t launch_shared_merge(const SharedArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? launch_merge_d<bf16_bits, 128>(a, s) : launch_merge_d<bf16_bits, 64>(a, s);
  return head_dim == 128 ? launch_merge_d<float, 128>(a, s) : launch_merge_d<float, 64>(a, s);
}

}  // namespace skv
