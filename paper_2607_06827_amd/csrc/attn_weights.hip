// The attention weight that cache entries gather from queries: for entry c the sum
// of exp(scale q.k_c - lse) over the rows that see it, added to what it has.
//
// S^T = K Q^T on the 16x16 matrix products (operand A: 16 keys, B: 16 rows, the
// query heads of the group and queries), the weights straight from it, summed per
// key in a lane's own registers over the rows; the 16 lanes of a key add up once,
// at the end.  Keys and rows come through LDS by direct loads of whole rows:
// loaded straight into the operands, whose neighbouring lanes hold different rows,
// every 16 bytes are an access of their own (128 cycles an instruction of 64 lanes
// instead of 16; the prompts of 8 users 59 us).  16-byte chunks of a row are
// swizzled by the row so that operand reads are spread over the banks.
//
// Few rows (a decoding step): the rows stay in LDS and each wave streams keys of its
// own, 32 a step, one step ahead.  Bound by reading the keys: 16 sequences of 7660 keys
// of 8 heads take 46 us, 259 MB at 5.6 TB/s (reads alone reach 6.4); in fp32, one block
// a CU, 103 us, 510 MB at 5.0, and 4 of them 31, 4.1.
// Many rows (a prompt): a block holds 64 keys in its waves' registers, or two
// stretches of 64, the waves deal the row tiles out, each streaming those of its own,
// and add up through LDS.  8 prompts of 1596 tokens of 16 heads over 471 entries take
// 28 to 30 us, 400 TFLOP/s, with two stretches a block: the first and the last, the second
// and the last but one and so on, so that all blocks are alike and one round of them
// is enough (34 with one: two rounds that load their keys first, 8 us of them
// without the loop, and 210 MB of rows into LDS for 152).  Nothing splits the rows of a
// stretch: few (sequence, KV head)s leave CUs idle beside the blocks of the first keys,
// and one or two of these prompts take 24 us as well.  They are bound by what
// overlaps in part: the rows' way into LDS (a CU reads about 57 GB/s: 10 us), the
// products with their exponentials (16 us with nothing to wait for), the block's own
// keys and its sums (5).  With two stretches a wave adds one row tile at a time: two
// need more than 256 registers (60 us, as each key fragment read back from memory
// waits for all loads); row addresses are scalar for the same reason (30.8).  Four
// waves a block, all blocks at once, took 46 us: the first keys, which every row sees,
// set the time; six waves and two blocks a CU 38.
#include <algorithm>

#include "kernels_shared.hpp"
#include "tile_attn.hpp"

namespace skv {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;                  // few rows
constexpr int kManyWaves = 8, kManyThreads = 64 * kManyWaves;  // many rows
constexpr int kCus = 256;
constexpr int kSpreadUnits = 32;  // pairs from which an XCD takes pairs of its own

// Rows of 16-byte chunks in LDS: chunk c of row r at position c ^ swizzle(r).
template <typename T, int D>
struct Rows16 {
  static constexpr int kBytes = D * (int)sizeof(T);  // of a row
  static constexpr int kChunks = kBytes / 16;
  static constexpr int kPieces = kChunks / 4;         // 16-byte pieces of a row per lane
  static constexpr int kPerLoad = 64 / kChunks;       // rows of a direct load
  static constexpr int kTileLoads = 16 / kPerLoad;    // direct loads of 16 rows
  static constexpr int kTileBytes = 16 * kBytes;
  static __device__ __forceinline__ int swizzle(int row) { return kChunks == 8 ? (row >> 1) & 7 : row & 15; }
  // pieces of row `col` of the 16 rows at `lds`: chunks 4 p + quarter
  static __device__ __forceinline__ void read(u32x4_t (&x)[kPieces], uint32_t lds, int col, int quarter) {
    typedef __attribute__((address_space(3))) const u32x4_t* lds_ptr;
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
      x[p] = *(lds_ptr)(uintptr_t)(lds + col * kBytes + (((4 * p + quarter) ^ swizzle(col)) << 4));
  }
};

// 16 bytes per lane from the per-lane address p into LDS at lds + 16 * lane,
// untracked like lds_dma16; kOnce: without keeping the line in the caches.
template <bool kOnce>
__device__ __forceinline__ void lds_dma16_from(const void* p, uint32_t lds) {
  if constexpr (kOnce)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" : : "v"(p), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds) : "memory", "m0");
}

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

// v[j] summed over the 16 lanes of a row, for j = the lane's number in the row
// (mod the number of values).
template <int n>
__device__ __forceinline__ float transposed_sum(float (&v)[n], int lane) {
  auto step = [&](auto half, auto ctrl) __attribute__((always_inline)) {
    constexpr int m = decltype(half)::value;
    const bool up = lane & m;
#pragma unroll
    for (int k = 0; k < m; ++k) {
      if constexpr (m < n) {
        const float keep = up ? v[k + m] : v[k], send = up ? v[k] : v[k + m];
        v[k] = keep + dpp<decltype(ctrl)::value>(send);
      } else {
        v[k] += dpp<decltype(ctrl)::value>(v[k]);
      }
    }
  };
  static_assert(n == 8 || n == 16, "values of a lane");
  step(std::integral_constant<int, 8>(), std::integral_constant<int, kDppRowRor8>());
  step(std::integral_constant<int, 4>(), std::integral_constant<int, kDppHalfMirror>());
  step(std::integral_constant<int, 2>(), std::integral_constant<int, kDppQuadXor2>());
  step(std::integral_constant<int, 1>(), std::integral_constant<int, kDppQuadXor1>());
  return v[0];
}

// A block's (sequence, KV head) and its number among that pair's blocks.
struct Unit {
  int pair, part, b, g, len;
};
__device__ __forceinline__ bool unit_of(const WeightArgs& a, Unit& u) {
  const int heads = a.cache.pv.kv_heads, pairs = a.batch * heads;
  // The first keys of all pairs, which most rows of a prompt see, come first.  An
  // XCD (block index mod 8) takes neighbouring pairs: the KV heads of a sequence,
  // whose rows lie beside each other.
  if (pairs >= kSpreadUnits) {
    a.by_pairs.divide((int)(blockIdx.x >> 3), u.part, u.pair);
    u.pair += (int)(blockIdx.x & 7) * a.by_pairs.d;
    if (u.pair >= pairs) return false;
  } else {
    a.by_pairs.divide((int)blockIdx.x, u.part, u.pair);
  }
  a.by_heads.divide(u.pair, u.b, u.g);
  const PagedView& pv = a.cache.pv;
  u.len = (int)min((int64_t)min(max(a.cache.len[u.b], 0), a.cache.max_len), (int64_t)pv.max_pages << pv.page_shift);
  return true;
}

// Direct loads of 16 n keys from key kb on into LDS at `to`, by one wave (which
// takes every `share`-th load); keys behind the last read the last, keys without a
// page rows of page 0.  `entry`: lane lane0 + i has the block-table entry of the
// 2^kRun keys from kb + 2^kRun i on (or of the last).
template <typename T, int D, int kTiles, int kRun, bool kOnce>
__device__ __forceinline__ void load_keys(const WeightArgs& a, const Unit& u, int kb, int entry, int lane0, uint32_t to,
                                          int lane, int first, int share) {
  typedef Rows16<T, D> L;
  const PagedView& pv = a.cache.pv;
  const int lrow = lane / L::kChunks, lpos = lane % L::kChunks;
#pragma unroll
  for (int n = 0; n < kTiles * L::kTileLoads; ++n) {
    if (share > 1 && n % share != first) continue;
    const int row = n * L::kPerLoad + lrow, key = min(kb + row, u.len - 1);
    const int e = __shfl(entry, lane0 + ((key - kb) >> kRun), 64);
    const int64_t page = e >= 0 && e < pv.num_pages ? e : 0;
    const char* from = static_cast<const char*>(a.cache.k_pages) +
                       page_row<D>(page, u.g, key & ((1 << pv.page_shift) - 1), pv) * (int)sizeof(T) +
                       ((lpos ^ L::swizzle(row)) << 4);
    lds_dma16_from<kOnce>(from, __builtin_amdgcn_readfirstlane(to + n * 1024));
  }
}

// Address of row r (0 .. 15) of row tile rt, query head r % G of the tile's query
// r / G; rows behind the last read query 0.
template <typename T>
__device__ __forceinline__ const char* row_of(const WeightArgs& a, const Unit& u, int rt, int r) {
  const int i = rt * (16 >> a.group_shift) + (r >> a.group_shift);
  const int h = (u.g << a.group_shift) + (r & ((1 << a.group_shift) - 1));
  return reinterpret_cast<const char*>(static_cast<const T*>(a.q.p) + u.b * a.q.sb + (i < a.num_rows ? i : 0) * a.q.ss +
                                       h * a.q.sh);
}

// Direct loads of row tile rt into LDS at `to`, by one wave.  (One after the other: the
// last tile takes this way, and four loads' addresses would take the registers of
// keys.)
template <typename T, int D>
__device__ __forceinline__ void load_rows(const WeightArgs& a, const Unit& u, int rt, uint32_t to, int lane) {
  typedef Rows16<T, D> L;
  const int lrow = lane / L::kChunks, lpos = lane % L::kChunks;
#pragma nounroll
  for (int n = 0; n < L::kTileLoads; ++n) {
    const int row = n * L::kPerLoad + lrow;
    lds_dma16_from<false>(row_of<T>(a, u, rt, row) + ((lpos ^ L::swizzle(row)) << 4),
                          __builtin_amdgcn_readfirstlane(to + n * 1024));
  }
}

// Where this lane's row of tile rt has its lse and its number of seen entries.
__device__ __forceinline__ const float* lse_of(const WeightArgs& a, const Unit& u, int rt, int col) {
  const int i = rt * (16 >> a.group_shift) + (col >> a.group_shift);
  const int h = (u.g << a.group_shift) + (col & ((1 << a.group_shift) - 1));
  return a.lse + u.b * a.lse_b + h * a.lse_h + (i < a.num_rows ? i : 0) * a.lse_s;
}
__device__ __forceinline__ const int32_t* seen_at(const WeightArgs& a, const Unit& u, int i) {
  // (without a list the length: a load that no branch depends on)
  return a.visible ? a.visible + (int64_t)u.b * a.num_rows + (i < a.num_rows ? i : 0) : a.cache.len + u.b;
}
// What query i sees, of what the list says.
__device__ __forceinline__ int seen_of(const WeightArgs& a, const Unit& u, int n, int i) {
  if (!a.visible) n = u.len - (a.num_rows - 1 - i);
  return i < a.num_rows ? min(max(n, 0), u.len) : 0;
}

// What a lane needs of its row of a tile: the pieces, the lse, the entries it sees.
template <typename T, int D>
struct Row {
  u32x4_t x[Rows16<T, D>::kPieces];
  float l;  // in powers of 2
  int seen;
  __device__ __forceinline__ void set(float lse, int n) {
    l = lse * 1.4426950408889634f;
    seen = l == neg_inf() ? 0 : n;  // (a row that saw nothing)
  }
};

// Adds the weights that the rows of n tiles give the keys k (16 a tile, from key kb
// on): sum element 4 t + e is of key 16 t + 4 quarter + e, over this lane's rows.
template <typename T, int D, int kTiles, int n>
__device__ __forceinline__ void add_rows(const WeightArgs& a, const u32x4_t (&k)[kTiles][Rows16<T, D>::kPieces],
                                         const Row<T, D> (&y)[n], int kb, int quarter, float (&sum)[4 * kTiles]) {
  f32x4_t st[n][kTiles];
#pragma unroll
  for (int m = 0; m < n; ++m)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) st[m][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // (the sums in turn: a product waits for the one before it of its sum)
#pragma unroll
  for (int p = 0; p < Rows16<T, D>::kPieces; ++p)
#pragma unroll
    for (int m = 0; m < n; ++m)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) st[m][t] = product<T>(k[t][p], y[m].x[p], st[m][t]);
  int least = y[0].seen;
#pragma unroll
  for (int m = 1; m < n; ++m) least = min(least, y[m].seen);
  if (!__builtin_amdgcn_ballot_w64(least < kb + 16 * kTiles)) {  // every row sees all keys
#pragma unroll
    for (int m = 0; m < n; ++m)
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[4 * t + e] += fast_exp2(__builtin_fmaf(st[m][t][e], a.scale_log2, -y[m].l));
  } else {
#pragma unroll
    for (int m = 0; m < n; ++m) {
      const int most = y[m].seen - kb - 4 * quarter;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = fast_exp2(__builtin_fmaf(st[m][t][e], a.scale_log2, -y[m].l));
          sum[4 * t + e] += 16 * t + e < most ? w : 0.f;
        }
    }
  }
}

// Key (of 16 kTiles) whose total transposed_sum leaves in this lane.
template <int kTiles>
__device__ __forceinline__ int key_of(int col, int quarter) {
  return 16 * ((col >> 2) & (kTiles - 1)) + 4 * quarter + (col & 3);
}

// ---------------------------------------------------------------- few rows

// Blocks that run at once on a CU: fp32 rows of 128 elements take 152 KB of LDS a block.
constexpr int few_blocks(int row_bytes) { return row_bytes > 256 ? 1 : 2; }

template <typename T, int D>
__global__ __launch_bounds__(kThreads, few_blocks(Rows16<T, D>::kBytes)) void weights_few_kernel(WeightArgs a) {
  typedef Rows16<T, D> L;
  constexpr int kTiles = kWeightStep / 16, kStepBytes = kTiles * L::kTileBytes, kN = kTiles * L::kTileLoads;
  __shared__ __attribute__((aligned(1024))) unsigned char s_q[kWeightFew * L::kTileBytes];
  __shared__ __attribute__((aligned(1024))) unsigned char s_k[kWaves][2][kStepBytes];
  __shared__ float s_sum[kWaves * kWeightSteps * kWeightStep];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  Unit u;
  if (!unit_of(a, u)) return;
  // a block has a stretch of keys, its waves steps of 32 of it in turn
  const int block_keys = kWaves * a.steps * kWeightStep, k0 = u.part * block_keys;
  if (k0 >= u.len) return;
  const int steps = min(a.steps, max((u.len - k0 + kWeightStep - 1) / kWeightStep - wave + kWaves - 1, 0) / kWaves);
  auto key0 = [&](int step) { return k0 + (step * kWaves + wave) * kWeightStep; };
  const int32_t* table = a.cache.table + (int64_t)u.b * a.cache.pv.max_pages;
  // lane 4 s + i has the table entry of keys 8 i .. of step s (pages hold at least 8)
  static_assert(kWeightSteps * kWeightStep / 8 <= 64 && kWeightStep == 32, "a lane for every 8 keys");
  int entry = table[min(key0(lane >> 2) + 8 * (lane & 3), u.len - 1) >> a.cache.pv.page_shift];
  // the rows' lse and what they see; all of it has arrived before the first direct
  // load of a key, which the compiler does not count
  float l[kWeightFew];
  int seen[kWeightFew];
#pragma unroll
  for (int rt = 0; rt < kWeightFew; ++rt) {
    const int i = rt * (16 >> a.group_shift) + (col >> a.group_shift);
    l[rt] = *lse_of(a, u, rt, col);
    seen[rt] = seen_of(a, u, *seen_at(a, u, i), i);
  }
  const uint32_t sq = lds_addr(s_q), sk = lds_addr(s_k[wave]);
  for (int rt = wave; rt < a.row_tiles; rt += kWaves) load_rows<T, D>(a, u, rt, sq + rt * L::kTileBytes, lane);
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
#pragma unroll
  for (int rt = 0; rt < kWeightFew; ++rt) asm volatile("" : "+v"(l[rt]), "+v"(seen[rt]));
  asm volatile("" : "+v"(entry));
  __builtin_amdgcn_sched_barrier(0);
  __syncthreads();  // the rows are in LDS

  const uint64_t pages = __builtin_amdgcn_ballot_w64(entry >= 0 && entry < a.cache.pv.num_pages);
  // (always: what waits for the others counts on it; behind the last step the keys
  // of the last one again)
  auto request = [&](int step) __attribute__((always_inline)) {
    const int s = min(step, max(steps - 1, 0));
    load_keys<T, D, kTiles, 3, true>(a, u, key0(s), entry, 4 * s, sk + (step & 1) * kStepBytes, lane, 0, 1);
  };
  request(0);
  request(1);
  for (int step = 0; step < steps; ++step) {
    const int kb = key0(step);
    const uint32_t ok = ((((uint32_t)(pages >> (4 * step)) & 15u) * 0x00204081u) & 0x01010101u) * 0xffu;  // a byte each
    wait_vm<kN>();
    u32x4_t k[kTiles][L::kPieces];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) L::read(k[t], sk + (step & 1) * kStepBytes + t * L::kTileBytes, col, quarter);
    wait_lds();
    request(step + 2);
    float sum[4 * kTiles];
#pragma unroll
    for (int j = 0; j < 4 * kTiles; ++j) sum[j] = 0.f;
#pragma unroll
    for (int rt = 0; rt < kWeightFew; ++rt)
      if (rt < a.row_tiles) {
        Row<T, D> y[1];
        L::read(y[0].x, sq + rt * L::kTileBytes, col, quarter);
        y[0].set(l[rt], seen[rt]);
        add_rows<T, D, kTiles>(a, k, y, kb, quarter, sum);
      }
    const float total = transposed_sum(sum, lane);
    const int at = key_of<kTiles>(col, quarter);
    s_sum[(step * kWaves + wave) * kWeightStep + at] = ok >> at & 1 ? total : 0.f;
  }
  wait_vm<0>();
  __syncthreads();
  const int64_t row = (int64_t)u.pair * a.capacity + k0;
  for (int c = tid; c < min(block_keys, u.len - k0); c += kThreads)
    a.weights_out[row + c] = (a.weights ? a.weights[row + c] : 0.f) + s_sum[c];
}

// --------------------------------------------------------------- many rows

// kStretches: stretches of kKeys keys that a block holds, 1 or 2.  With two, block p has
// stretch p and, of n, stretch n - 1 - p: in a prompt, where later keys have fewer
// rows, all blocks have as many products, and the rows of the later are among those of
// the earlier.
template <typename T, int D, int kStretches>
__global__ __launch_bounds__(kManyThreads) void weights_many_kernel(WeightArgs a) {
  typedef Rows16<T, D> L;
  constexpr int kKeys = weight_keys(L::kBytes), kTiles = kKeys / 16;
  constexpr int kAhead = L::kBytes > 256 ? 2 : 4;  // row tiles of a wave on their way
  constexpr int kOnce = kStretches == 2 ? 1 : kAhead / 2;  // row tiles added at once
  constexpr int kN = L::kTileLoads + 1;            // direct loads of a row tile
  __shared__ __attribute__((aligned(1024))) unsigned char s_row[kManyWaves][kAhead][L::kTileBytes];
  __shared__ int s_info[kManyWaves][kAhead][64];  // lanes 0 .. 31: the rows' lse, 32 .. 63: what they see
  __shared__ float s_part[kManyWaves][kStretches * kKeys];
  __shared__ uint64_t s_sees[kManyWaves];
  static_assert(sizeof(s_row) >= kStretches * kTiles * L::kTileBytes, "the keys come through the rows' place");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  Unit u;
  if (!unit_of(a, u)) return;
  const int kb = u.part * kKeys;  // first key of the first stretch
  int kb2 = kb;                   // and of the second, the same if there is none
  if constexpr (kStretches == 2) kb2 = ((u.len + kKeys - 1) / kKeys - 1 - u.part) * kKeys;
  if (kb >= u.len || kb2 < kb) return;

  float sum[kStretches][4 * kTiles];
#pragma unroll
  for (int c = 0; c < kStretches; ++c)
#pragma unroll
    for (int j = 0; j < 4 * kTiles; ++j) sum[c][j] = 0.f;
  const int queries = 16 >> a.group_shift, in = col >> a.group_shift;

  // kManyWaves * 64 row tiles at a time, 64 a wave: lane n finds out whether any row
  // of tile n sees these keys.  Every wave then goes through those tiles of its own
  // (one in kManyWaves) that do, kAhead of them requested ahead.  From the last row to
  // the first: in a prompt the last rows see most, so the blocks of a sequence read
  // the same rows at the same time, out of one L2.
  auto scan = [&](int rt0) {
    int most = 0;
#pragma unroll 8
    for (int n = 0; n < queries; ++n) {
      const int i = (rt0 + 64 * wave + lane) * queries + n;
      most = max(most, seen_of(a, u, *seen_at(a, u, i), i));
    }
    return __builtin_amdgcn_ballot_w64(most > kb);
  };
  int rt0 = (a.row_tiles - 1) / (64 * kManyWaves) * (64 * kManyWaves);
  const int rt0_first = rt0;
  uint64_t sees;

  u32x4_t k[kStretches][kTiles][L::kPieces];
  uint64_t present[kStretches];  // keys that have a page
  {
    const int32_t* table = a.cache.table + (int64_t)u.b * a.cache.pv.max_pages;
    int entry[kStretches];
#pragma unroll
    for (int c = 0; c < kStretches; ++c)
      entry[c] = table[min((c ? kb2 : kb) + lane, u.len - 1) >> a.cache.pv.page_shift];
    const uint32_t sk = lds_addr(s_row);
#pragma unroll
    for (int c = 0; c < kStretches; ++c) {
      present[c] = __builtin_amdgcn_ballot_w64(entry[c] >= 0 && entry[c] < a.cache.pv.num_pages);
      load_keys<T, D, kTiles, 0, false>(a, u, c ? kb2 : kb, entry[c], 0, sk + c * kTiles * L::kTileBytes, lane, wave,
                                        kManyWaves);
    }
    sees = scan(rt0);  // (on its way with the keys)
    wait_vm<0>();
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kStretches; ++c)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) L::read(k[c][t], sk + (c * kTiles + t) * L::kTileBytes, col, quarter);
    wait_lds();
    __syncthreads();  // the keys are in registers: rows take their place
  }

  const uint32_t s_rows = lds_addr(s_row[wave]), s_infos = lds_addr(s_info[wave]);
  // A lane reads chunk `lpos` (swizzled) of row `lrow` of each load.  Rows r = n
  // kPerLoad + lrow of a tile have no carry between the two, neither in their query
  // nor in their head: the first gives a scalar base, the second this lane's offset
  // (where 32 bits hold it).
  const int lrow = lane / L::kChunks, gmask = (1 << a.group_shift) - 1;
  const int64_t lane_at = ((lrow >> a.group_shift) * a.q.ss + (lrow & gmask) * a.q.sh) * (int)sizeof(T);
  const bool near = !__builtin_amdgcn_ballot_w64(lane_at > INT32_MAX);
  const uint32_t lane_off = (uint32_t)lane_at, lane_chunk = (lane % L::kChunks ^ L::swizzle(lrow)) << 4;
  const int64_t row_step = queries * a.q.ss * (int)sizeof(T);
  auto request = [&](int rt, int buffer) __attribute__((always_inline)) {
    if (near && (rt + 1) * queries <= a.num_rows) {
#pragma unroll
      for (int n = 0; n < L::kTileLoads; ++n) {
        const int row = n * L::kPerLoad;  // (a constant)
        const char* base = row_of<T>(a, u, 0, row) + rt * row_step;
        lds_dma16(base, lane_off + (lane_chunk ^ (L::swizzle(row) << 4)),
                  __builtin_amdgcn_readfirstlane(s_rows + buffer * L::kTileBytes + n * 1024));
      }
    } else {
      load_rows<T, D>(a, u, rt, s_rows + buffer * L::kTileBytes, lane);
    }
    lds_dma4(lane < 32 ? static_cast<const void*>(lse_of(a, u, rt, col)) : seen_at(a, u, rt * queries + in),
             __builtin_amdgcn_readfirstlane(s_infos + buffer * 256));
  };

  static_assert(kManyWaves == 8, "tiles of a wave");
  const uint64_t mine = 0x0101010101010101ull << wave;  // bits of the tiles that are this wave's
  for (bool more = true; more; more = (rt0 -= 64 * kManyWaves) >= 0) {
    if (rt0 != rt0_first) sees = scan(rt0);
    __syncthreads();  // (the last masks have been read)
    if (lane == 0) s_sees[wave] = sees;
    __syncthreads();
    int count = 0, word = kManyWaves;
#pragma unroll
    for (int w = 0; w < kManyWaves; ++w) count += __builtin_popcountll(s_sees[w] & mine);
    count = __builtin_amdgcn_readfirstlane(count);
    if (!count) continue;
    uint64_t todo = 0;
    int last = rt0;
    auto next = [&]() {  // the wave's next tile, the last one again behind it
      while (!todo && word > 0) {
        --word;
        const uint64_t x = s_sees[word] & mine;
        todo = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 |
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x);
      }
      if (todo) {
        const int bit = 63 - __builtin_clzll(todo);
        todo ^= (uint64_t)1 << bit;
        last = rt0 + 64 * word + bit;
      }
      return __builtin_amdgcn_readfirstlane(last);
    };
    int tile[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) request(tile[j] = next(), j);
    for (int at = 0; at < count; at += kAhead) {
#pragma unroll
      for (int j = 0; j < kAhead; j += kOnce) {
        wait_vm<(kAhead - kOnce) * kN>();
        Row<T, D> y[kOnce];
#pragma unroll
        for (int m = 0; m < kOnce; ++m) {
          L::read(y[m].x, s_rows + (j + m) * L::kTileBytes, col, quarter);
          const int n = seen_of(a, u, s_info[wave][j + m][32 + col], tile[j + m] * queries + in);
          y[m].set(__int_as_float(s_info[wave][j + m][col]), at + j + m < count ? n : 0);
        }
        wait_lds();
#pragma unroll
        for (int m = 0; m < kOnce; ++m) request(tile[j + m] = next(), j + m);  // (always: what waits counts on it)
        if (at + j < count) {
          add_rows<T, D, kTiles>(a, k[0], y, kb, quarter, sum[0]);
          if constexpr (kStretches == 2) {
            int most = y[0].seen;
#pragma unroll
            for (int m = 1; m < kOnce; ++m) most = max(most, y[m].seen);
            if (__builtin_amdgcn_ballot_w64(most > kb2)) add_rows<T, D, kTiles>(a, k[1], y, kb2, quarter, sum[1]);
          }
        }
      }
    }
    wait_vm<0>();
  }
#pragma unroll
  for (int c = 0; c < kStretches; ++c)
    s_part[wave][c * kKeys + key_of<kTiles>(col, quarter)] = transposed_sum(sum[c], lane);
  __syncthreads();
#pragma unroll
  for (int c = 0; c < kStretches; ++c) {
    if (c && kb2 == kb) break;
    const int key = (c ? kb2 : kb) + tid;
    if (tid < kKeys && key < u.len) {
      float total = 0.f;
#pragma unroll
      for (int v = 0; v < kManyWaves; ++v) total += s_part[v][c * kKeys + tid];
      const int64_t to = (int64_t)u.pair * a.capacity + key;
      a.weights_out[to] = (a.weights ? a.weights[to] : 0.f) + (present[c] >> tid & 1 ? total : 0.f);
    }
  }
}

}  // namespace

template <typename T, int D>
hipError_t launch_weights_d(const WeightArgs& args, hipStream_t s) {
  WeightArgs a = args;
  a.by_heads = FastDivide(a.cache.pv.kv_heads);
  const int64_t pairs = (int64_t)a.batch * a.cache.pv.kv_heads;
  const bool spread = pairs >= kSpreadUnits;
  a.by_pairs = FastDivide((int32_t)(spread ? (pairs + 7) / 8 : pairs));  // (of an XCD)
  const dim3 grid((uint32_t)((spread ? (pairs + 7) / 8 * 8 : pairs) * a.key_blocks));
  if (a.row_tiles <= kWeightFew) return launch_struct(weights_few_kernel<T, D>, grid, dim3(kThreads), s, a);
  return a.stretches == 2 ? launch_struct(weights_many_kernel<T, D, 2>, grid, dim3(kManyThreads), s, a)
                          : launch_struct(weights_many_kernel<T, D, 1>, grid, dim3(kManyThreads), s, a);
}

hipError_t launch_weights(const WeightArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? launch_weights_d<bf16_bits, 128>(a, s) : launch_weights_d<bf16_bits, 64>(a, s);
  return head_dim == 128 ? launch_weights_d<float, 128>(a, s) : launch_weights_d<float, 64>(a, s);
}

// Many rows: one or two stretches of keys a block, what an estimate says is faster.
// A CU holds one block at a time, which takes 5 us and 0.105 for a row tile and
// stretch (128-wide bf16 heads; 0.07 with 64-wide ones, 0.37 in fp32).  As many rows
// see a stretch as in a prompt: single ones, the largest first, end together but for
// half of the last, pairs are all alike.  (Measured: 8 sequences of 471 entries, 1596
// rows, 33.6 us with one and 28.9 with two; of 300 entries, where pairs are 192 blocks,
// 25.2 and 29.9.  Of 25 shapes the choice is the faster form or within 5% of it.)
static int stretches_of(int64_t pairs, int64_t all, int row_tiles, int dim, int elt_size) {
  const double block = 5.0, rows = row_tiles * (elt_size == 4 ? 0.37 : dim == 128 ? 0.105 : 0.07);
  const double n = (double)pairs * all, tail = n > kCus ? 0.5 * (block + rows / all) : 0.0;
  const double one = std::max(block + rows, (n * block + rows * pairs * (all + 1) / 2) / kCus + tail);
  const double rounds = (double)((pairs * ((all + 1) / 2) + kCus - 1) / kCus);
  return rounds * (1.1 * block + rows * (1.0 + 1.0 / all)) < one ? 2 : 1;
}

// Few rows: steps of a wave that spread the keys over the blocks that run at once, so
// that they end together.  (Cut for two blocks a CU where one fits, 4 sequences of 7660
// keys of 8 heads in fp32 took 36 us for 30 and one took 17 for 13.)  Where that is more
// steps than a wave has, one block a CU goes in whole rounds (9 of them 62 us, 77 with 16
// steps a wave); two a CU overlap, and whole rounds are as often slower (20 sequences of
// 64-wide bf16 keys 28 us with 16 steps and 33 in rounds, 34 of 4000 128-wide ones 63
// and 58).
void plan_weights(WeightArgs& a, int dim, int elt_size) {
  const int row_bytes = dim * elt_size;
  const int64_t pairs = (int64_t)a.batch * a.cache.pv.kv_heads;
  if (a.row_tiles > kWeightFew) {
    const int64_t all = ((int64_t)a.cache.max_len + weight_keys(row_bytes) - 1) / weight_keys(row_bytes);
    a.steps = 1;
    a.stretches = all > 1 ? stretches_of(pairs, all, a.row_tiles, dim, elt_size) : 1;
    a.key_blocks = (int)((all + a.stretches - 1) / a.stretches);
    return;
  }
  const int64_t tiles = ((int64_t)a.cache.max_len + kWeightStep - 1) / kWeightStep;
  const int64_t waves = (int64_t)kCus * few_blocks(row_bytes) * kWaves, all = pairs * tiles;
  const int64_t rounds =
      few_blocks(row_bytes) > 1 ? 1 : std::max<int64_t>(1, (all + waves * kWeightSteps - 1) / (waves * kWeightSteps));
  a.steps = (int)std::max<int64_t>(1, std::min<int64_t>((all + waves * rounds - 1) / (waves * rounds), kWeightSteps));
  a.key_blocks = (int)((tiles + kWaves * a.steps - 1) / (kWaves * a.steps));
}

}  // namespace skv
