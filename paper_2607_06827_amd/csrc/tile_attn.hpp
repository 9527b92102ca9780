// Steps over a tile of 32 keys shared by the kernels that attend with 32 rows a
// wave: K or V rows in LDS (unpadded, 16-byte chunks XOR-swizzled so that operand
// reads are spread over the banks), S^T = K Q^T and O^T += V^T P^T on the 32x32
// matrix products, one row per lane column.
#pragma once

#include "attn_mfma.hpp"
#include "kernels_draft.hpp"

namespace skv {

// The running maximum may lag the true one by up to 2^kSlack before the sums are
// rescaled; the division by the weight sum makes the choice exact.
constexpr float kSlack = 8.f;
constexpr int kKeys = kTreeKeys;  // keys per tile
static_assert(kKeys == 32, "a tile's keys are the bits of a word and the rows of a 32x32 product");

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

}  // namespace skv
