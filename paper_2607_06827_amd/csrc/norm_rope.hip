// Norms of queries and keys for each head with the rotation by position, and
// their gradients.
//
// A row x of a head becomes y = R (gamma o r x), r = (mean x^2 + eps)^-1/2, R the
// rotation of its element pairs by a_j = position * inv_freq[j].  The gradient
// turns back first: g = R^-1 dy, h = gamma o g, dgamma = sum g o r x,
// dx = r (h - r x mean(h o r x)); r is computed again, as x is read for dx anyway.
//
// A thread holds 16 elements of a row, two 8-element chunks: the two whose
// elements turn together, or two of the elements that stay.  D / 16 neighbouring
// lanes hold a row and add their sums with lane exchanges.  A wave takes the
// queries (or the keys, or the values) of some tokens and needs no other wave:
// its lanes work out an angle each, whose sine and cosine the rows share through
// LDS.  Angles are counted in turns, whose whole part drops out in 64 bits, so that
// far positions lose nothing.
//
// Sums, norms, the rotation and gradients are fp32; each output is rounded once.
//
// Bound by HBM: the prompts of 8 users (12768 tokens of 16 + 8 heads, bf16) take 33 us
// forward, 157 MB at 4.8 TB/s, and 51.5 backward, 235 MB at 4.6 (a large copy reaches
// 5.1); the counters give the bytes of the rows, no more.  What small calls wait for is
// the chain of loads: row counts, rows, and backward the sums' second launch.  With a
// block of 256 threads a token and two barriers for its angles the backward took 142
// us; with more tokens a step both take 1 to 3 us longer, and non-temporal stores,
// unrolled rows or fewer registers change nothing.
#include <algorithm>

#include "kernels_norm.hpp"

namespace skv {

namespace {

constexpr int kThreads = 256;

// Rows are read once.  (An fp32 chunk takes two loads of the same lines, which
// costs more non-temporally than it saves.)
__device__ __forceinline__ void load_row(Chunk<bf16_bits>& c, const bf16_bits* p) {
  const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  c.raw = make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void load_row(Chunk<float>& c, const float* p) { c.load(p); }

// Sum over the D / 16 lanes of a row (the same in each).
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<kDppQuadXor1>(x);
  x += dpp<kDppQuadXor2>(x);
  if (D == 128) x += dpp<kDppHalfMirror>(x);
  return x;
}

// Which elements a lane holds: 8 c0 .. and 8 c1 .. of a row.
struct Place {
  int p, c0, c1;
  bool turns;
  template <typename A>
  __device__ __forceinline__ Place(int lane, const A& a) : p(lane), turns(lane < a.rot / 16) {
    const bool halves = turns && !a.pairs;
    c0 = halves ? p : 2 * p;
    c1 = halves ? p + a.rot / 16 : 2 * p + 1;
  }
};

// The pairs of a lane's 16 elements (u: its first chunk, w: its second) turn by
// the angles whose (cos, sin) are at t; kBack: the other way.
template <bool kBack>
__device__ __forceinline__ void turn(float (&u)[8], float (&w)[8], const float2* t, bool pairs) {
  if (pairs) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float& x = j < 4 ? u[2 * j] : w[2 * j - 8];
      float& y = j < 4 ? u[2 * j + 1] : w[2 * j - 7];
      const float c = t[j].x, s = kBack ? -t[j].y : t[j].y, z = x;
      x = z * c - y * s;
      y = z * s + y * c;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float c = t[j].x, s = kBack ? -t[j].y : t[j].y, z = u[j];
      u[j] = z * c - w[j] * s;
      w[j] = z * s + w[j] * c;
    }
  }
}

// LDS that a wave writes before its own lanes read it.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's tokens: where the rows of head 0 start in up to three tensors, in
// elements, and their (cos, sin), D / 2 apart.
template <int D>
struct Step {
  float2 turn[kNormTokens * (D / 2)];
  int64_t at[3][kNormTokens];
  int there[kNormTokens];
};

// Fills the step of tokens first .. first + n: f(token, b, i) gives the three
// places and whether the token is there.
template <int D, typename F>
__device__ __forceinline__ void fill_step(const NormArgs& a, int first, int n, bool turns, int lane, Step<D>& s, F f) {
  wave_fence();  // (the last step's have been read)
  if (lane < n) {
    const int t = first + lane;
    int b, i;
    a.by_rows.divide(min(t, a.tokens - 1), b, i);
    const int rows = a.row_len ? a.row_len[b] : a.num_rows;
    int64_t at[3] = {0, 0, 0};
    s.there[lane] = f(t, b, i, t < a.tokens && i < rows, at);
#pragma unroll
    for (int x = 0; x < 3; ++x) s.at[x][lane] = at[x];
  }
  if (turns) {
    const int j = lane % (D / 2);
    const bool used = j < a.rot / 2;
    const double inv = used ? (double)a.inv_freq[j] * 0.15915494309189535 : 0.0;
    const int axis = used && a.axis ? min(max(a.axis[j], 0), a.num_axes - 1) : 0;
    for (int in = lane / (D / 2); in < n; in += 64 / (D / 2)) {
      const int t = min(first + in, a.tokens - 1);
      const double x = (double)a.positions[(int64_t)axis * a.tokens + t] * inv;
      float sn, cs;
      sincospif(2.f * (float)(x - __builtin_rint(x)), &sn, &cs);
      s.turn[in * (D / 2) + j] = make_float2(cs, sn);
    }
  }
  wave_fence();
}

__device__ __forceinline__ int64_t offset_of(const HeadRows& x, int b, int i) { return b * x.sb + i * x.ss; }

__device__ __forceinline__ void load_gamma(float (&x)[8], float (&y)[8], const float* gamma, const Place& at) {
  Chunk<float> c, d;
  c.a = c.b = d.a = d.b = make_float4(1.f, 1.f, 1.f, 1.f);
  if (gamma) {
    c.load(gamma + 8 * at.c0);
    d.load(gamma + 8 * at.c1);
  }
  c.to_float(x);
  d.to_float(y);
}

template <int D>
__device__ __forceinline__ float inverse_size(const float (&u)[8], const float (&w)[8], float eps) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += u[e] * u[e];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += w[e] * w[e];
  return 1.f / sqrtf(row_sum<D>(sum) * (1.f / D) + eps);
}

// Which kind of rows a block has, and its number among those blocks.
__device__ __forceinline__ int kind_of(const NormArgs& a, int& block) {
  block = blockIdx.x;
  for (int kind = 0; kind < 2; ++kind) {
    if (block < a.part[kind].blocks) return kind;
    block -= a.part[kind].blocks;
  }
  return 2;
}

// kAppend: keys and values go behind the cache's entries.
template <typename T, int D, bool kAppend>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  constexpr int kLanes = D / 16, kGroups = 64 / kLanes;  // lanes of a row, rows of a wave
  __shared__ Step<D> s_step[kThreads / 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int block;
  const int kind = kind_of(a, block);
  const NormPart& part = a.part[kind];
  const int id = block * (kThreads / 64) + wave, step = id / part.split, share = id % part.split;
  if (step >= part.steps) return;
  const Place at(lane % kLanes, a);
  const bool turning = a.rot && kind < 2;
  Step<D>& s = s_step[wave];
  const HeadRows& src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
  const bool paged = kAppend && kind > 0;
  fill_step<D>(a, step * part.tokens, part.tokens, turning, lane, s, [&](int, int b, int i, bool there, int64_t (&to)[3]) {
    to[0] = offset_of(src, b, i);
    if (!paged) {
      to[1] = offset_of(kind ? a.k_out : a.q_out, b, i);
      return there;
    }
    const int len = max(a.cache_len[b], 0);
    if (kind == 1 && i == 0 && a.cache_len_out) {
      const int n = a.row_len ? min(max(a.row_len[b], 0), a.num_rows) : a.num_rows;
      a.cache_len_out[b] = (int32_t)min((int64_t)len + n, (int64_t)INT32_MAX);
    }
    const int64_t slot = (int64_t)len + i, index = slot >> a.pv.page_shift;
    if (!there || index >= a.pv.max_pages) return false;
    const int64_t page = a.table[(int64_t)b * a.pv.max_pages + index];
    to[1] = page_row<D>(page, 0, (int)(slot & ((1 << a.pv.page_shift) - 1)), a.pv);
    return page >= 0 && page < a.pv.num_pages;
  });
  T* const out = static_cast<T*>(paged ? (kind == 1 ? a.k_pages : a.v_pages) : kind ? a.k_out.p : a.q_out.p);
  const int64_t out_head = paged ? (int64_t)D << a.pv.page_shift : kind ? a.k_out.sh : a.q_out.sh;
  const bool normed = a.normalise && kind < 2, turns = turning && at.turns;
  const float* gamma = kind ? a.gamma_k : a.gamma_q;
  for (int r = lane / kLanes + kGroups * share; r < part.tokens * part.heads; r += kGroups * part.split) {
    int in, h;
    part.by_heads.divide(r, in, h);
    if (!s.there[in]) continue;
    const T* from = static_cast<const T*>(src.p) + s.at[0][in] + h * src.sh;
    T* dst = out + s.at[1][in] + h * out_head;
    Chunk<T> x, y;
    load_row(x, from + 8 * at.c0);
    load_row(y, from + 8 * at.c1);
    if (normed || turns) {
      float u[8], w[8];
      x.to_float(u);
      y.to_float(w);
      if (normed) {
        const float size = inverse_size<D>(u, w, a.eps);
        float gu[8], gw[8];
        load_gamma(gu, gw, gamma, at);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] *= size * gu[e];
          w[e] *= size * gw[e];
        }
      }
      if (turns) turn<false>(u, w, s.turn + in * (D / 2) + 8 * at.p, a.pairs);
      x.from_float(u);
      y.from_float(w);
    }
    x.store(dst + 8 * at.c0);
    y.store(dst + 8 * at.c1);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(NormArgs a) {
  constexpr int kLanes = D / 16, kGroups = 64 / kLanes, kWaves = kThreads / 64;
  __shared__ Step<D> s_step[kWaves];
  __shared__ float s_sum[kWaves * kGroups][D + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int block;
  const int kind = kind_of(a, block);
  const NormPart& part = a.part[kind];
  const Place at(lane % kLanes, a);
  Step<D>& s = s_step[wave];
  const HeadRows &src = kind ? a.k : a.q, &grad = kind ? a.k_out : a.q_out, &to = kind ? a.dk : a.dq;
  float gu[8], gw[8], dgu[8] = {}, dgw[8] = {};  // gamma, this lane's sums of dgamma
  if (a.normalise) load_gamma(gu, gw, kind ? a.gamma_k : a.gamma_q, at);
  const bool turns = a.rot && at.turns;
  for (int id = block * kWaves + wave; id < part.steps * part.split; id += part.blocks * kWaves) {
    const int step = id / part.split, share = id % part.split;
    fill_step<D>(a, step * part.tokens, part.tokens, a.rot, lane, s, [&](int, int b, int i, bool there, int64_t (&x)[3]) {
      x[0] = offset_of(src, b, i);
      x[1] = offset_of(grad, b, i);
      x[2] = offset_of(to, b, i);
      return there;
    });
    for (int r = lane / kLanes + kGroups * share; r < part.tokens * part.heads; r += kGroups * part.split) {
      int in, h;
      part.by_heads.divide(r, in, h);
      if (!s.there[in]) continue;
      const T* dy = static_cast<const T*>(grad.p) + s.at[1][in] + h * grad.sh;
      const T* from = static_cast<const T*>(src.p) + s.at[0][in] + h * src.sh;
      T* dst = static_cast<T*>(to.p) + s.at[2][in] + h * to.sh;
      Chunk<T> x, y, cx, cy;
      load_row(x, dy + 8 * at.c0);
      load_row(y, dy + 8 * at.c1);
      if (a.normalise) {
        load_row(cx, from + 8 * at.c0);
        load_row(cy, from + 8 * at.c1);
      }
      if (a.normalise || turns) {
        float u[8], w[8];
        x.to_float(u);
        y.to_float(w);
        if (turns) turn<true>(u, w, s.turn + in * (D / 2) + 8 * at.p, a.pairs);
        if (a.normalise) {
          float xu[8], xw[8];
          cx.to_float(xu);
          cy.to_float(xw);
          const float size = inverse_size<D>(xu, xw, a.eps);
          float dot = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            xu[e] *= size;
            xw[e] *= size;
            dgu[e] += u[e] * xu[e];
            dgw[e] += w[e] * xw[e];
            u[e] *= gu[e];
            w[e] *= gw[e];
            dot += u[e] * xu[e] + w[e] * xw[e];
          }
          dot = row_sum<D>(dot) * (1.f / D);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            u[e] = size * (u[e] - xu[e] * dot);
            w[e] = size * (w[e] - xw[e] * dot);
          }
        }
        x.from_float(u);
        y.from_float(w);
      }
      x.store(dst + 8 * at.c0);
      y.store(dst + 8 * at.c1);
    }
  }
  if (!a.partial) return;
  // the block's sums, group by group in order
  const int group = wave * kGroups + lane / kLanes;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    s_sum[group][8 * at.c0 + e] = dgu[e];
    s_sum[group][8 * at.c1 + e] = dgw[e];
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float sum = 0.f;
#pragma unroll 8
    for (int g = 0; g < kWaves * kGroups; ++g) sum += s_sum[g][threadIdx.x];
    a.partial[(int64_t)blockIdx.x * D + threadIdx.x] = sum;
  }
}

// dgamma from the blocks' sums, in a fixed order: a block takes 32 elements of one
// of the two, 128 threads every four elements.
constexpr int kGammaThreads = 1024;
template <int D>
__global__ __launch_bounds__(kGammaThreads) void norm_gamma_kernel(NormArgs a) {
  constexpr int kParts = kGammaThreads / 8;
  __shared__ f32x4_t s_sum[kParts][8];
  const int kind = blockIdx.x / (D / 32), e = threadIdx.x % 8, at = threadIdx.x / 8;
  const int col = blockIdx.x % (D / 32) * 32 + 4 * e;
  float* to = kind ? a.dgamma_k : a.dgamma_q;
  if (!to) return;
  const int first = kind ? a.part[0].blocks : 0, n = a.part[kind].blocks;
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = at; i < n; i += kParts) {
    const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a.partial + (int64_t)(first + i) * D + col);
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] += x[k];
  }
  s_sum[at][e] = sum;
#pragma unroll
  for (int half = kParts / 2; half >= 1; half /= 2) {
    __syncthreads();
    if (at < half) {
      const f32x4_t x = s_sum[at + half][e];
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] += x[k];
      s_sum[at][e] = sum;
    }
  }
  if (at == 0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) to[col + k] = sum[k];
  }
}

// Waves that fill the chip (256 CUs of four SIMDs, some waves each).
constexpr int kFull = 8192;

// A wave's step: about four rows a lane group, so that the angles are worked out
// for several rows, but only while the steps fill the chip; with few of them the
// waves share a step's rows, until they fill the chip eight times over (4095 tokens
// of more than 136 heads of 128: behind it a lane group takes several rows, as a wave
// for every eight could pass 2^32 threads of a launch).
NormPart part_of(int tokens, int heads, int head_dim) {
  const int groups = 64 / (head_dim / 16);
  NormPart p;
  p.heads = heads;
  p.tokens = 1;
  p.steps = tokens;
  p.split = 1;
  p.blocks = 0;
  p.by_heads = FastDivide(heads ? heads : 1);
  if (!heads) return p;
  while (p.tokens < kNormTokens && p.tokens * heads < 4 * groups && tokens / (2 * p.tokens) >= kFull) p.tokens *= 2;
  p.steps = (tokens + p.tokens - 1) / p.tokens;
  if (p.steps < kFull / 2) p.split = std::min((p.tokens * heads + groups - 1) / groups, 1 + 8 * kFull / p.steps);
  p.blocks = (int)(((int64_t)p.steps * p.split + kThreads / 64 - 1) / (kThreads / 64));
  return p;
}

// Blocks of a part of the backward: those of the forward, but no more than what
// runs at once (each writes its sums of dgamma), queries and keys by their heads.
void limit_blocks(NormPart (&p)[3]) {
  const int64_t heads = p[0].heads + p[1].heads;
  for (int kind = 0; kind < 2; ++kind)
    if (p[kind].heads) p[kind].blocks = (int)std::min<int64_t>(p[kind].blocks, 1 + kFull / 4 * (int64_t)p[kind].heads / heads);
}

}  // namespace

// (As many waves as tokens with every split, which is what part_of() gives few tokens
// and more than it gives many: its steps halve and its splits end where they fill the
// chip: 1.05 MB of sums at 4095 tokens of 16 heads of 128, half of it at 4096.)
int norm_bwd_blocks(int tokens, int q_heads, int k_heads, int head_dim) {
  const int heads[2] = {q_heads, k_heads}, groups = 64 / (head_dim / 16);
  NormPart p[3] = {};
  for (int kind = 0; kind < 2; ++kind) {
    p[kind].heads = heads[kind];
    const int64_t waves = (int64_t)tokens * ((heads[kind] + groups - 1) / groups);
    p[kind].blocks = (int)std::min<int64_t>((waves + kThreads / 64 - 1) / (kThreads / 64), kFull);
  }
  limit_blocks(p);
  return p[0].blocks + p[1].blocks;
}

template <typename T, int D>
hipError_t launch_norm_d(const NormArgs& args, bool append, hipStream_t s) {
  NormArgs a = args;
  a.by_rows = FastDivide(a.num_rows);
  a.part[0] = part_of(a.tokens, a.q_heads, D);
  a.part[1] = part_of(a.tokens, a.k_heads, D);
  a.part[2] = part_of(a.tokens, append ? a.k_heads : 0, D);
  const dim3 grid((uint32_t)(a.part[0].blocks + a.part[1].blocks + a.part[2].blocks)), block(kThreads);
  return append ? launch_struct(norm_kernel<T, D, true>, grid, block, s, a)
                : launch_struct(norm_kernel<T, D, false>, grid, block, s, a);
}

hipError_t launch_norm(const NormArgs& a, bool append, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? launch_norm_d<bf16_bits, 128>(a, append, s) : launch_norm_d<bf16_bits, 64>(a, append, s);
  return head_dim == 128 ? launch_norm_d<float, 128>(a, append, s) : launch_norm_d<float, 64>(a, append, s);
}

template <typename T, int D>
hipError_t launch_norm_bwd_d(const NormArgs& args, hipStream_t s) {
  NormArgs a = args;
  a.by_rows = FastDivide(a.num_rows);
  a.part[0] = part_of(a.tokens, a.q_heads, D);
  a.part[1] = part_of(a.tokens, a.k_heads, D);
  a.part[2] = part_of(a.tokens, 0, D);
  limit_blocks(a.part);
  const dim3 grid((uint32_t)(a.part[0].blocks + a.part[1].blocks)), block(kThreads);
  const hipError_t e = launch_struct(norm_bwd_kernel<T, D>, grid, block, s, a);
  if (e != hipSuccess || !a.partial) return e;
  return launch_struct(norm_gamma_kernel<D>, dim3(2 * D / 32), dim3(kGammaThreads), s, a);
}

hipError_t launch_norm_bwd(const NormArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? launch_norm_bwd_d<bf16_bits, 128>(a, s) : launch_norm_bwd_d<bf16_bits, 64>(a, s);
  return head_dim == 128 ? launch_norm_bwd_d<float, 128>(a, s) : launch_norm_bwd_d<float, 64>(a, s);
}

}  // namespace skv
