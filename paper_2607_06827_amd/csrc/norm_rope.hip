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
// lanes hold a row and add their sums with lane exchanges.  A block takes some
// tokens (rows of q and k of one position): their sines and cosines are computed
// once, by a thread each, and shared through LDS.  Angles are counted in turns,
// whose whole part drops out in 64 bits, so that far positions lose nothing.
//
// Sums, norms, the rotation and gradients are fp32; each output is rounded once.
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

// A block's tokens: sequence and row of token t, whether the sequence has it.
struct Token {
  int b, i;
  bool there;
};
__device__ __forceinline__ Token token(const NormArgs& a, int t) {
  const bool in = t < a.tokens;
  int b, i;
  a.by_rows.divide(in ? t : 0, b, i);
  const int n = a.row_len ? a.row_len[b] : a.num_rows;
  return {b, i, in && i < n};
}

// (cos, sin) of the angles of the block's tokens, D / 2 apart.
template <int D>
__device__ __forceinline__ void fill_turns(const NormArgs& a, int first, float2* s_turn) {
  const int half = a.rot / 2, batch_rows = a.tokens;
  for (int x = threadIdx.x; x < a.per_block * (D / 2); x += kThreads) {
    const int j = x % (D / 2), t = first + x / (D / 2);
    if (j >= half || t >= batch_rows) continue;
    const Token k = token(a, t);
    if (!k.there) continue;
    const int axis = a.axis ? min(max(a.axis[j], 0), a.num_axes - 1) : 0;
    const double n = (double)a.positions[(int64_t)axis * batch_rows + t] * ((double)a.inv_freq[j] * 0.15915494309189535);
    float s, c;
    sincospif(2.f * (float)(n - __builtin_rint(n)), &s, &c);
    s_turn[x] = make_float2(c, s);
  }
}

template <typename T>
__device__ __forceinline__ const T* row_at(const HeadRows& x, const Token& k, int h) {
  return static_cast<const T*>(x.p) + k.b * x.sb + k.i * x.ss + h * x.sh;
}

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

// kAppend: keys and values go behind the cache's entries.
template <typename T, int D, bool kAppend>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  constexpr int kLanes = D / 16;  // of a row
  __shared__ float2 s_turn[kNormTokens * (D / 2)];
  const int tid = threadIdx.x, first = blockIdx.x * a.per_block;
  const Place at(tid % kLanes, a);
  if (a.rot) {
    fill_turns<D>(a, first, s_turn);
    __syncthreads();
  }
  // what goes where: q rows, k rows and v rows of one token after the other
  auto move = [&](const T* src, T* dst, const float2* t, const float* gamma, bool plain) {
    Chunk<T> x, y;
    load_row(x, src + 8 * at.c0);
    load_row(y, src + 8 * at.c1);
    if (!plain && (a.normalise || at.turns)) {
      float u[8], w[8];
      x.to_float(u);
      y.to_float(w);
      if (a.normalise) {
        const float r = inverse_size<D>(u, w, a.eps);
        float gu[8], gw[8];
        load_gamma(gu, gw, gamma, at);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] *= r * gu[e];
          w[e] *= r * gw[e];
        }
      }
      if (at.turns) turn<false>(u, w, t + 8 * at.p, a.pairs);
      x.from_float(u);
      y.from_float(w);
    }
    x.store(dst + 8 * at.c0);
    y.store(dst + 8 * at.c1);
  };
  for (int r = tid / kLanes; r < a.per_block * a.q_heads; r += kThreads / kLanes) {
    int in, h;
    a.by_q.divide(r, in, h);
    const Token k = token(a, first + in);
    if (!k.there) continue;
    move(row_at<T>(a.q, k, h), const_cast<T*>(row_at<T>(a.q_out, k, h)), s_turn + in * (D / 2), a.gamma_q, false);
  }
  const int k_rows = a.k_heads * (kAppend ? 2 : 1);
  for (int r = tid / kLanes; r < a.per_block * k_rows; r += kThreads / kLanes) {
    int in, h;
    a.by_k.divide(r, in, h);
    const bool is_v = kAppend && in >= a.per_block;  // (all keys first)
    if (is_v) in -= a.per_block;
    const Token k = token(a, first + in);
    if (!k.there) continue;
    T* dst;
    if constexpr (kAppend) {
      const int64_t slot = (int64_t)max(a.cache_len[k.b], 0) + k.i;
      const int64_t index = slot >> a.pv.page_shift;
      if (index >= a.pv.max_pages) continue;
      const int64_t page = a.table[(int64_t)k.b * a.pv.max_pages + index];
      if (page < 0 || page >= a.pv.num_pages) continue;
      dst = static_cast<T*>(is_v ? a.v_pages : a.k_pages) +
            page_row<D>(page, h, (int)(slot & ((1 << a.pv.page_shift) - 1)), a.pv);
    } else {
      dst = const_cast<T*>(row_at<T>(a.k_out, k, h));
    }
    move(row_at<T>(is_v ? a.v : a.k, k, h), dst, s_turn + in * (D / 2), a.gamma_k, is_v);
  }
  if constexpr (kAppend) {
    if (a.cache_len_out && tid < a.per_block && first + tid < a.tokens) {
      int b, i;
      a.by_rows.divide(first + tid, b, i);
      const int n = a.row_len ? min(max(a.row_len[b], 0), a.num_rows) : a.num_rows;
      if (i == 0) a.cache_len_out[b] = (int32_t)min((int64_t)max(a.cache_len[b], 0) + n, (int64_t)INT32_MAX);
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(NormArgs a) {
  constexpr int kLanes = D / 16, kGroups = kThreads / kLanes;
  __shared__ float2 s_turn[kNormTokens * (D / 2)];
  __shared__ float s_sum[kGroups][D + 4];
  const int tid = threadIdx.x, group = tid / kLanes;
  const Place at(tid % kLanes, a);
  float dgu[2][8] = {}, dgw[2][8] = {};  // this lane's sums of dgamma_q and dgamma_k
  for (int first = blockIdx.x * a.per_block; first < a.tokens; first += a.blocks * a.per_block) {
    if (a.rot) {
      __syncthreads();  // (the last tokens' angles have been read)
      fill_turns<D>(a, first, s_turn);
      __syncthreads();
    }
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const HeadRows &src = kind ? a.k : a.q, &grad = kind ? a.k_out : a.q_out, &to = kind ? a.dk : a.dq;
      const int heads = kind ? a.k_heads : a.q_heads;
      float gu[8], gw[8];
      if (a.normalise) load_gamma(gu, gw, kind ? a.gamma_k : a.gamma_q, at);
      for (int r = group; r < a.per_block * heads; r += kGroups) {
        int in, h;
        (kind ? a.by_k : a.by_q).divide(r, in, h);
        const Token k = token(a, first + in);
        if (!k.there) continue;
        const T* dy = row_at<T>(grad, k, h);
        Chunk<T> x, y;
        load_row(x, dy + 8 * at.c0);
        load_row(y, dy + 8 * at.c1);
        if (a.normalise || at.turns) {
          float u[8], w[8];
          x.to_float(u);
          y.to_float(w);
          if (at.turns) turn<true>(u, w, s_turn + in * (D / 2) + 8 * at.p, a.pairs);
          if (a.normalise) {
            const T* from = row_at<T>(src, k, h);
            float xu[8], xw[8];
            Chunk<T> c;
            load_row(c, from + 8 * at.c0);
            c.to_float(xu);
            load_row(c, from + 8 * at.c1);
            c.to_float(xw);
            const float s = inverse_size<D>(xu, xw, a.eps);
            float dot = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              xu[e] *= s;
              xw[e] *= s;
              dgu[kind][e] += u[e] * xu[e];
              dgw[kind][e] += w[e] * xw[e];
              u[e] *= gu[e];
              w[e] *= gw[e];
              dot += u[e] * xu[e] + w[e] * xw[e];
            }
            dot = row_sum<D>(dot) * (1.f / D);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              u[e] = s * (u[e] - xu[e] * dot);
              w[e] = s * (w[e] - xw[e] * dot);
            }
          }
          x.from_float(u);
          y.from_float(w);
        }
        T* dst = const_cast<T*>(row_at<T>(to, k, h));
        x.store(dst + 8 * at.c0);
        y.store(dst + 8 * at.c1);
      }
    }
  }
  if (!a.partial) return;
  // the block's sums, group by group in order
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s_sum[group][8 * at.c0 + e] = dgu[kind][e];
      s_sum[group][8 * at.c1 + e] = dgw[kind][e];
    }
    __syncthreads();
    if (tid < D) {
      float sum = 0.f;
      for (int g = 0; g < kGroups; ++g) sum += s_sum[g][tid];
      a.partial[((int64_t)blockIdx.x * 2 + kind) * D + tid] = sum;
    }
  }
}

// dgamma from the blocks' sums, in a fixed order: a block takes 8 elements of one
// of the two, 32 threads an element.
template <int D>
__global__ __launch_bounds__(kThreads) void norm_gamma_kernel(NormArgs a) {
  __shared__ float s_sum[32][9];
  const int kind = blockIdx.x / (D / 8), e = blockIdx.x % (D / 8) * 8 + threadIdx.x % 8, part = threadIdx.x / 8;
  float* to = kind ? a.dgamma_k : a.dgamma_q;
  if (!to) return;
  float sum = 0.f;
  for (int n = part; n < a.blocks; n += 32) sum += a.partial[((int64_t)n * 2 + kind) * D + e];
  s_sum[part][threadIdx.x % 8] = sum;
  __syncthreads();
  if (part == 0) {
    sum = 0.f;
    for (int n = 0; n < 32; ++n) sum += s_sum[n][threadIdx.x];
    to[e] = sum;
  }
}

NormArgs with_divisors(const NormArgs& a) {
  NormArgs x = a;
  x.by_rows = FastDivide(a.num_rows);
  x.by_q = FastDivide(a.q_heads ? a.q_heads : 1);
  x.by_k = FastDivide(a.k_heads ? a.k_heads : 1);
  return x;
}

}  // namespace

int norm_bwd_blocks(int tokens) { return tokens < 1024 ? tokens : 1024; }

template <typename T, int D>
hipError_t launch_norm_d(const NormArgs& a, bool append, hipStream_t s) {
  const dim3 grid((uint32_t)((a.tokens + a.per_block - 1) / a.per_block)), block(kThreads);
  return append ? launch_struct(norm_kernel<T, D, true>, grid, block, s, a)
                : launch_struct(norm_kernel<T, D, false>, grid, block, s, a);
}

hipError_t launch_norm(const NormArgs& args, bool append, int dtype, int head_dim, hipStream_t s) {
  NormArgs a = with_divisors(args);
  a.per_block = 1;
  if (dtype == 1) return head_dim == 128 ? launch_norm_d<bf16_bits, 128>(a, append, s) : launch_norm_d<bf16_bits, 64>(a, append, s);
  return head_dim == 128 ? launch_norm_d<float, 128>(a, append, s) : launch_norm_d<float, 64>(a, append, s);
}

hipError_t launch_norm_bwd(const NormArgs& args, int dtype, int head_dim, hipStream_t s) {
  NormArgs a = with_divisors(args);
  a.per_block = 1;
  const dim3 grid((uint32_t)a.blocks), block(kThreads);
  if (dtype == 1) {
    if (head_dim == 128) return launch_struct(norm_bwd_kernel<bf16_bits, 128>, grid, block, s, a);
    return launch_struct(norm_bwd_kernel<bf16_bits, 64>, grid, block, s, a);
  }
  if (head_dim == 128) return launch_struct(norm_bwd_kernel<float, 128>, grid, block, s, a);
  return launch_struct(norm_bwd_kernel<float, 64>, grid, block, s, a);
}

hipError_t launch_norm_gamma(const NormArgs& a, int head_dim, hipStream_t s) {
  const dim3 grid(2 * head_dim / 8), block(kThreads);
  return head_dim == 128 ? launch_struct(norm_gamma_kernel<128>, grid, block, s, a)
                         : launch_struct(norm_gamma_kernel<64>, grid, block, s, a);
}

}  // namespace skv
