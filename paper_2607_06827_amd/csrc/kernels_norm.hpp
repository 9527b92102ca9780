// Internal interface between the C-ABI host layer and the kernels of the per-head
// norms with rotation (include/speechkv_norm.h).
#pragma once

#include "kernels_draft.hpp"

namespace skv {

// Rows of one tensor: element (b, i, h, e) at p + b*sb + i*ss + h*sh + e.
struct HeadRows {
  void* p;
  int64_t sb, ss, sh;
};

// Most tokens of a wave's step.
constexpr int kNormTokens = 8;

// How one kind of rows (queries, keys or values) is dealt out: a step of a wave
// takes the rows of `tokens` tokens, `split` waves share a step, and the kind has
// `blocks` blocks.
struct NormPart {
  int heads;     // 0: there are none
  int tokens, steps, split, blocks;
  FastDivide by_heads;
};

struct NormArgs {
  HeadRows q, k, v;        // inputs (v: appended values)
  HeadRows q_out, k_out;   // k_out: not of the append
  HeadRows dq, dk;         // backward: gradients of the inputs (q_out, k_out: of the outputs)
  int q_heads, k_heads;    // 0: without them
  int num_rows, tokens;    // rows of a sequence, rows in all
  FastDivide by_rows;      // num_rows (set by the launcher, as the parts)
  NormPart part[3];        // queries, keys, values
  const int32_t* row_len;  // may be null: num_rows
  int normalise;
  const float* gamma_q;    // may be null: 1
  const float* gamma_k;
  float eps;
  int rot;                 // rotated elements of a head
  int pairs;               // neighbouring elements (else halves)
  const int32_t* positions;
  const float* inv_freq;
  const int32_t* axis;     // may be null: the first
  int num_axes;
  // the append's cache
  const int32_t* cache_len;
  void* k_pages;
  void* v_pages;
  const int32_t* table;
  PagedView pv;
  int32_t* cache_len_out;  // may be null
  // backward
  float* partial;          // [blocks of the queries, then of the keys][D] sums of dgamma, null: none wanted
  float* dgamma_q;         // may be null
  float* dgamma_k;
};

// dtype: 0 = fp32, 1 = bf16.  Each launcher returns the launch status.
hipError_t launch_norm(const NormArgs& a, bool append, int dtype, int head_dim, hipStream_t s);
// The backward, and with a.partial the sums of dgamma behind it.
hipError_t launch_norm_bwd(const NormArgs& a, int dtype, int head_dim, hipStream_t s);
// Most blocks that write sums of dgamma in any backward of up to so many tokens.
int norm_bwd_blocks(int tokens, int q_heads, int k_heads, int head_dim);

}  // namespace skv
