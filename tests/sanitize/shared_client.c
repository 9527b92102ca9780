/*
 * Exercises the host layers of include/speechkv_norm.h and
 * include/speechkv_shared.h (argument checks, overlap checks of strided views, the
 * choice of block shapes and splits) under AddressSanitizer and
 * UndefinedBehaviorSanitizer.  Pointers are fake, 16-byte aligned device addresses
 * that are never dereferenced on these paths: every call is either rejected by a
 * host check, or (with the argument "nodevice", on a machine without a GPU) passes
 * every check and fails at the device, which returns SPEECHKV_ERR_HIP.  Prints "ok
 * <count>" when every call returned what it may.
 */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "speechkv_shared.h"

#define P(x) ((void*)(uintptr_t)(x))
#define AT(i) P(0x10000000ull + ((unsigned long long)(i) << 24))

static int checks = 0, failures = 0, nodevice = 0;

/* A refusal, or the device's, where there is none. */
static void refused(int got, const char* what) {
  ++checks;
  if (got > SPEECHKV_OK || got < SPEECHKV_ERR_SCRATCH || (got == SPEECHKV_ERR_HIP && !nodevice)) {
    ++failures;
    printf("FAIL %s: got %d\n", what, got);
  }
}

static speechkv_paged_kv cache(int32_t heads, int32_t dtype) {
  speechkv_paged_kv c;
  c.k_pages = AT(0);
  c.v_pages = AT(1);
  c.block_table = (const int32_t*)AT(2);
  c.num_pages = 64;
  c.page_size = 16;
  c.max_pages_per_seq = 8;
  c.num_kv_heads = heads;
  c.head_dim = 64;
  c.dtype = dtype;
  return c;
}

static speechkv_heads heads(int at, int64_t sb, int64_t ss, int64_t sh, int32_t n) {
  speechkv_heads h;
  h.data = AT(at);
  h.stride_b = sb;
  h.stride_s = ss;
  h.stride_h = sh;
  h.num_heads = n;
  return h;
}

int main(int argc, char** argv) {
  const int64_t wide[] = {0, 8, 4, -8, 64, 512, 768, INT64_MAX, INT64_MIN, INT64_MAX - 7, (int64_t)1 << 62, (int64_t)1 << 59};
  const int32_t counts[] = {1, 0, -1, 2, 3, 65535, 65536, 1 << 24, INT32_MAX, INT32_MIN};
  const int nw = (int)(sizeof wide / sizeof *wide), nc = (int)(sizeof counts / sizeof *counts);
  speechkv_head_norm norm = {(const float*)AT(20), (const float*)AT(21), 1e-6f};
  speechkv_rope rope = {(const int32_t*)AT(22), (const float*)AT(23), (const int32_t*)AT(24), 3, 64, SPEECHKV_ROPE_HALVES};
  int i, j, k, l;
  nodevice = argc > 1 && !strcmp(argv[1], "nodevice");
  /* strides of every view against each other */
  for (i = 0; i < nw; ++i)
    for (j = 0; j < nw; ++j)
      for (k = 0; k < nw; ++k) {
        speechkv_heads q = heads(8, wide[i], wide[j], wide[k], 4), o = heads(9, wide[k], wide[i], wide[j], 4);
        speechkv_heads kk = heads(8, wide[j], wide[j], wide[k], 2), dense = heads(10, 3 * 256, 256, 64, 4);
        speechkv_paged_kv c = cache(2, SPEECHKV_DTYPE_BF16);
        refused(speechkv_norm_rope(&q, NULL, 2, 3, NULL, 64, SPEECHKV_DTYPE_BF16, &norm, &rope, &o, NULL, NULL), "norm");
        refused(speechkv_norm_rope(&dense, &kk, 2, 3, NULL, 64, SPEECHKV_DTYPE_F32, NULL, &rope, &o, &kk, NULL), "in place");
        refused(speechkv_norm_rope_bwd(&q, NULL, &dense, NULL, 2, 3, NULL, 64, SPEECHKV_DTYPE_BF16, &norm, &rope, &o, NULL,
                                       (float*)AT(30), NULL, AT(31), 1 << 20, NULL),
                "backward");
        refused(speechkv_norm_append_kv(&q, &kk, &kk, 2, 3, NULL, &norm, &rope, (const int32_t*)AT(25), &c, &o,
                                        (int32_t*)AT(26), NULL),
                "append");
        refused(speechkv_attn_weights(&q, 2, 3, (const float*)AT(27), wide[k], wide[j], wide[i], NULL, &c,
                                      (const int32_t*)AT(25), 100, 0.125f, NULL, (float*)AT(28), 120, NULL),
                "weights");
      }
  /* counts and sizes */
  for (i = 0; i < nc; ++i)
    for (j = 0; j < nc; ++j)
      for (k = 0; k < nc; ++k) {
        speechkv_heads q = heads(8, 0, 0, 64, counts[k] > 0 && counts[k] < 65536 ? counts[k] : 4);
        speechkv_paged_kv c = cache(counts[k], SPEECHKV_DTYPE_F32);
        speechkv_evict_layer y;
        refused(speechkv_norm_rope(&q, NULL, counts[i], counts[j], NULL, 64, SPEECHKV_DTYPE_F32, &norm, &rope, &q, NULL, NULL),
                "norm counts");
        refused(speechkv_attn_weights(&q, counts[i], counts[j], (const float*)AT(27), 0, 0, 0, (const int32_t*)AT(26), &c,
                                      (const int32_t*)AT(25), 100, 0.125f, NULL, (float*)P(1ull << 62), counts[k], NULL),
                "weights counts");
        (void)speechkv_norm_rope_bwd_workspace_bytes(counts[i], counts[j], counts[k], counts[i], 64);
        for (l = 0; l < nc; ++l) {
          (void)speechkv_shared_num_splits(counts[i], counts[j], counts[k], 16, 8, 128, SPEECHKV_DTYPE_BF16, counts[l], 100);
          (void)speechkv_shared_workspace_bytes(counts[i], counts[j], counts[k], counts[l], 2, 64, 100, 100, counts[l]);
          ++checks;
          c = cache(2, SPEECHKV_DTYPE_BF16);
          refused(speechkv_shared_attn(AT(8), counts[i], 4, &c, (const int32_t*)AT(9), 100, (const int32_t*)AT(10), counts[j],
                                       counts[k], &c, (const int32_t*)AT(11), 100, 0.125f, counts[l], P(1ull << 60), NULL,
                                       P(1ull << 61), (size_t)1 << 58, NULL),
                  "shared counts");
          c = cache(counts[i], SPEECHKV_DTYPE_BF16);
          y.cache = c;
          y.cache_len = (const int32_t*)AT(11);
          y.cache_len_out = NULL;
          y.weights = y.weights_out = (float*)P(1ull << 60);
          y.kept = (int32_t*)P(1ull << 62);
          refused(speechkv_evict(&y, 1, counts[j], (const int32_t*)AT(9), counts[k], counts[l], counts[i], counts[j], NULL),
                  "evict counts");
        }
      }
  if (failures) printf("failed %d of %d\n", failures, checks);
  else printf("ok %d\n", checks);
  return failures != 0;
}
