/*
 * Exercises the host layer of include/speechkv_draft.h (argument checks,
 * overlap checks, the choice of block shape and splits) under AddressSanitizer
 * and UndefinedBehaviorSanitizer.  Pointers are fake, 16-byte aligned device
 * addresses that are never dereferenced on these paths: every call is either
 * rejected by a host check, or (with the argument "nodevice", on a machine
 * without a GPU) passes every check and fails at the device, which returns
 * SPEECHKV_ERR_HIP.  Prints "ok <count>" when every call returned what it
 * should.
 */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "speechkv_draft.h"

#define P(x) ((void*)(uintptr_t)(x))
#define AT(i) P(0x10000000ull + ((unsigned long long)(i) << 24))

static int checks = 0, failures = 0;

static void expect(long long got, long long want, const char* what) {
  ++checks;
  if (got != want) {
    ++failures;
    printf("FAIL %s: got %lld want %lld\n", what, got, want);
  }
}

static speechkv_paged_kv cache(void) {
  speechkv_paged_kv c;
  c.k_pages = AT(0);
  c.v_pages = AT(1);
  c.block_table = (const int32_t*)AT(2);
  c.num_pages = 64;
  c.page_size = 16;
  c.max_pages_per_seq = 8;
  c.num_kv_heads = 2;
  c.head_dim = 64;
  c.dtype = SPEECHKV_DTYPE_BF16;
  return c;
}

static int append(const speechkv_paged_kv* c, int64_t sb, int64_t ss, int64_t sh, int32_t batch, int32_t n, int32_t rot,
                  void* q_out) {
  return speechkv_append_kv(AT(8), sb, ss, sh, 4, AT(9), AT(10), sb, ss, sh, batch, n, NULL, (const int32_t*)AT(11),
                            (const float*)AT(12), rot, SPEECHKV_ROPE_HALVES, (const int32_t*)AT(13), c, q_out, NULL,
                            NULL);
}

static int tree(const speechkv_paged_kv* c, int32_t batch, int32_t n, int32_t hq, int32_t max_len, int64_t stride,
                float scale, int32_t splits, size_t ws) {
  return speechkv_tree_attn(AT(8), batch, n, hq, c, (const int32_t*)AT(9), max_len, NULL, (const uint32_t*)AT(10),
                            stride, scale, splits, AT(11), AT(40), ws, NULL);
}

int main(int argc, char** argv) {
  const int nodevice = argc > 1 && !strcmp(argv[1], "nodevice");
  speechkv_paged_kv c = cache();
  const int64_t wide[] = {0, 8, 4, -8, 512, INT64_MAX, INT64_MIN, INT64_MAX - 7, (int64_t)1 << 62};
  for (unsigned i = 0; i < sizeof wide / sizeof *wide; ++i) {
    const int bad = wide[i] < 0 || wide[i] % 8 || wide[i] > ((int64_t)1 << 60);
    if (bad || nodevice) {
      expect(append(&c, wide[i], 256, 64, 2, 3, 64, AT(14)), bad ? SPEECHKV_ERR_INVALID_ARG : SPEECHKV_ERR_HIP, "sb");
      expect(append(&c, 768, wide[i], 64, 2, 3, 64, AT(14)), bad ? SPEECHKV_ERR_INVALID_ARG : SPEECHKV_ERR_HIP, "ss");
      expect(append(&c, 768, 256, wide[i], 2, 3, 64, AT(14)), bad ? SPEECHKV_ERR_INVALID_ARG : SPEECHKV_ERR_HIP, "sh");
    }
  }
  for (int32_t rot = -16; rot <= 80; rot += 8) {
    const int bad = rot < 0 || rot > 64 || rot % 16;
    if (bad || nodevice)
      expect(append(&c, 768, 256, 64, 2, 3, rot, AT(14)), bad ? SPEECHKV_ERR_INVALID_ARG : SPEECHKV_ERR_HIP, "rot");
  }
  expect(append(&c, 768, 256, 64, INT32_MAX, 3, 64, AT(14)), SPEECHKV_ERR_INVALID_ARG, "batch");
  expect(append(&c, 768, 256, 64, 2, INT32_MAX, 64, AT(14)), SPEECHKV_ERR_INVALID_ARG, "num_new");
  expect(append(&c, 768, 256, 64, 2, 3, 64, AT(9)), SPEECHKV_ERR_ALIAS, "q_out over k");
  expect(append(NULL, 768, 256, 64, 2, 3, 64, AT(14)), SPEECHKV_ERR_INVALID_ARG, "no cache");

  const int32_t counts[] = {INT32_MIN, -1, 0, 1, 2, 31, 1024, 1025, 65535, 65536, INT32_MAX};
  const int nc = (int)(sizeof counts / sizeof *counts);
  for (int i = 0; i < nc; ++i)
    for (int j = 0; j < nc; ++j)
      for (int k = 0; k < nc; ++k) {
        const int32_t b = counts[i], n = counts[j], len = counts[k];
        const int32_t s = speechkv_tree_num_splits(b, n, 16, 8, 128, SPEECHKV_DTYPE_BF16, len);
        const int ok = b >= 1 && n >= 1 && n <= SPEECHKV_MAX_TREE_NODES && len >= 0;
        expect(ok ? s >= 1 && s <= 32 : s == -1, 1, "splits");
        const size_t ws = speechkv_tree_workspace_bytes(b, n, 16, 8, 128, len, 0);
        expect(ok || ws == 0, 1, "workspace");
        expect(speechkv_tree_workspace_bytes(b, n, 16, 8, 128, len, -1) == 0, 1, "no workspace");
        const int fits = b <= 65535 && len <= 128;
        if (!ok || !fits) expect(tree(&c, b, n, 4, len, 1, 0.125f, 1, 0), SPEECHKV_ERR_INVALID_ARG, "tree sizes");
      }
  for (int i = 0; i < nc; ++i) {
    const int32_t x = counts[i];
    if (x < 0 || x > 65535) expect(tree(&c, 2, 5, 4, 100, 5, 0.125f, x, 1u << 20), SPEECHKV_ERR_INVALID_ARG, "splits");
    if (x > 1 && x <= 65535) expect(tree(&c, 2, 5, 4, 100, 5, 0.125f, x, 64), SPEECHKV_ERR_WORKSPACE, "small");
    if (x != 4 && x != 2 && x != 8 && x != 16)
      expect(tree(&c, 2, 5, x, 100, 5, 0.125f, 1, 0), x == 65536 ? SPEECHKV_ERR_UNSUPPORTED
             : x == 1024 ? SPEECHKV_ERR_UNSUPPORTED : SPEECHKV_ERR_INVALID_ARG, "heads");
  }
  expect(tree(&c, 2, 5, 4, 100, INT64_MAX, 0.125f, 1, 0), SPEECHKV_ERR_INVALID_ARG, "mask stride");
  expect(tree(&c, 2, 5, 4, 100, -1, 0.125f, 1, 0), SPEECHKV_ERR_INVALID_ARG, "mask stride");
  if (nodevice) {
    expect(tree(&c, 2, 5, 4, 100, 5, 0.125f, 1, 0), SPEECHKV_ERR_HIP, "tree");
    expect(tree(&c, 2, 5, 4, 128, 0, 0.125f, 3, 1u << 20), SPEECHKV_ERR_HIP, "tree in splits");
  }

  static speechkv_layer_cache layers[SPEECHKV_MAX_COMMIT_LAYERS + 1];
  for (int i = 0; i <= SPEECHKV_MAX_COMMIT_LAYERS; ++i) {
    layers[i].cache = cache();
    layers[i].cache_len = (const int32_t*)AT(3);
    layers[i].cache_len_out = (int32_t*)((char*)AT(4) + 64 * i);
  }
  const int32_t* path = (const int32_t*)AT(5);
  const int32_t* plen = (const int32_t*)AT(6);
  for (int i = 0; i < nc; ++i) {
    const int32_t x = counts[i];
    if (x < 1 || x > SPEECHKV_MAX_COMMIT_LAYERS)
      expect(speechkv_tree_commit(layers, x, 2, path, 3, plen, 5, NULL), SPEECHKV_ERR_INVALID_ARG, "layers");
    if (x < 1 || x > 65535) expect(speechkv_tree_commit(layers, 1, x, path, 3, plen, 5, NULL), SPEECHKV_ERR_INVALID_ARG, "batch");
    if (x < 1 || x > 5) expect(speechkv_tree_commit(layers, 1, 2, path, x, plen, 5, NULL), SPEECHKV_ERR_INVALID_ARG, "path");
    if (x < 3 || x > SPEECHKV_MAX_TREE_NODES)
      expect(speechkv_tree_commit(layers, 1, 2, path, 3, plen, x, NULL), SPEECHKV_ERR_INVALID_ARG, "nodes");
  }
  expect(speechkv_tree_commit(NULL, 1, 2, path, 3, plen, 5, NULL), SPEECHKV_ERR_INVALID_ARG, "no layers");
  if (nodevice) {
    expect(speechkv_tree_commit(layers, SPEECHKV_MAX_COMMIT_LAYERS, 2, path, 3, plen, 5, NULL), SPEECHKV_ERR_HIP, "all layers");
    expect(speechkv_tree_commit(layers, 33, 2, path, 1, plen, 1024, NULL), SPEECHKV_ERR_HIP, "33 layers");
  }
  layers[200].cache_len_out = (int32_t*)AT(6);
  expect(speechkv_tree_commit(layers, 256, 2, path, 3, plen, 5, NULL), SPEECHKV_ERR_ALIAS, "out over path_len");
  if (failures) return 1;
  printf("ok %d\n", checks);
  return 0;
}
