/* Host-side exercise of the calls around a verification step's attention for sanitizer builds, in plain C.  Every call here
 * must be answered by argument checks and workspace sizing alone, before any device work; device pointers are made up. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "moespec.h"

static int failures = 0;

#define EXPECT(cond)                                                   \
  do {                                                                 \
    if (!(cond)) {                                                     \
      fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
      ++failures;                                                      \
    }                                                                  \
  } while (0)

static void *fake(uintptr_t a) { return (void *)a; }

static moespec_attn_desc make_desc(int h, int hk, int d, int cap, int dtype) {
  moespec_attn_desc ds;
  memset(&ds, 0, sizeof ds);
  ds.n_heads = h;
  ds.n_kv_heads = hk;
  ds.head_dim = d;
  ds.capacity = cap;
  ds.dtype = dtype;
  ds.scale = 0.125f;
  return ds;
}

static moespec_tree make_tree(int n_seq, int M, int max_tree) {
  moespec_tree t;
  memset(&t, 0, sizeof t);
  t.n_seq = n_seq;
  t.n_tokens = M;
  t.max_tree = max_tree;
  t.tree_off = fake(0x90000);
  return t;
}

static void descriptors_and_workspaces(void) {
  const int dims[] = {64, 96, 128, 192, 256};
  for (size_t i = 0; i < sizeof dims / sizeof dims[0]; ++i)
    for (int dt = MOESPEC_F32; dt <= MOESPEC_BF16; ++dt) {
      moespec_attn_desc ds = make_desc(32, 4, dims[i], 70000, dt);
      EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_OK);
      size_t prev = 0;
      for (int len = 0; len <= 70000; len += 3500) { /* a longer cache never needs less */
        const size_t w = moespec_attn_workspace_bytes(&ds, 4, 252, 63, len);
        EXPECT(w > 0 && w >= prev);
        prev = w;
      }
      prev = 0;
      for (int t = 1; t <= 511; t += 17) { /* nor does a larger tree, nor more sequences */
        const size_t w = moespec_attn_workspace_bytes(&ds, 1, 511, t, 4000);
        EXPECT(w >= prev && moespec_attn_workspace_bytes(&ds, 2, 1022, t, 4000) >= w);
        prev = w;
      }
    }
  EXPECT(moespec_check_attn_desc(NULL) == MOESPEC_ERR_INVALID_ARG);
  moespec_attn_desc ds = make_desc(32, 4, 128, 100, 7);
  EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_ERR_INVALID_ARG);
  ds = make_desc(30, 4, 128, 100, MOESPEC_BF16);
  EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_ERR_INVALID_ARG);
  ds = make_desc(32, 4, 80, 100, MOESPEC_BF16);
  EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_ERR_UNSUPPORTED_SHAPE);
  ds = make_desc(2048, 4, 128, 100, MOESPEC_BF16);
  EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_ERR_UNSUPPORTED_SHAPE);
  ds = make_desc(32, 4, 128, 0, MOESPEC_BF16);
  EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_ERR_INVALID_ARG);
  const float scales[] = {0.f, -1.f, NAN, INFINITY};
  for (size_t i = 0; i < 4; ++i) {
    ds = make_desc(32, 4, 128, 100, MOESPEC_BF16);
    ds.scale = scales[i];
    EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_ERR_INVALID_ARG);
    EXPECT(moespec_attn_workspace_bytes(&ds, 1, 8, 8, 50) == 0);
  }
  ds = make_desc(1024, 1024, 256, INT32_MAX, MOESPEC_F32);
  const int32_t big[] = {1, 2, 65535, 65536, INT32_MAX, -1, 0, INT32_MIN};
  for (size_t i = 0; i < 8; ++i)
    for (size_t j = 0; j < 8; ++j) {
      (void)moespec_attn_workspace_bytes(&ds, big[i], 65535, big[j], INT32_MAX);
      (void)moespec_attn_workspace_bytes(&ds, 65535, big[i], big[j], big[(i + j) % 8]);
      (void)moespec_evict_workspace_bytes(&ds, 1, big[i], big[j]);
    }
  EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_ERR_UNSUPPORTED_SHAPE); /* entries in whole tiles have to fit 32 bits */
  ds.capacity = 0x7fff0000;
  EXPECT(moespec_check_attn_desc(&ds) == MOESPEC_OK);
  for (size_t i = 0; i < 8; ++i)
    for (size_t j = 0; j < 8; ++j) {
      (void)moespec_attn_workspace_bytes(&ds, big[i], 65535, big[j], 0x7fff0000);
      (void)moespec_attn_workspace_bytes(&ds, 65535, big[i], big[j], big[(i + j) % 8]);
    }
  EXPECT(moespec_attn_workspace_bytes(&ds, 1, 8, 9, 50) == 0);  /* a tree larger than all tokens */
  EXPECT(moespec_attn_workspace_bytes(&ds, 0, 8, 8, 50) == 0);
  EXPECT(moespec_evict_workspace_bytes(&ds, 0, 1, 8) == 0);
  EXPECT(moespec_evict_workspace_bytes(NULL, 1, 1, 8) == 0);
}

static moespec_status attend(const moespec_attn_desc *ds, const moespec_tree *t, uintptr_t q, uintptr_t kc, uintptr_t len,
                             int max_len, uintptr_t out, uintptr_t ws, size_t bytes) {
  return moespec_tree_attention(ds, t, fake(q), fake(0x20000), fake(0x30000), fake(kc), fake(kc), fake(len), max_len, fake(out),
                                NULL, fake(ws), bytes, NULL);
}

static void attention_arguments(void) {
  moespec_attn_desc ds = make_desc(8, 2, 64, 100, MOESPEC_BF16);
  moespec_tree t = make_tree(2, 16, 8);
  const size_t need = moespec_attn_workspace_bytes(&ds, 2, 16, 8, 100);
  const uintptr_t q = 0x10000, kc = 0x40000, len = 0x50000, out = 0x60000, ws = 0x70000;
  EXPECT(attend(&ds, &t, q, kc, len, 100, out, ws, need - 1) == MOESPEC_ERR_WORKSPACE_TOO_SMALL);
  EXPECT(attend(&ds, &t, 0, kc, len, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q + 8, kc, len, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, 0, len, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, kc, 0, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, kc, len + 2, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, kc, len, 101, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, kc, len, -1, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, kc, len, 100, 0, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, kc, len, 100, out, 0, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, &t, q, kc, len, 100, out, ws + 16, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(NULL, &t, q, kc, len, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(attend(&ds, NULL, q, kc, len, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  const int bad[][3] = {{0, 16, 8}, {2, 0, 8}, {2, 16, 0}, {2, 16, 17}, {65536, 16, 8}, {2, 65536, 8}, {-1, -1, -1}};
  for (size_t i = 0; i < sizeof bad / sizeof bad[0]; ++i) {
    moespec_tree b = make_tree(bad[i][0], bad[i][1], bad[i][2]);
    EXPECT(attend(&ds, &b, q, kc, len, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  }
  moespec_tree b = t;
  b.tree_off = NULL; /* only one sequence does without offsets */
  EXPECT(attend(&ds, &b, q, kc, len, 100, out, ws, need) == MOESPEC_ERR_INVALID_ARG);
  const int64_t strides[] = {511, 513, -8, ((int64_t)1 << 20) + 8, INT64_MAX, INT64_MIN};
  for (size_t i = 0; i < sizeof strides / sizeof strides[0]; ++i) {
    b = t;
    b.q_stride = strides[i];
    EXPECT(attend(&ds, &b, q, kc, len, 100, out, ws, need) != MOESPEC_OK);
    b = t;
    b.kv_stride = strides[i] == 511 ? 127 : strides[i];
    EXPECT(attend(&ds, &b, q, kc, len, 100, out, ws, need) != MOESPEC_OK);
  }
}

static void weight_arguments(void) {
  moespec_attn_desc ds = make_desc(8, 2, 64, 100, MOESPEC_BF16);
  moespec_tree t = make_tree(2, 16, 8);
  const size_t need = moespec_attn_workspace_bytes(&ds, 2, 16, 8, 100);
  void *p = fake(0x10000), *ws = fake(0x70000);
  EXPECT(moespec_cache_weights(&ds, &t, p, p, p, p, 100, p, NULL, 1.f, NULL, p, NULL, ws, need - 1, NULL) ==
         MOESPEC_ERR_WORKSPACE_TOO_SMALL);
  EXPECT(moespec_cache_weights(&ds, &t, p, p, p, p, 100, NULL, NULL, 1.f, NULL, p, NULL, ws, need, NULL) ==
         MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_weights(&ds, &t, p, p, p, p, 100, p, NULL, NAN, NULL, p, NULL, ws, need, NULL) ==
         MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_weights(&ds, &t, p, p, p, p, 100, p, NULL, 1.f, NULL, NULL, p, ws, need, NULL) ==
         MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_weights(&ds, &t, p, p, NULL, p, 100, p, NULL, 1.f, NULL, p, p, ws, need, NULL) ==
         MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_weights(&ds, &t, p, p, p, p, 100, p, fake(0x10002), 1.f, NULL, p, p, ws, need, NULL) ==
         MOESPEC_ERR_INVALID_ARG);
}

static void cache_arguments(void) {
  moespec_attn_desc ds = make_desc(8, 2, 64, 100, MOESPEC_BF16);
  moespec_tree t = make_tree(2, 16, 8);
  int32_t *p = fake(0x10000), *l = fake(0x20000);
  float *w = fake(0x30000);
  EXPECT(moespec_cache_commit(&ds, 0, &t, p, p, NULL, p, l, 4, p, p, NULL, l, p, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_commit(&ds, 1, &t, p, p, NULL, p, l, 0, p, p, NULL, l, p, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_commit(&ds, 1, &t, p, p, w, p, l, 4, p, p, NULL, l, p, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_commit(&ds, 1, &t, p, p, NULL, p, p, 4, p, p, NULL, l, l, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_commit(&ds, 1, &t, p, p, NULL, p, l, 4, p, p, NULL, p, l, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_commit(&ds, 1, &t, p, NULL, NULL, p, l, 4, p, p, NULL, l, p, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_commit(&ds, 1, &t, p, p, NULL, NULL, l, 4, p, p, NULL, l, p, NULL) == MOESPEC_ERR_INVALID_ARG);
  moespec_tree b = make_tree(65535, 65535, 1);
  EXPECT(moespec_cache_commit(&ds, 4096, &b, p, p, NULL, p, l, 65535, p, p, NULL, l, p, NULL) == MOESPEC_ERR_UNSUPPORTED_SHAPE);

  int32_t *ko = fake(0x40000), *vo = fake(0x50000), *ws = fake(0x70000);
  float *wo = fake(0x60000);
  int32_t *v = fake(0x80000);
  const size_t need = moespec_evict_workspace_bytes(&ds, 1, 2, 50);
  EXPECT(need >= 2 * 2 * 50 * 4);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, 50, 10, 50, ko, vo, wo, NULL, NULL, ws, need - 1, NULL) ==
         MOESPEC_ERR_WORKSPACE_TOO_SMALL);
  const int bad[][3] = {{0, 0, 50}, {50, 51, 50}, {50, -1, 50}, {51, 10, 50}, {-1, -1, -1}};
  for (size_t i = 0; i < sizeof bad / sizeof bad[0]; ++i)
    EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, bad[i][0], bad[i][1], bad[i][2], ko, vo, wo, NULL, NULL, ws, need, NULL) ==
           MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, 50, 10, 50, p, vo, wo, NULL, NULL, ws, need, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, 50, 10, 50, ko, ko, wo, NULL, NULL, ws, need, NULL) ==
         MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, 50, 10, 50, ko, vo, w, NULL, NULL, ws, need, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, 50, 10, 50, ko, vo, wo, NULL, l, ws, need, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, 50, 10, 50, ko, vo, wo, l, NULL, ws, need, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, w, l, 50, 10, 50, ko, vo, wo, p, p, ws, need, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_cache_evict(&ds, 1, 2, p, v, NULL, l, 50, 10, 50, ko, vo, wo, NULL, NULL, ws, need, NULL) ==
         MOESPEC_ERR_INVALID_ARG);
}

static void norm_arguments(void) {
  moespec_desc ds;
  memset(&ds, 0, sizeof ds);
  ds.d = 256;
  ds.n_experts = ds.top_k = 1;
  ds.d_ff = 256;
  ds.dtype = MOESPEC_BF16;
  moespec_block b;
  memset(&b, 0, sizeof b);
  b.scale = 1.f;
  void *y = fake(0x10000), *r = fake(0x20000), *x = fake(0x30000), *odd = fake(0x30008);
  EXPECT(moespec_block_norm(&ds, NULL, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_block_norm(&ds, &b, NULL, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 0, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 70000, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, NULL, NULL, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, r, r, NULL) == MOESPEC_ERR_INVALID_ARG);
  EXPECT(moespec_block_norm(&ds, &b, y, odd, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  const moespec_block ok = b;
  b.gate_kind = MOESPEC_BLOCK_GATE_TOKEN; /* a kind without a gate */
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  b = ok;
  b.gate = y; /* a gate without a kind */
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  b = ok;
  b.w_post = y; /* a weight of a norm that is not wanted */
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  b = ok;
  b.gate_kind = 4;
  b.gate = y;
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  const float eps[] = {-1.f, NAN, INFINITY};
  for (size_t i = 0; i < 3; ++i) {
    b = ok;
    b.eps = eps[i];
    EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  }
  b = ok;
  b.scale = NAN;
  EXPECT(moespec_block_norm(&ds, &b, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_INVALID_ARG);
  ds.d = 250;
  EXPECT(moespec_block_norm(&ds, &ok, y, NULL, 4, r, x, NULL) == MOESPEC_ERR_UNSUPPORTED_SHAPE);
}

int main(void) {
  descriptors_and_workspaces();
  attention_arguments();
  weight_arguments();
  cache_arguments();
  norm_arguments();
  if (failures) {
    fprintf(stderr, "%d host checks failed\n", failures);
    return 1;
  }
  printf("host checks passed\n");
  return 0;
}
