/* Host-side exercise of the calls around a serving step for sanitizer builds, in plain C.  Every call here must be answered by argument
 * checks and workspace sizing alone, before any device work; device pointers are made up. */
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

#define INVALID MOESPEC_ERR_INVALID_ARG
#define UNSUPPORTED MOESPEC_ERR_UNSUPPORTED_SHAPE

static void *fake(uintptr_t a) { return (void *)(a << 32); } /* buffers 4 GB apart */

static moespec_attn_desc make_desc(int h, int hk, int d, int dtype) {
  moespec_attn_desc ds = {h, hk, d, 4096, dtype, 0.125f};
  return ds;
}
static moespec_tree make_tree(int n_seq, int M, int max_tree) {
  moespec_tree t;
  memset(&t, 0, sizeof t);
  t.n_seq = n_seq;
  t.n_tokens = M;
  t.max_tree = max_tree;
  t.tree_off = fake(90);
  return t;
}
static moespec_paged_cache make_cache(int code) {
  moespec_paged_cache c;
  memset(&c, 0, sizeof c);
  c.code = code;
  c.n_pages = 64;
  c.page_size = 32;
  c.max_pages = 16;
  c.k_pages = fake(10);
  c.v_pages = fake(11);
  if (code != MOESPEC_CACHE_PLAIN) {
    c.k_scale = fake(12);
    c.v_scale = fake(13);
  }
  c.page_table = fake(14);
  return c;
}

static void rope_arguments(void) {
  moespec_attn_desc ds = make_desc(8, 2, 64, MOESPEC_BF16);
  moespec_tree t = make_tree(2, 16, 8);
  moespec_rope base, r;
  memset(&base, 0, sizeof base);
  base.rot_dim = 64;
  base.norm = 1;
  base.eps = 1e-6f;
  base.freq = fake(20);
  base.cache_len = fake(21);
#define ROPE(q, k, qo, ko) moespec_head_rope(&ds, &r, &t, q, k, qo, ko, NULL)
  r = base;
  EXPECT(moespec_head_rope(NULL, &r, &t, fake(1), fake(2), fake(3), fake(4), NULL) == INVALID);
  EXPECT(moespec_head_rope(&ds, NULL, &t, fake(1), fake(2), fake(3), fake(4), NULL) == INVALID);
  EXPECT(moespec_head_rope(&ds, &r, NULL, fake(1), fake(2), fake(3), fake(4), NULL) == INVALID);
  EXPECT(ROPE(NULL, NULL, NULL, NULL) == INVALID);
  EXPECT(ROPE(fake(1), NULL, NULL, NULL) == INVALID);
  EXPECT(ROPE(NULL, fake(2), fake(3), fake(4)) == INVALID);
  EXPECT(ROPE((char *)fake(1) + 8, fake(2), fake(3), fake(4)) == INVALID);
  EXPECT(ROPE(fake(1), fake(2), fake(3), (char *)fake(4) + 2) == INVALID);
#define BAD(change, status)                                        \
  do {                                                             \
    r = base;                                                      \
    change;                                                        \
    EXPECT(ROPE(fake(1), fake(2), fake(3), fake(4)) == (status));  \
  } while (0)
  BAD(r.rot_dim = 24, UNSUPPORTED);
  BAD(r.rot_dim = 80, INVALID);
  BAD(r.rot_dim = -16, INVALID);
  BAD(r.rot_dim = 0, INVALID); /* with frequencies */
  BAD(r.freq = NULL, INVALID);
  BAD(r.interleaved = 2, INVALID);
  BAD(r.norm = -1, INVALID);
  BAD(r.eps = -1.f, INVALID);
  BAD(r.eps = NAN, INVALID);
  BAD(r.eps = INFINITY, INVALID);
  BAD((r.norm = 0, r.w_q = fake(5)), INVALID);
  BAD(r.positions = fake(6), INVALID); /* beside cache_len */
  BAD(r.w_k = (char *)fake(5) + 4, INVALID);
  BAD(r.q_out_stride = 8, INVALID);
  BAD(r.q_out_stride = 513, INVALID);
  BAD(r.k_out_stride = 1 << 21, UNSUPPORTED);
  BAD(r.k_out_stride = -8, INVALID);
  t.q_stride = 511;
  BAD((void)0, INVALID);
  t.q_stride = 0;
  t.max_tree = 17;
  BAD((void)0, INVALID);
  t.max_tree = 8;
  /* outputs on something else that the call uses; rows between each other's are fine, which a call that launches shows */
  r = base;
  EXPECT(ROPE(fake(1), fake(2), fake(3), fake(3)) == INVALID);
  EXPECT(ROPE(fake(1), fake(2), fake(2), fake(4)) == INVALID);
  EXPECT(ROPE(fake(1), fake(2), (char *)fake(1) + 16, fake(4)) == INVALID);
  EXPECT(ROPE(fake(1), fake(2), (char *)fake(1) + 1024, fake(4)) == INVALID);
  EXPECT(ROPE(fake(1), fake(2), fake(90), fake(4)) == INVALID);
  EXPECT(ROPE(fake(1), fake(2), fake(20), fake(4)) == INVALID);
  EXPECT(ROPE(fake(1), fake(2), fake(3), fake(21)) == INVALID);
  t.q_stride = t.kv_stride = r.q_out_stride = r.k_out_stride = 12 * 64; /* one projection: heads of q, k, v in a row */
  EXPECT(ROPE(fake(1), (char *)fake(1) + 1024, fake(1), (char *)fake(1) + 1024 - 128) == INVALID);
  EXPECT(ROPE(fake(1), (char *)fake(1) + 1024, (char *)fake(1) + 512, (char *)fake(1) + 1024) == INVALID);
  r.q_out_stride = 0;
  EXPECT(ROPE(fake(1), (char *)fake(1) + 1024, fake(1), (char *)fake(1) + 1024) == INVALID); /* the same place, other strides */
#undef BAD
}

static void paged_arguments(void) {
  moespec_attn_desc ds = make_desc(8, 2, 64, MOESPEC_BF16);
  moespec_tree t = make_tree(2, 16, 8);
  const moespec_paged_cache base = make_cache(MOESPEC_CACHE_I8);
  moespec_paged_cache c = base;
#define WRITE(L, path, n_path, max_path, new_len) \
  moespec_paged_write(&ds, L, &c, &t, fake(1), fake(2), path, n_path, max_path, fake(5), new_len, NULL)
#define READ(L, n_seq, max_len, k, v) moespec_paged_read(&ds, L, n_seq, &c, NULL, fake(5), max_len, k, v, NULL)
#define ATTEND(n_seq, q, stride, max_len, out, lse, ws, bytes) \
  moespec_paged_attention(&ds, &c, n_seq, q, stride, fake(5), max_len, out, lse, ws, bytes, NULL)
#define BAD(change, status)                                                                                      \
  do {                                                                                                           \
    c = base;                                                                                                    \
    change;                                                                                                      \
    EXPECT(WRITE(1, NULL, NULL, 0, NULL) == (status));                                                           \
    EXPECT(READ(1, 2, 100, fake(3), fake(4)) == (status));                                                       \
    EXPECT(ATTEND(2, fake(3), 0, 100, fake(4), NULL, fake(6), 1 << 20) == (status));                             \
    EXPECT(moespec_paged_attention_workspace_bytes(&ds, &c, 2, 100) == 0);                                       \
  } while (0)
  BAD(c.code = 3, INVALID);
  BAD(c.code = -1, INVALID);
  BAD(c.n_pages = 0, INVALID);
  BAD(c.max_pages = 0, INVALID);
  BAD(c.page_size = 0, INVALID);
  BAD(c.page_size = 8, UNSUPPORTED);
  BAD(c.page_size = 48, UNSUPPORTED);
  BAD(c.page_size = 512, UNSUPPORTED);
  BAD(c.max_pages = 1 << 26, UNSUPPORTED);
  BAD(c.k_pages = NULL, INVALID);
  BAD(c.v_pages = (char *)fake(11) + 8, INVALID);
  BAD(c.k_scale = NULL, INVALID);
  BAD(c.v_scale = (float *)((char *)fake(13) + 4), INVALID);
  BAD(c.page_table = NULL, INVALID);
  BAD(c.code = MOESPEC_CACHE_PLAIN, INVALID); /* with scales */
  BAD(ds.head_dim = 80, UNSUPPORTED);
  ds.head_dim = 64;
  BAD(ds.dtype = 9, INVALID);
  ds.dtype = MOESPEC_BF16;
  c = base;
  EXPECT(moespec_paged_write(&ds, 1, NULL, &t, fake(1), fake(2), NULL, NULL, 0, fake(5), NULL, NULL) == INVALID);
  EXPECT(WRITE(0, NULL, NULL, 0, NULL) == INVALID);
  EXPECT(WRITE(4097, NULL, NULL, 0, NULL) == INVALID);
  EXPECT(WRITE(1, fake(7), NULL, 4, NULL) == INVALID);
  EXPECT(WRITE(1, NULL, fake(8), 4, NULL) == INVALID);
  EXPECT(WRITE(1, fake(7), fake(8), 0, NULL) == INVALID);
  EXPECT(WRITE(1, fake(7), fake(8), 65536, NULL) == INVALID);
  EXPECT(WRITE(1, NULL, NULL, 0, fake(5)) == INVALID);  /* new_len on cache_len */
  EXPECT(WRITE(1, NULL, NULL, 0, fake(14)) == INVALID); /* ... on the table */
  EXPECT(moespec_paged_write(&ds, 1, &c, &t, fake(10), fake(2), NULL, NULL, 0, fake(5), NULL, NULL) == INVALID); /* pages on their source */
  EXPECT(moespec_paged_write(&ds, 1, &c, &t, fake(1), fake(13), NULL, NULL, 0, fake(5), NULL, NULL) == INVALID);
  EXPECT(moespec_paged_write(&ds, 1, &c, &t, fake(1), NULL, NULL, NULL, 0, fake(5), NULL, NULL) == INVALID);
  EXPECT(moespec_paged_write(&ds, 1, &c, &t, fake(1), fake(2), NULL, NULL, 0, NULL, NULL, NULL) == INVALID);
  c.v_pages = c.k_pages;
  EXPECT(WRITE(1, NULL, NULL, 0, NULL) == INVALID);
  c = base;
  t.n_tokens = 65535;
  t.max_tree = 65535;
  t.n_seq = 65535;
  EXPECT(WRITE(1, NULL, NULL, 0, NULL) == UNSUPPORTED); /* threads of a launch */
  EXPECT(READ(1, 2, -1, fake(3), fake(4)) == INVALID);
  EXPECT(READ(1, 2, 513, fake(3), fake(4)) == INVALID); /* the table has room for 512 */
  ds.capacity = 99;
  EXPECT(READ(1, 2, 100, fake(3), fake(4)) == INVALID);
  ds.capacity = 4096;
  EXPECT(READ(1, 0, 100, fake(3), fake(4)) == INVALID);
  EXPECT(READ(1, 65536, 100, fake(3), fake(4)) == INVALID);
  EXPECT(READ(4096, 65535, 512, fake(3), fake(4000)) == UNSUPPORTED);
  EXPECT(READ(1, 2, 100, fake(3), fake(3)) == INVALID);
  EXPECT(READ(1, 2, 100, fake(10), fake(4)) == INVALID);
  EXPECT(READ(1, 2, 100, fake(3), fake(12)) == INVALID);
  EXPECT(READ(1, 2, 100, NULL, fake(4)) == INVALID);
  const size_t need = moespec_paged_attention_workspace_bytes(&ds, &c, 2, 512);
  EXPECT(need > 0);
  EXPECT(ATTEND(2, NULL, 0, 512, fake(4), NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 512, NULL, NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 513, fake(4), NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), -1, 512, fake(4), NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 511, 512, fake(4), NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 516, 512, fake(4), NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 1 << 21, 512, fake(4), NULL, fake(6), need) == UNSUPPORTED);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(4), NULL, fake(6), need - 1) == MOESPEC_ERR_WORKSPACE_TOO_SMALL);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(4), NULL, (char *)fake(6) + 16, need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(4), NULL, NULL, need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(3), NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(4), fake(4), fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(11), NULL, fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(4), fake(14), fake(6), need) == INVALID);
  EXPECT(ATTEND(2, fake(3), 0, 512, fake(4), fake(6), fake(6), need) == INVALID);
  EXPECT(ATTEND(0, fake(3), 0, 512, fake(4), NULL, fake(6), need) == INVALID);
#undef BAD
}

static void workspaces_grow_with_the_call(void) {
  const int heads[][2] = {{32, 4}, {32, 8}, {8, 8}, {64, 1}, {1024, 1024}, {1024, 1}};
  for (int i = 0; i < 6; ++i)
    for (int dt = MOESPEC_F32; dt <= MOESPEC_BF16; ++dt)
      for (int code = MOESPEC_CACHE_PLAIN; code <= MOESPEC_CACHE_E4M3; ++code) {
        moespec_attn_desc ds = make_desc(heads[i][0], heads[i][1], 128, dt);
        moespec_paged_cache c = make_cache(code);
        c.max_pages = 1 << 16;
        for (int s = 1; s <= 4096; s = s * 3 / 2 + 1) {
          size_t prev = 0;
          for (int len = 0; len <= 1 << 20; len = len * 2 + 7) {
            const size_t w = moespec_paged_attention_workspace_bytes(&ds, &c, s, len);
            EXPECT(w > 0 && w >= prev && moespec_paged_attention_workspace_bytes(&ds, &c, s + 1, len) >= w);
            prev = w;
          }
        }
        const int32_t big[] = {1, 65535, 65536, INT32_MAX, -1, 0, INT32_MIN};
        for (int a = 0; a < 7; ++a)
          for (int b = 0; b < 7; ++b) (void)moespec_paged_attention_workspace_bytes(&ds, &c, big[a], big[b]);
      }
}

static void verify_arguments(void) {
  moespec_verify base, v;
  memset(&base, 0, sizeof base);
  base.vocab = 1000;
  base.dtype = MOESPEC_BF16;
  base.logits = fake(1);
  moespec_tree t = make_tree(2, 16, 8);
  size_t need = moespec_verify_workspace_bytes(&base, 2, 16);
  EXPECT(need > 0);
#define VERIFY(max_path, path, token, accepted, ws, bytes) \
  moespec_draft_verify(&v, &t, fake(2), fake(3), fake(4), path, fake(6), max_path, token, accepted, ws, bytes, NULL)
#define BAD(change, status)                                                                 \
  do {                                                                                      \
    v = base;                                                                               \
    change;                                                                                 \
    EXPECT(VERIFY(8, fake(5), fake(7), NULL, fake(8), 1 << 20) == (status));                \
  } while (0)
  EXPECT(moespec_draft_verify(NULL, &t, fake(2), fake(3), fake(4), fake(5), fake(6), 8, fake(7), NULL, fake(8), need, NULL) == INVALID);
  BAD(v.vocab = 1, INVALID);
  BAD(v.vocab = (1 << 24) + 1, INVALID);
  BAD(v.dtype = 2, INVALID);
  BAD(v.logit_stride = 999, INVALID);
  BAD(v.logit_stride = (int64_t)1 << 40, UNSUPPORTED);
  BAD(v.draft_stride = -1, INVALID);
  BAD(v.logits = NULL, INVALID);
  BAD(v.logits = (char *)fake(1) + 2, INVALID);
  BAD(v.draft_logits = (char *)fake(9) + 4, INVALID);
  BAD(v.temperature = (float *)((char *)fake(9) + 2), INVALID);
  t.tree_mask = fake(91);
  BAD(v.draft_logits = fake(9), INVALID); /* sampled drafts in a tree */
  t.tree_mask = NULL;
  t.tree_off = NULL;
  BAD((void)0, INVALID);
  t = make_tree(2, 65535, 2049);
  BAD((void)0, UNSUPPORTED);
  t = make_tree(2, 16, 17);
  BAD((void)0, INVALID);
  t = make_tree(2, 16, 8);
  v = base;
  EXPECT(VERIFY(0, fake(5), fake(7), NULL, fake(8), need) == INVALID);
  EXPECT(VERIFY(8, NULL, fake(7), NULL, fake(8), need) == INVALID);
  EXPECT(VERIFY(8, fake(5), NULL, NULL, fake(8), need) == INVALID);
  EXPECT(VERIFY(8, fake(5), fake(7), NULL, fake(8), need - 1) == MOESPEC_ERR_WORKSPACE_TOO_SMALL);
  EXPECT(VERIFY(8, fake(5), fake(7), NULL, NULL, need) == INVALID);
  EXPECT(VERIFY(8, fake(5), fake(5), NULL, fake(8), need) == INVALID);
  EXPECT(VERIFY(8, fake(1), fake(7), NULL, fake(8), need) == INVALID);
  EXPECT(VERIFY(8, fake(5), fake(7), fake(3), fake(8), need) == INVALID);
  EXPECT(VERIFY(8, fake(5), fake(2), NULL, fake(8), need) == INVALID);
  EXPECT(VERIFY(8, fake(5), fake(4), NULL, fake(8), need) == INVALID);
  EXPECT(VERIFY(8, fake(5), fake(90), NULL, fake(8), need) == INVALID);
  EXPECT(moespec_draft_verify(&v, &t, NULL, fake(3), fake(4), fake(5), fake(6), 8, fake(7), NULL, fake(8), need, NULL) == INVALID);
  EXPECT(moespec_draft_verify(&v, &t, fake(2), (double *)((char *)fake(3) + 4), fake(4), fake(5), fake(6), 8, fake(7), NULL, fake(8), need,
                              NULL) == INVALID);
  v.draft_logits = fake(9);
  EXPECT(VERIFY(8, fake(5), fake(7), NULL, fake(8), need) == MOESPEC_ERR_WORKSPACE_TOO_SMALL); /* twice the rows */
  t = make_tree(1, 65535, 8);
  v.vocab = 1 << 24;
  EXPECT(VERIFY(8, fake(5), fake(7), NULL, fake(8), (size_t)1 << 50) == UNSUPPORTED); /* threads of a launch */
  size_t prev = 0;
  for (int m = 1; m < 60000; m = m * 2 + 1) {
    const size_t w = moespec_verify_workspace_bytes(&base, 1, m);
    EXPECT(w >= prev);
    prev = w;
  }
  EXPECT(moespec_verify_workspace_bytes(&base, 0, 8) == 0 && moespec_verify_workspace_bytes(&base, 1, 65536) == 0);
  EXPECT(moespec_verify_workspace_bytes(NULL, 1, 8) == 0);
}

int main(void) {
  rope_arguments();
  paged_arguments();
  workspaces_grow_with_the_call();
  verify_arguments();
  if (failures) return 1;
  printf("host checks passed\n");
  return 0;
}
