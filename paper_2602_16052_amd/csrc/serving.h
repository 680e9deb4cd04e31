// What the kernels around a serving step share: sequences of token rows, pages of a cache, 8-bit codes.
#pragma once

#include <float.h>

#include "attention.h"

namespace moespec {

// The sequence that owns a token row (the number of sequences that end at or in front of it), the same in every lane of a wave; n_seq
// for rows of none.  One trip to memory for every 64 sequences, in each wave: right for some hundreds.  (Rotation of one token of each of 256 sequences 4.5
// us, of 4096 31, of 65535 5522; the same tokens as one sequence with given places 5.0, 6.8 and 86.)
__device__ __forceinline__ int seq_of_row(const int32_t *tree_off, int n_seq, int row) {
  if (!tree_off) return 0;
  const int lane = threadIdx.x & 63;
  int s = 0;
  for (int base = 0; base < n_seq; base += kWave) {
    const int i = base + lane;
    s += __popcll(__ballot(i < n_seq && tree_off[min(i, n_seq - 1) + 1] <= row));
  }
  return s;
}

// First row and rows of sequence s, clamped to what the buffers hold.
struct SeqRows {
  int row0, T;
};
__device__ __forceinline__ SeqRows seq_rows(const int32_t *tree_off, int s, int M, int max_tree) {
  SeqRows g{0, M};
  if (tree_off) {
    g.row0 = min(max(tree_off[s], 0), M);
    g.T = min(max(tree_off[s + 1], g.row0), M) - g.row0;
  }
  g.T = min(g.T, max_tree);
  return g;
}

// Pages of n_layers layers.  log_page: page_size is 2^log_page.
struct Pages {
  const unsigned char *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *table;
  int n_pages, max_pages, log_page, Hk;
  __device__ __forceinline__ int64_t entries() const { return (int64_t)max_pages << log_page; }
  // Page of entry e (< entries()) of sequence s, -1 if it is outside of the pool.
  __device__ __forceinline__ int page_of(int s, int64_t e) const {
    const int p = table[(int64_t)s * max_pages + (e >> log_page)];
    return p >= 0 && p < n_pages ? p : -1;
  }
  // Row (of D elements) of entry e in page p.
  __device__ __forceinline__ int64_t row(int layer, int p, int hk, int64_t e) const {
    return ((((int64_t)layer * n_pages + p) * Hk + hk) << log_page) + (e & ((1 << log_page) - 1));
  }
};

inline Pages pages_of(const moespec_attn_desc &ds, const moespec_paged_cache &c) {
  return Pages{static_cast<const unsigned char *>(c.k_pages), static_cast<const unsigned char *>(c.v_pages), c.k_scale, c.v_scale,
               c.page_table, c.n_pages, c.max_pages, __builtin_ctz(c.page_size), ds.n_kv_heads};
}

hipError_t launch_head_rope(const moespec_attn_desc &ds, const moespec_rope &rope, const moespec_tree &tree, const void *q,
                            const void *k, void *q_out, void *k_out, hipStream_t st);
hipError_t launch_paged_write(const moespec_attn_desc &ds, int n_layers, const moespec_paged_cache &cache, const moespec_tree &tree,
                              const void *k_tree, const void *v_tree, const int32_t *path, const int32_t *n_path, int max_path,
                              const int32_t *cache_len, int32_t *new_len, hipStream_t st);
hipError_t launch_paged_read(const moespec_attn_desc &ds, int n_layers, int n_seq, const moespec_paged_cache &cache,
                             const int32_t *first, const int32_t *cache_len, int max_len, void *k_cache, void *v_cache,
                             hipStream_t st);
size_t paged_attention_ws(const moespec_attn_desc &ds, const moespec_paged_cache &cache, int n_seq, int max_len);
hipError_t launch_paged_attention(const moespec_attn_desc &ds, const moespec_paged_cache &cache, int n_seq, const void *q,
                                  int64_t q_stride, const int32_t *cache_len, int max_len, void *out, float *lse, void *ws,
                                  hipStream_t st);
constexpr int kMaxVerifyTree = 2048;  // rows of a tree that the walk holds in LDS
constexpr int kVerifyChunk = 2048;    // logits of a wave
constexpr int kVerifyGroups = 32;     // workgroups of 1024 threads a sequence, at most, that sum p - q (sampled drafts)
size_t draft_verify_ws(const moespec_verify &v, int n_seq, int M);
hipError_t launch_draft_verify(const moespec_verify &v, const moespec_tree &tree, const int32_t *tokens, const double *u_accept,
                               const double *u_sample, int32_t *path, int32_t *n_path, int max_path, int32_t *next_token,
                               float *accepted, void *ws, hipStream_t st);

}  // namespace moespec
