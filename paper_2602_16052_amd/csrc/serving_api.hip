// C ABI of the calls around a serving step (head norm and rotation, paged cache, verification): argument checks on the host, before any launch.
#include <math.h>

#include "call_checks.h"
#include "serving.h"

using namespace moespec;

namespace {

constexpr int kMostLayers = 4096;
constexpr int kMostVocab = 1 << 24;

bool aligned8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// Rows of `row` bytes, `stride` bytes apart.
struct RowSpan {
  const void *p;
  double n, stride, row;
};
// Whether two sets of rows share a byte.  Rows the same distance apart may lie between each other's (heads of queries, keys and values in
// one row of a projection).
bool rows_overlap(const RowSpan &a, const RowSpan &b) {
  const Span x{a.p, (a.n - 1) * a.stride + a.row}, y{b.p, (b.n - 1) * b.stride + b.row};
  if (!overlap(x, y)) return false;
  if (a.stride != b.stride) return true;
  const uint64_t stride = (uint64_t)a.stride, low = (uint64_t)reinterpret_cast<uintptr_t>(a.p), high = (uint64_t)reinterpret_cast<uintptr_t>(b.p);
  const uint64_t d = low <= high ? (high - low) % stride : (stride - (low - high) % stride) % stride;  // from a row of a to the next of b
  return (double)d < a.row || (double)(stride - d) < b.row;
}

// A pool of pages and its table.  Bytes of the pool's pages and of its scales.
struct PoolBytes {
  double pages, scales, table;
};
moespec_status check_cache(const moespec_attn_desc &ds, const moespec_paged_cache *c, int32_t n_layers, int32_t n_seq, PoolBytes *bytes) {
  if (!c || n_layers < 1 || n_layers > kMostLayers || n_seq < 1 || n_seq > kMost) return MOESPEC_ERR_INVALID_ARG;
  if (c->code < MOESPEC_CACHE_PLAIN || c->code > MOESPEC_CACHE_E4M3 || c->n_pages < 1 || c->max_pages < 1) return MOESPEC_ERR_INVALID_ARG;
  switch (c->page_size) {
    case 16: case 32: case 64: case 128: case 256: break;
    default: return c->page_size < 1 ? MOESPEC_ERR_INVALID_ARG : MOESPEC_ERR_UNSUPPORTED_SHAPE;
  }
  if ((int64_t)c->max_pages * c->page_size > kMaxEntries) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  if (!c->k_pages || !c->v_pages || !c->page_table || !aligned16(c->k_pages) || !aligned16(c->v_pages) || !aligned4(c->page_table))
    return MOESPEC_ERR_INVALID_ARG;
  const bool codes = c->code != MOESPEC_CACHE_PLAIN;
  if (codes != (c->k_scale != nullptr) || codes != (c->v_scale != nullptr) || !aligned16(c->k_scale) || !aligned16(c->v_scale))
    return MOESPEC_ERR_INVALID_ARG;
  const double rows = (double)n_layers * c->n_pages * ds.n_kv_heads * c->page_size;
  // row numbers and byte offsets are 64 bits; a pool beyond 2^50 rows is no pool
  if (rows > 1125899906842624.) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  *bytes = PoolBytes{rows * ds.head_dim * (codes ? 1. : elem_bytes(ds)), codes ? 4. * rows : 0., 4. * (double)n_seq * c->max_pages};
  return MOESPEC_OK;
}
int64_t entries_of(const moespec_paged_cache &c) { return (int64_t)c.max_pages * c.page_size; }
// Entries that a workgroup of 256 threads writes or reads.
int64_t rows_of_group(const moespec_attn_desc &ds) { return 256 / pow2_ceil(ds.head_dim * (int)elem_bytes(ds) / 16); }

moespec_status check_verify(const moespec_verify *v) {
  if (!v || (v->dtype != MOESPEC_F32 && v->dtype != MOESPEC_BF16) || v->vocab < 2 || v->vocab > kMostVocab) return MOESPEC_ERR_INVALID_ARG;
  for (const int64_t stride : {v->logit_stride, v->draft_stride}) {
    if (stride != 0 && stride < v->vocab) return MOESPEC_ERR_INVALID_ARG;
    if (stride > 2 * (int64_t)kMostVocab) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  }
  return MOESPEC_OK;
}

}  // namespace

extern "C" {

moespec_status moespec_head_rope(const moespec_attn_desc *desc, const moespec_rope *rope, const moespec_tree *tree, const void *q,
                                 const void *k, void *q_out, void *k_out, void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK || (s = check_tree(*desc, tree, 0, true)) != MOESPEC_OK) return s;
  if (!rope || (!q && !k) || (q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr)) return MOESPEC_ERR_INVALID_ARG;
  const moespec_rope &r = *rope;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(r.w_q) || !aligned16(r.w_k) ||
      !aligned4(r.freq) || !aligned4(r.positions) || !aligned4(r.cache_len))
    return MOESPEC_ERR_INVALID_ARG;
  if ((r.interleaved != 0 && r.interleaved != 1) || (r.norm != 0 && r.norm != 1) || !(r.eps >= 0.f) || !isfinite(r.eps) ||
      r.rot_dim < 0 || r.rot_dim > desc->head_dim || (r.rot_dim > 0) != (r.freq != nullptr))
    return MOESPEC_ERR_INVALID_ARG;
  if (r.rot_dim % 16 != 0) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  if (!r.norm && (r.w_q || r.w_k)) return MOESPEC_ERR_INVALID_ARG;
  if (r.positions && r.cache_len) return MOESPEC_ERR_INVALID_ARG;
  const double es = elem_bytes(*desc), M = tree->n_tokens, D = desc->head_dim;
  const int64_t qrow = (int64_t)desc->n_heads * desc->head_dim, krow = (int64_t)desc->n_kv_heads * desc->head_dim;
  for (const auto &x : {std::pair<int64_t, int64_t>{r.q_out_stride, qrow}, {r.k_out_stride, krow}}) {
    if (x.first > kMaxStride) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
    if (x.first != 0 && (x.first < x.second || x.first * (int64_t)es % 16 != 0)) return MOESPEC_ERR_INVALID_ARG;
  }
  const RowSpan in[2] = {{q, M, (tree->q_stride ? tree->q_stride : qrow) * es, qrow * es}, {k, M, (tree->kv_stride ? tree->kv_stride : krow) * es, krow * es}};
  const RowSpan out[2] = {{q_out, M, (r.q_out_stride ? r.q_out_stride : qrow) * es, qrow * es}, {k_out, M, (r.k_out_stride ? r.k_out_stride : krow) * es, krow * es}};
  const double words = (tree->max_tree + 31) / 32;
  if (rows_overlap(out[0], out[1])) return MOESPEC_ERR_INVALID_ARG;
  for (int o = 0; o < 2; ++o) {
    for (int i = 0; i < 2; ++i) {
      const bool in_place = o == i && out[o].p == in[i].p && out[o].stride == in[i].stride;
      if (!in_place && rows_overlap(out[o], in[i])) return MOESPEC_ERR_INVALID_ARG;
    }
    for (const Span &x : {Span{r.w_q, D * es}, Span{r.w_k, D * es}, Span{r.freq, 2. * r.rot_dim}, Span{r.positions, 4. * M},
                          Span{r.cache_len, 4. * tree->n_seq}, Span{tree->tree_off, 4. * (tree->n_seq + 1.)},
                          Span{r.positions ? nullptr : tree->tree_mask, 4. * M * words}})
      if (rows_overlap(out[o], RowSpan{x.p, 1., x.bytes, x.bytes})) return MOESPEC_ERR_INVALID_ARG;
  }
  return from_hip(launch_head_rope(*desc, r, *tree, q, k, q_out, k_out, static_cast<hipStream_t>(hip_stream)));
}

moespec_status moespec_paged_write(const moespec_attn_desc *desc, int32_t n_layers, const moespec_paged_cache *cache,
                                   const moespec_tree *tree, const void *k_tree, const void *v_tree, const int32_t *path,
                                   const int32_t *n_path, int32_t max_path, const int32_t *cache_len, int32_t *new_len,
                                   void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK || (s = check_tree(*desc, tree, 0, false)) != MOESPEC_OK) return s;
  PoolBytes pool;
  if ((s = check_cache(*desc, cache, n_layers, tree->n_seq, &pool)) != MOESPEC_OK) return s;
  if (!k_tree || !v_tree || !cache_len || !aligned16(k_tree) || !aligned16(v_tree) || !aligned4(path) || !aligned4(n_path) ||
      !aligned4(cache_len) || !aligned4(new_len))
    return MOESPEC_ERR_INVALID_ARG;
  if ((path == nullptr) != (n_path == nullptr) || (path && (max_path < 1 || max_path > kMost))) return MOESPEC_ERR_INVALID_ARG;
  const int64_t most = path ? max_path : tree->max_tree, rows = rows_of_group(*desc);
  if ((double)((most + rows - 1) / rows) * desc->n_kv_heads * tree->n_seq * n_layers * 256. > (double)kMaxThreads)
    return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const double es = elem_bytes(*desc), D = desc->head_dim, M = tree->n_tokens, n_seq = tree->n_seq, Hk = desc->n_kv_heads;
  const double kv = rows_bytes(n_layers * M, tree->kv_stride ? (double)tree->kv_stride : Hk * D, Hk * D, es);
  if (!apart({{cache->k_pages, pool.pages}, {cache->v_pages, pool.pages}, {cache->k_scale, pool.scales}, {cache->v_scale, pool.scales},
              {new_len, 4. * n_seq}},
             {{k_tree, kv}, {v_tree, kv}, {path, 4. * n_seq * most}, {n_path, 4. * n_seq}, {cache_len, 4. * n_seq},
              {cache->page_table, pool.table}, {tree->tree_off, 4. * (n_seq + 1.)}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_paged_write(*desc, n_layers, *cache, *tree, k_tree, v_tree, path, n_path, max_path, cache_len, new_len,
                                     static_cast<hipStream_t>(hip_stream)));
}

moespec_status moespec_paged_read(const moespec_attn_desc *desc, int32_t n_layers, int32_t n_seq,
                                  const moespec_paged_cache *cache, const int32_t *first, const int32_t *cache_len,
                                  int32_t max_len, void *k_cache, void *v_cache, void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK) return s;
  PoolBytes pool;
  if ((s = check_cache(*desc, cache, n_layers, n_seq, &pool)) != MOESPEC_OK) return s;
  if (!cache_len || !k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache) || !aligned4(first) || !aligned4(cache_len) ||
      max_len < 0 || max_len > desc->capacity || max_len > entries_of(*cache))
    return MOESPEC_ERR_INVALID_ARG;
  // a workgroup of 256 threads a head at least, several where there are few
  if ((double)desc->n_kv_heads * n_seq * n_layers * 256. + 4096. * 256. > (double)kMaxThreads) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const double dense = cache_entries(*desc, n_layers, n_seq) * desc->head_dim * elem_bytes(*desc);
  if (!apart({{k_cache, dense}, {v_cache, dense}},
             {{cache->k_pages, pool.pages}, {cache->v_pages, pool.pages}, {cache->k_scale, pool.scales}, {cache->v_scale, pool.scales},
              {cache->page_table, pool.table}, {first, 4. * n_seq}, {cache_len, 4. * n_seq}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_paged_read(*desc, n_layers, n_seq, *cache, first, cache_len, max_len, k_cache, v_cache,
                                    static_cast<hipStream_t>(hip_stream)));
}

size_t moespec_paged_attention_workspace_bytes(const moespec_attn_desc *desc, const moespec_paged_cache *cache, int32_t n_seq,
                                               int32_t max_len) {
  PoolBytes pool;
  if (check_desc(desc) != MOESPEC_OK || check_cache(*desc, cache, 1, n_seq, &pool) != MOESPEC_OK || max_len < 0 || max_len > entries_of(*cache)) return 0;
  return paged_attention_ws(*desc, *cache, n_seq, max_len);
}

moespec_status moespec_paged_attention(const moespec_attn_desc *desc, const moespec_paged_cache *cache, int32_t n_seq,
                                       const void *q, int64_t q_stride, const int32_t *cache_len, int32_t max_len, void *out,
                                       float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK) return s;
  PoolBytes pool;
  if ((s = check_cache(*desc, cache, 1, n_seq, &pool)) != MOESPEC_OK) return s;
  const double es = elem_bytes(*desc), row = (double)desc->n_heads * desc->head_dim;
  if (!q || !out || !cache_len || !aligned16(q) || !aligned16(out) || !aligned4(lse) || !aligned4(cache_len) || max_len < 0 ||
      max_len > entries_of(*cache) || q_stride < 0 || (q_stride > 0 && ((double)q_stride < row || q_stride * (int64_t)es % 16 != 0)))
    return MOESPEC_ERR_INVALID_ARG;
  if (q_stride > kMaxStride) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const size_t need = paged_attention_ws(*desc, *cache, n_seq, max_len);
  if ((s = check_ws(ws, ws_bytes, need)) != MOESPEC_OK) return s;
  const int64_t tiles = (desc->n_heads / desc->n_kv_heads + 15) / 16;
  if (((int64_t)n_seq * desc->n_kv_heads + 7 + 1024) * tiles * 256 > kMaxThreads) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  if (!apart({{out, n_seq * row * es}, {lse, 4. * n_seq * desc->n_heads}, {ws, (double)need}},
             {{q, rows_bytes(n_seq, q_stride ? (double)q_stride : row, row, es)}, {cache_len, 4. * n_seq}, {cache->k_pages, pool.pages},
              {cache->v_pages, pool.pages}, {cache->k_scale, pool.scales}, {cache->v_scale, pool.scales}, {cache->page_table, pool.table}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_paged_attention(*desc, *cache, n_seq, q, q_stride, cache_len, max_len, out, lse, ws,
                                         static_cast<hipStream_t>(hip_stream)));
}

size_t moespec_verify_workspace_bytes(const moespec_verify *verify, int32_t n_seq, int32_t M_max) {
  if (check_verify(verify) != MOESPEC_OK || n_seq < 1 || n_seq > kMost || M_max < 1 || M_max > kMost) return 0;
  return draft_verify_ws(*verify, n_seq, M_max);
}

moespec_status moespec_draft_verify(const moespec_verify *verify, const moespec_tree *tree, const int32_t *tokens,
                                    const double *u_accept, const double *u_sample, int32_t *path, int32_t *n_path,
                                    int32_t max_path, int32_t *next_token, float *accepted, void *ws, size_t ws_bytes,
                                    void *hip_stream) {
  moespec_status s = check_verify(verify);
  if (s != MOESPEC_OK) return s;
  const moespec_verify &v = *verify;
  if (!tree || tree->n_seq < 1 || tree->n_seq > kMost || tree->n_tokens < 1 || tree->n_tokens > kMost || tree->max_tree < 1 ||
      tree->max_tree > tree->n_tokens || (!tree->tree_off && tree->n_seq != 1) || !aligned4(tree->tree_off) || !aligned4(tree->tree_mask))
    return MOESPEC_ERR_INVALID_ARG;
  if (tree->max_tree > kMaxVerifyTree) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  if (!v.logits || !aligned16(v.logits) || !aligned16(v.draft_logits) || !aligned4(v.temperature) || !tokens || !aligned4(tokens) ||
      !u_accept || !u_sample || !aligned8(u_accept) || !aligned8(u_sample) || !path || !n_path || !next_token || !aligned4(path) ||
      !aligned4(n_path) || !aligned4(next_token) || !aligned4(accepted) || max_path < 1 || max_path > kMost)
    return MOESPEC_ERR_INVALID_ARG;
  if (v.draft_logits && tree->tree_mask) return MOESPEC_ERR_INVALID_ARG;  // sampled drafts: chains
  const size_t need = draft_verify_ws(v, tree->n_seq, tree->n_tokens);
  if ((s = check_ws(ws, ws_bytes, need)) != MOESPEC_OK) return s;
  const double M = tree->n_tokens, n_seq = tree->n_seq, es = v.dtype == MOESPEC_BF16 ? 2 : 4;
  if (M * ((v.vocab + kVerifyChunk - 1) / kVerifyChunk) * (v.draft_logits ? 2 : 1) * 64. + M * 2 * 192. > (double)kMaxThreads ||
      n_seq * kVerifyGroups * 1024. > (double)kMaxThreads)
    return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const double words = (tree->max_tree + 31) / 32;
  if (!apart({{path, 4. * n_seq * max_path}, {n_path, 4. * n_seq}, {next_token, 4. * n_seq}, {accepted, 4. * M}, {ws, (double)need}},
             {{v.logits, rows_bytes(M, v.logit_stride ? (double)v.logit_stride : v.vocab, v.vocab, es)},
              {v.draft_logits, rows_bytes(M, v.draft_stride ? (double)v.draft_stride : v.vocab, v.vocab, es)},
              {v.temperature, 4. * n_seq}, {tokens, 4. * M}, {u_accept, 8. * M}, {u_sample, 8. * n_seq},
              {tree->tree_off, 4. * (n_seq + 1.)}, {tree->tree_mask, 4. * M * words}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_draft_verify(v, *tree, tokens, u_accept, u_sample, path, n_path, max_path, next_token, accepted, ws,
                                      static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
