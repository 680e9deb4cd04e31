// C ABI of the calls around a verification step's attention: argument checks on the host, before any launch.
#include <float.h>
#include <math.h>

#include "call_checks.h"

using namespace moespec;

namespace {

KeyArgs key_args(const moespec_attn_desc &ds, const moespec_tree &t, const void *q, const void *k_tree, const void *v_tree,
                 const void *k_cache, const void *v_cache, const int32_t *cache_len, int32_t max_len) {
  KeyArgs a{};
  a.q = q;
  a.k_tree = k_tree;
  a.v_tree = v_tree;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.cache_len = cache_len;
  a.tree_off = t.tree_off;
  a.tree_mask = t.tree_mask;
  a.q_stride = t.q_stride ? t.q_stride : (int64_t)ds.n_heads * ds.head_dim;
  a.kv_stride = t.kv_stride ? t.kv_stride : (int64_t)ds.n_kv_heads * ds.head_dim;
  a.capacity = ds.capacity;
  a.n_seq = t.n_seq;
  a.M = t.n_tokens;
  a.max_tree = t.max_tree;
  a.words = (t.max_tree + 31) / 32;
  a.max_len = max_len;
  a.H = ds.n_heads;
  a.Hk = ds.n_kv_heads;
  a.G = ds.n_heads / ds.n_kv_heads;
  a.c = (float)((double)ds.scale * 1.4426950408889634);
  const double u = a.c >= FLT_MIN ? (double)a.c / ds.scale : 1.4426950408889634;  // (a c without all of its bits says nothing)
  a.u = (float)u;
  a.u_rest = (float)(u - a.u);
  return a;
}

size_t attn_ws(const moespec_attn_desc &ds, int64_t n_seq, int64_t max_tree, int64_t max_len) {
  const size_t a = tree_attention_ws(ds, n_seq, max_tree, max_len), b = cache_weights_ws(ds, n_seq, max_tree, max_len);
  return a > b ? a : b;
}

}  // namespace

extern "C" {

moespec_status moespec_check_attn_desc(const moespec_attn_desc *desc) { return check_desc(desc); }

size_t moespec_attn_workspace_bytes(const moespec_attn_desc *desc, int32_t n_seq, int32_t M_max, int32_t max_tree,
                                    int32_t max_len) {
  if (check_desc(desc) != MOESPEC_OK || !batch_ok(*desc, n_seq, M_max, max_tree, max_len)) return 0;
  return attn_ws(*desc, n_seq, max_tree, max_len);
}

moespec_status moespec_tree_attention(const moespec_attn_desc *desc, const moespec_tree *tree, const void *q,
                                      const void *k_tree, const void *v_tree, const void *k_cache, const void *v_cache,
                                      const int32_t *cache_len, int32_t max_len, void *out, float *lse, void *ws,
                                      size_t ws_bytes, void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK || (s = check_tree(*desc, tree, max_len, true)) != MOESPEC_OK) return s;
  if (!q || !k_tree || !v_tree || !out || !aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(out) ||
      !aligned4(lse))
    return MOESPEC_ERR_INVALID_ARG;
  if (max_len > 0 && (!k_cache || !v_cache || !cache_len || !aligned16(k_cache) || !aligned16(v_cache) || !aligned4(cache_len)))
    return MOESPEC_ERR_INVALID_ARG;
  const size_t need = attn_ws(*desc, tree->n_seq, tree->max_tree, max_len);
  if ((s = check_ws(ws, ws_bytes, need)) != MOESPEC_OK) return s;
  // workgroups of 256 threads: row tiles of 128 rows or more above 64 rows, parts only where there are few, up to seven more groups
  const int64_t rows = (int64_t)tree->max_tree * (desc->n_heads / desc->n_kv_heads), tiles = rows <= 64 ? 1 : (rows + 127) / 128;
  if ((((int64_t)tree->n_seq * desc->n_kv_heads + 7) * tiles + 1024) * 256 > kMaxThreads) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const KeyArgs a = key_args(*desc, *tree, q, k_tree, v_tree, k_cache, v_cache, cache_len, max_len);
  const double M = a.M, es = elem_bytes(*desc), kv = rows_bytes(M, a.kv_stride, (double)a.Hk * desc->head_dim, es);
  const double cache = max_len > 0 ? cache_entries(*desc, 1, a.n_seq) * desc->head_dim * es : 0.;
  if (!apart({{out, M * a.H * desc->head_dim * es}, {lse, 4. * M * a.H}, {ws, (double)need}},
             {{q, rows_bytes(M, a.q_stride, (double)a.H * desc->head_dim, es)}, {k_tree, kv}, {v_tree, kv}, {k_cache, cache},
              {v_cache, cache}, {cache_len, max_len > 0 ? 4. * a.n_seq : 0.}, {a.tree_off, 4. * (a.n_seq + 1.)},
              {a.tree_mask, 4. * M * a.words}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_tree_attention(*desc, a, out, lse, ws, static_cast<hipStream_t>(hip_stream)));
}

moespec_status moespec_cache_weights(const moespec_attn_desc *desc, const moespec_tree *tree, const void *q,
                                     const void *k_tree, const void *k_cache, const int32_t *cache_len, int32_t max_len,
                                     const float *lse, const float *row_weight, float decay, const float *cache_w_in,
                                     float *cache_w_out, float *tree_w, void *ws, size_t ws_bytes, void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK || (s = check_tree(*desc, tree, max_len, true)) != MOESPEC_OK) return s;
  if (!q || !k_tree || !lse || !aligned16(q) || !aligned16(k_tree) || !aligned4(lse) || !aligned4(row_weight) ||
      !aligned4(cache_w_in) || !aligned4(tree_w) || !isfinite(decay))
    return MOESPEC_ERR_INVALID_ARG;
  if (max_len > 0 &&
      (!k_cache || !cache_len || !cache_w_out || !aligned16(k_cache) || !aligned4(cache_len) || !aligned4(cache_w_out)))
    return MOESPEC_ERR_INVALID_ARG;
  const size_t need = attn_ws(*desc, tree->n_seq, tree->max_tree, max_len);
  if ((s = check_ws(ws, ws_bytes, need)) != MOESPEC_OK) return s;
  const int64_t tiles = ((int64_t)max_len + 127) / 128 + (tree->max_tree + 127) / 128;
  if ((int64_t)tree->n_seq * desc->n_kv_heads * tiles * 256 > kMaxThreads) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const KeyArgs a = key_args(*desc, *tree, q, k_tree, nullptr, k_cache, nullptr, cache_len, max_len);
  const double M = a.M, es = elem_bytes(*desc), entries = max_len > 0 ? cache_entries(*desc, 1, a.n_seq) : 0.;
  if (!apart({{cache_w_out, 4. * entries}, {tree_w, 4. * M * a.Hk}, {ws, (double)need}},
             {{q, rows_bytes(M, a.q_stride, (double)a.H * desc->head_dim, es)},
              {k_tree, rows_bytes(M, a.kv_stride, (double)a.Hk * desc->head_dim, es)}, {k_cache, entries * desc->head_dim * es},
              {cache_len, max_len > 0 ? 4. * a.n_seq : 0.}, {lse, 4. * M * a.H}, {row_weight, 4. * M},
              {cache_w_in == cache_w_out ? nullptr : cache_w_in, 4. * entries}, {a.tree_off, 4. * (a.n_seq + 1.)},
              {a.tree_mask, 4. * M * a.words}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_cache_weights(*desc, a, lse, row_weight, decay, cache_w_in, cache_w_out, tree_w, ws,
                                       static_cast<hipStream_t>(hip_stream)));
}

moespec_status moespec_cache_commit(const moespec_attn_desc *desc, int32_t n_layers, const moespec_tree *tree,
                                    const void *k_tree, const void *v_tree, const float *tree_w, const int32_t *path,
                                    const int32_t *n_path, int32_t max_path, void *k_cache, void *v_cache, float *cache_w,
                                    const int32_t *cache_len, int32_t *new_len, void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK || (s = check_tree(*desc, tree, 0, false)) != MOESPEC_OK) return s;
  if (n_layers < 1 || n_layers > 4096 || max_path < 1 || max_path > kMost) return MOESPEC_ERR_INVALID_ARG;
  if (!k_tree || !v_tree || !path || !n_path || !k_cache || !v_cache || !cache_len || !aligned16(k_tree) || !aligned16(v_tree) ||
      !aligned16(k_cache) || !aligned16(v_cache) || !aligned4(path) || !aligned4(n_path) || !aligned4(cache_len) ||
      !aligned4(new_len) || !aligned4(tree_w) || !aligned4(cache_w))
    return MOESPEC_ERR_INVALID_ARG;
  if ((tree_w == nullptr) != (cache_w == nullptr) || new_len == cache_len || (new_len && new_len == n_path))
    return MOESPEC_ERR_INVALID_ARG;
  // threads: 16 bytes of a row each
  const int64_t pieces = (int64_t)desc->head_dim * (desc->dtype == MOESPEC_BF16 ? 2 : 4) / 16;
  if ((double)n_layers * tree->n_seq * max_path * desc->n_kv_heads * pieces > (double)kMaxThreads)
    return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const double es = elem_bytes(*desc), D = desc->head_dim, M = tree->n_tokens, n_seq = tree->n_seq, Hk = desc->n_kv_heads;
  const double entries = cache_entries(*desc, n_layers, tree->n_seq);
  const double kv = rows_bytes(n_layers * M, tree->kv_stride ? (double)tree->kv_stride : Hk * D, Hk * D, es);
  if (!apart({{k_cache, entries * D * es}, {v_cache, entries * D * es}, {cache_w, 4. * entries}, {new_len, 4. * n_seq}},
             {{k_tree, kv}, {v_tree, kv}, {tree_w, 4. * n_layers * M * Hk}, {path, 4. * n_seq * max_path}, {n_path, 4. * n_seq},
              {cache_len, 4. * n_seq}, {tree->tree_off, 4. * (n_seq + 1.)}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_cache_commit(*desc, n_layers, *tree, k_tree, v_tree, tree_w, path, n_path, max_path, k_cache, v_cache,
                                      cache_w, cache_len, new_len, static_cast<hipStream_t>(hip_stream)));
}

size_t moespec_evict_workspace_bytes(const moespec_attn_desc *desc, int32_t n_layers, int32_t n_seq, int32_t budget) {
  if (check_desc(desc) != MOESPEC_OK || n_layers < 1 || n_layers > 4096 || n_seq < 1 || n_seq > kMost || budget < 1) return 0;
  return align_up(sizeof(int32_t) * (size_t)n_layers * n_seq * desc->n_kv_heads * budget, 256);
}

moespec_status moespec_cache_evict(const moespec_attn_desc *desc, int32_t n_layers, int32_t n_seq, const void *k_cache,
                                   const void *v_cache, const float *cache_w, const int32_t *cache_len, int32_t budget,
                                   int32_t recent, int32_t out_capacity, void *k_out, void *v_out, float *w_out, int32_t *kept,
                                   int32_t *new_len, void *ws, size_t ws_bytes, void *hip_stream) {
  moespec_status s = check_desc(desc);
  if (s != MOESPEC_OK) return s;
  if (n_layers < 1 || n_layers > 4096 || n_seq < 1 || n_seq > kMost || budget < 1 || budget > out_capacity || recent < 0 ||
      recent > budget)
    return MOESPEC_ERR_INVALID_ARG;
  if (!k_cache || !v_cache || !cache_w || !cache_len || !k_out || !v_out || !w_out || !aligned16(k_cache) ||
      !aligned16(v_cache) || !aligned16(k_out) || !aligned16(v_out) || !aligned4(cache_w) || !aligned4(cache_len) ||
      !aligned4(w_out) || !aligned4(kept) || !aligned4(new_len))
    return MOESPEC_ERR_INVALID_ARG;
  if (k_out == k_cache || k_out == v_cache || v_out == k_cache || v_out == v_cache || k_out == v_out || w_out == cache_w ||
      new_len == cache_len || kept == cache_len || (kept && kept == new_len))
    return MOESPEC_ERR_INVALID_ARG;
  if ((s = check_ws(ws, ws_bytes, moespec_evict_workspace_bytes(desc, n_layers, n_seq, budget))) != MOESPEC_OK) return s;
  const int64_t pieces = (int64_t)desc->head_dim * (desc->dtype == MOESPEC_BF16 ? 2 : 4) / 16;
  const int64_t heads = (int64_t)n_layers * n_seq * desc->n_kv_heads;
  if (heads * 1024 > kMaxThreads || (double)heads * (((double)budget * pieces) / 1024 + 1) * 256 > (double)kMaxThreads)
    return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  const double es = elem_bytes(*desc), D = desc->head_dim, in = cache_entries(*desc, n_layers, n_seq), out = (double)heads * out_capacity;
  const Span list = {kept ? static_cast<void *>(kept) : ws, 4. * heads * budget};
  if (!apart({{k_out, out * D * es}, {v_out, out * D * es}, {w_out, 4. * out}, list, {new_len, 4. * n_seq}},
             {{k_cache, in * D * es}, {v_cache, in * D * es}, {cache_w, 4. * in}, {cache_len, 4. * n_seq}}))
    return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_cache_evict(*desc, n_layers, n_seq, k_cache, v_cache, cache_w, cache_len, budget, recent, out_capacity,
                                     k_out, v_out, w_out, kept ? kept : static_cast<int32_t *>(ws), new_len,
                                     static_cast<hipStream_t>(hip_stream)));
}

moespec_status moespec_block_norm(const moespec_desc *desc, const moespec_block *block, const void *y, const void *residual,
                                  int32_t M, void *r, void *x, void *hip_stream) {
  moespec_status s = moespec_check_desc(desc);
  if (s != MOESPEC_OK) return s;
  if (!block || M < 1 || M > kMost || !y || (!r && !x) || r == x) return MOESPEC_ERR_INVALID_ARG;
  if (!aligned16(y) || !aligned16(residual) || !aligned16(r) || !aligned16(x)) return MOESPEC_ERR_INVALID_ARG;
  const moespec_block &b = *block;
  if ((b.post_norm != 0 && b.post_norm != 1) || (b.gate_sigmoid != 0 && b.gate_sigmoid != 1) ||
      b.gate_kind < MOESPEC_BLOCK_GATE_NONE || b.gate_kind > MOESPEC_BLOCK_GATE_ELEMENT || !(b.eps >= 0.f) || !isfinite(b.eps) ||
      !isfinite(b.scale))
    return MOESPEC_ERR_INVALID_ARG;
  if ((b.gate_kind == MOESPEC_BLOCK_GATE_NONE) != (b.gate == nullptr) || (b.w_post && !b.post_norm)) return MOESPEC_ERR_INVALID_ARG;
  if (!aligned16(b.gate) || !aligned16(b.w_post) || !aligned16(b.w_pre)) return MOESPEC_ERR_INVALID_ARG;
  // a row is read before it is written: the same buffer is fine, another part of it is not
  const double es = desc->dtype == MOESPEC_BF16 ? 2 : 4, rows = (double)M * desc->d * es, d = desc->d * es;
  const bool element = b.gate_kind == MOESPEC_BLOCK_GATE_ELEMENT;
  const double gate = element ? rows : b.gate_kind == MOESPEC_BLOCK_GATE_TOKEN ? M * es : d;
  for (const void *o : {r, x})
    if (!apart({{o, rows}}, {{y == o ? nullptr : y, rows}, {residual == o ? nullptr : residual, rows},
                             {element && b.gate == o ? nullptr : b.gate, gate}, {b.w_post, d}, {b.w_pre, d},
                             {o == r ? x : r, rows}}))
      return MOESPEC_ERR_INVALID_ARG;
  return from_hip(launch_block_norm(*desc, b, y, residual, M, r, x, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
