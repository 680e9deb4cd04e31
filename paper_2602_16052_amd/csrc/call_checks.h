// Argument checks that the calls around attention share.  Host only.
#pragma once

#include <math.h>

#include <initializer_list>

#include "attention.h"

namespace moespec {

constexpr int kMost = 65535;                 // tokens, sequences
constexpr int32_t kMaxEntries = 0x7fff0000;   // the kernels round numbers of entries up to whole tiles in 32 bits
constexpr int64_t kMaxStride = 1 << 20;      // elements; the kernels reach the rows of a stage with 32-bit byte offsets
constexpr int64_t kMaxThreads = (1ll << 32) - 1024;  // threads of a launch

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline moespec_status from_hip(hipError_t e) { return e == hipSuccess ? MOESPEC_OK : MOESPEC_ERR_HIP; }

inline double elem_bytes(const moespec_attn_desc &ds) { return ds.dtype == MOESPEC_BF16 ? 2 : 4; }
inline double cache_entries(const moespec_attn_desc &ds, double layers, double n_seq) {
  return layers * n_seq * ds.n_kv_heads * ds.capacity;
}

inline moespec_status check_desc(const moespec_attn_desc *ds) {
  if (!ds) return MOESPEC_ERR_INVALID_ARG;
  if (ds->dtype != MOESPEC_F32 && ds->dtype != MOESPEC_BF16) return MOESPEC_ERR_INVALID_ARG;
  if (ds->n_heads < 1 || ds->n_kv_heads < 1 || ds->head_dim < 1 || ds->capacity < 1) return MOESPEC_ERR_INVALID_ARG;
  if (ds->n_heads % ds->n_kv_heads != 0) return MOESPEC_ERR_INVALID_ARG;
  if (!(ds->scale > 0.f) || !isfinite((float)((double)ds->scale * 1.4426950408889634))) return MOESPEC_ERR_INVALID_ARG;
  if (ds->n_heads > 1024 || ds->capacity > kMaxEntries) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  switch (ds->head_dim) {
    case 64: case 96: case 128: case 192: case 256: return MOESPEC_OK;
    default: return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  }
}

inline bool batch_ok(const moespec_attn_desc &ds, int32_t n_seq, int32_t M, int32_t max_tree, int32_t max_len) {
  return n_seq >= 1 && n_seq <= kMost && M >= 1 && M <= kMost && max_tree >= 1 && max_tree <= M && max_len >= 0 &&
         max_len <= ds.capacity;
}

// The batch: sizes, strides, offsets.  Queries (q) are checked where a call has them.
inline moespec_status check_tree(const moespec_attn_desc &ds, const moespec_tree *t, int32_t max_len, bool queries) {
  if (!t || !batch_ok(ds, t->n_seq, t->n_tokens, t->max_tree, max_len)) return MOESPEC_ERR_INVALID_ARG;
  if (!t->tree_off && t->n_seq != 1) return MOESPEC_ERR_INVALID_ARG;
  if (!aligned4(t->tree_off) || !aligned4(t->tree_mask)) return MOESPEC_ERR_INVALID_ARG;
  const int64_t es = ds.dtype == MOESPEC_BF16 ? 2 : 4;
  auto stride_ok = [&](int64_t stride, int64_t row) {
    return stride == 0 || (stride >= row && stride * es % 16 == 0);
  };
  const int64_t kv = (int64_t)ds.n_kv_heads * ds.head_dim, q = (int64_t)ds.n_heads * ds.head_dim;
  if (t->kv_stride < 0 || t->q_stride < 0) return MOESPEC_ERR_INVALID_ARG;
  if (t->kv_stride > kMaxStride || t->q_stride > kMaxStride) return MOESPEC_ERR_UNSUPPORTED_SHAPE;
  if (!stride_ok(t->kv_stride, kv) || (queries && !stride_ok(t->q_stride, q))) return MOESPEC_ERR_INVALID_ARG;
  return MOESPEC_OK;
}

inline moespec_status check_ws(const void *ws, size_t have, size_t need) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return MOESPEC_ERR_INVALID_ARG;
  return have < need ? MOESPEC_ERR_WORKSPACE_TOO_SMALL : MOESPEC_OK;
}

// Bytes of a call's buffer (none where p is NULL, 0 where the call does not touch it).  In floating point: a size may be beyond 64 bits, and is exact up to 2^53.
struct Span {
  const void *p;
  double bytes;
};
inline bool overlap(const Span &a, const Span &b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  if (!a.p || !b.p || !(a.bytes > 0.) || !(b.bytes > 0.)) return false;
  return x <= y ? (double)(y - x) < a.bytes : (double)(x - y) < b.bytes;
}
// Whether what a call writes lies apart from everything else that it uses.  Workgroups run in any order, so a result in the place of
// something that another one still reads would be a wrong one.
inline bool apart(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  for (const Span *w = written.begin(); w != written.end(); ++w) {
    for (const Span *v = written.begin(); v != w; ++v)
      if (overlap(*v, *w)) return false;
    for (const Span &r : read)
      if (overlap(*w, r)) return false;
  }
  return true;
}
inline double rows_bytes(double n, double stride, double row, double es) { return ((n - 1) * stride + row) * es; }

}  // namespace moespec
