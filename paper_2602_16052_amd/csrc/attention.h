// What the kernels over a cache of keys share: where a sequence's rows and entries lie, and how tiles of keys lie in LDS.
#pragma once

#include "common.h"

namespace moespec {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

constexpr int kMaxParts = 256;     // parts of a single sequence's keys
constexpr int kMaxShared = 256;    // sequences that share the parts of a launch

// The arguments that say which rows and entries there are (host pointers resolved, strides in elements, never 0).
struct KeyArgs {
  const void *q, *k_tree, *v_tree, *k_cache, *v_cache;
  const int32_t *cache_len, *tree_off;
  const uint32_t *tree_mask;
  int64_t q_stride, kv_stride, capacity;
  int n_seq, M, max_tree, words, max_len, H, Hk, G;
  float c;         // scale * log2(e): scores in units of log 2
  float u, u_rest;  // c / scale in two parts: an lse in the same units, with the rounding of c
};

// One sequence: first token row, rows of its tree, entries of its cache.  Device data, clamped to what the buffers hold.
struct SeqGeom {
  int row0, T, len;
};
__device__ __forceinline__ SeqGeom seq_geom(const KeyArgs &a, int s) {
  SeqGeom g{0, a.M, 0};
  if (a.tree_off) {
    g.row0 = min(max(a.tree_off[s], 0), a.M);
    g.T = min(max(a.tree_off[s + 1], g.row0), a.M) - g.row0;
  }
  g.T = min(g.T, a.max_tree);
  if (a.max_len > 0) g.len = min(max(a.cache_len[s], 0), a.max_len);
  return g;
}

// Sum of v over the wave, in every lane.
__device__ __forceinline__ int wave_sum(int v) {
  v = row16_sum(v);
  const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = (int)(a[0] + a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return (int)(b[0] + b[1]);
}

// The keys of a launch in parts.  slots == 0: a sequence's keys are one part, `index` is the sequence.  Otherwise the sequences share
// `slots` parts: with the smallest chunk of units (tiles of keys, by units(geometry); 0 where there is nothing to do) of which
// every sequence takes as many as it needs and all together fit, `index` is the part.  One sequence has all parts.
// first_of (may be NULL): [n_seq + 1], receives the first part of every sequence (of more than one).
struct Share {
  int s, part, parts;  // sequence (-1: none), which of how many parts
  // units part * chunk .. of a workgroup that has `all` of them
  __device__ __forceinline__ int first(int all) const { return (int)min((int64_t)all, (int64_t)part * ((all + parts - 1) / parts)); }
  __device__ __forceinline__ int last(int all) const { return (int)min((int64_t)all, (part + 1ll) * ((all + parts - 1) / parts)); }
};
template <typename Units>
__device__ __forceinline__ Share share_of(const KeyArgs &a, int slots, int index, Units units, int32_t *first_of) {
  if (slots == 0) return Share{index, 0, 1};
  if (a.n_seq == 1) return Share{0, index, slots};
  constexpr int NU = kMaxShared / kWave;
  const int lane = threadIdx.x & 63;
  int n[NU], total = 0;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int s = lane + kWave * u;
    n[u] = s < a.n_seq ? units(seq_geom(a, s)) : 0;
    total += n[u];
  }
  total = wave_sum(total);
  int lo = max((total + slots - 1) / slots, 1), hi = max((total + slots - a.n_seq - 1) / (slots - a.n_seq), lo);
  auto parts = [&](int units_of, int chunk) { return (units_of + chunk - 1) / chunk; };
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    int all = 0;
#pragma unroll
    for (int u = 0; u < NU; ++u)
      if (kWave * u < a.n_seq) all += parts(n[u], mid);
    if (__builtin_amdgcn_readfirstlane(wave_sum(all)) <= slots) hi = mid;
    else lo = mid + 1;
  }
  Share r{-1, 0, 1};
  int before = 0;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    if (kWave * u >= a.n_seq) break;
    const int mine = parts(n[u], lo);
    int scan = mine;  // parts of this sequence and of those in front of it
#pragma unroll
    for (int x = 1; x < kWave; x <<= 1) {
      const int up = __shfl_up(scan, x, kWave);
      if (lane >= x) scan += up;
    }
    scan += before;
    if (first_of && lane + kWave * u < a.n_seq) first_of[lane + kWave * u + 1] = scan;
    const uint64_t hit = __ballot(index >= scan - mine && index < scan);
    if (hit != 0) {
      const int l = __builtin_ctzll(hit), part = index - (__shfl(scan, l, kWave) - __shfl(mine, l, kWave));
      r = Share{kWave * u + l, __builtin_amdgcn_readfirstlane(part), __builtin_amdgcn_readfirstlane(__shfl(mine, l, kWave))};
    }
    before = __shfl(scan, 63, kWave);
  }
  if (first_of && lane == 0) first_of[0] = 0;
  return r;
}

__host__ __device__ constexpr int pow2_ceil(int x) {
  int p = 1;
  while (p < x) p <<= 1;
  return p;
}

// A tile of rows of D elements in LDS: a row is kSlots slots of 16 bytes (a power of two; the row's pieces and padding that is
// never read).  Piece p of row r sits in slot p ^ swz(r).  Reads of the same piece of 16 consecutive rows (keys as a matrix operand) then
// touch every bank once, and so do reads of the same 64 bytes of 4 rows in a row (bf16 values, transposed on the way out of
// LDS).  fp32 values are read as 128 bytes of two rows, 4 apart: swz_values puts those into different halves of the banks.
template <typename T, int D>
struct Rows {
  static constexpr int kPieceElems = 16 / (int)sizeof(T);
  static constexpr int kPieces = D / kPieceElems;
  static constexpr int kSlots = pow2_ceil(kPieces);
  static constexpr int kBytes = 16 * kSlots;
  static __device__ __forceinline__ int swz(int row) {
    return kSlots == 8 ? 4 * ((row >> 1) & 1) + ((row >> 2) & 3) : 4 * (row & 3) + ((row >> 2) & 3);
  }
  static __device__ __forceinline__ int swz_values(int row) { return sizeof(T) == 2 ? swz(row) : 8 * ((row >> 2) & 1); }
};

// The matrix operands of 32 rows x D: step i multiplies pieces 2 i (lanes 0-31) and 2 i + 1 (lanes 32-63) of every row, so
// that both operands load 16 bytes per lane and the order of the sum over D is the same in both.
template <typename T>
struct Frag;
template <>
struct Frag<uint16_t> {
  typedef bf16x8 type;
  static __device__ __forceinline__ f32x16 mma(type a, type b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Frag<float> {
  typedef f32x4 type;
  static __device__ __forceinline__ f32x16 mma(type a, type b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};

// An operand that has been loaded, for the compiler too: it does not see the fetches to LDS, and would else wait inside of a loop for
// the youngest of them where it means the operand.
template <typename F>
__device__ __forceinline__ void arrived(F &f) {
  asm volatile("" : "+v"(f));
}

// Row (of 32) of element i of a lane's 32 x 32 result; half = lane >> 5.  The column is lane & 31.
__device__ __forceinline__ int acc_row(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

// v of lane ^ 32 combined with the lane's own.
__device__ __forceinline__ float half_swap(float v, bool max_) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
  return max_ ? fmaxf(a, b) : a + b;
}

// Which of the 32 keys base .. base + 31 (of n) a row sees: all of a cache, a token's ancestors in its tree.
__host__ __device__ __forceinline__ uint32_t keys_below(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t tree_word(const KeyArgs &a, const SeqGeom &g, int t, int base) {
  if (base >= g.T) return 0;
  const uint32_t w = a.tree_mask ? a.tree_mask[(size_t)(g.row0 + t) * a.words + (base >> 5)] : keys_below(t + 1 - base);
  return w & keys_below(g.T - base);
}

// The bits of 32 places of a tile without those behind the last key (`there` places have one).  Places behind it repeat it in LDS
// and have nothing of their own in memory.
__host__ __device__ __forceinline__ uint32_t keys_there(uint32_t bits, int there) { return bits & keys_below(there); }

// What a lane holds of a finished row (elements acc_row(i, half) of every 32; m in units of log 2) written out, or left for the
// combine where the keys are in parts, of which this is number `index`.
template <typename T, int D>
__device__ __forceinline__ void finish_row(const KeyArgs &a, const f32x16 (&o)[D / 32], float m, float l, int slots,
                                           int index, int t, int h, size_t orow, int half, T *out, float *lse, float *part,
                                           float2 *part_ml) {
  if (slots == 0) {
    const bool none = l == 0.f;  // no key, or scores of -inf alone: 0, also where weights of 0 have met a value that is not finite
    const float inv = 1.f / l;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = none ? 0.f : o[b][i + e] * inv;
        Elem<T>::store4(out + orow * D + 32 * b + acc_row(i, half), v);
      }
    if (lse && half == 0) lse[orow] = none ? -INFINITY : (m + __log2f(l)) * 0.69314718055994531f;
  } else {
    const size_t at = (size_t)index * a.max_tree * a.H + (size_t)t * a.H + h;
    if (half == 0) part_ml[at] = make_float2(m, l);
    if (m == -INFINITY) return;  // the combine passes it over
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4 *>(part + at * D + 32 * b + acc_row(i, half)) =
            f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
  }
}

hipError_t launch_tree_attention(const moespec_attn_desc &ds, const KeyArgs &a, void *out, float *lse, void *ws,
                                 hipStream_t st);
size_t tree_attention_ws(const moespec_attn_desc &ds, int64_t n_seq, int64_t max_tree, int64_t max_len);
hipError_t launch_cache_weights(const moespec_attn_desc &ds, const KeyArgs &a, const float *lse, const float *row_weight,
                                float decay, const float *w_in, float *w_out, float *tree_w, void *ws, hipStream_t st);
size_t cache_weights_ws(const moespec_attn_desc &ds, int64_t n_seq, int64_t max_tree, int64_t max_len);
hipError_t launch_cache_commit(const moespec_attn_desc &ds, int n_layers, const moespec_tree &tree, const void *k_tree,
                               const void *v_tree, const float *tree_w, const int32_t *path, const int32_t *n_path,
                               int max_path, void *k_cache, void *v_cache, float *cache_w, const int32_t *cache_len,
                               int32_t *new_len, hipStream_t st);
hipError_t launch_cache_evict(const moespec_attn_desc &ds, int n_layers, int n_seq, const void *k_cache,
                              const void *v_cache, const float *cache_w, const int32_t *cache_len, int budget, int recent,
                              int out_capacity, void *k_out, void *v_out, float *w_out, int32_t *kept, int32_t *new_len,
                              hipStream_t st);
hipError_t launch_block_norm(const moespec_desc &ds, const moespec_block &b, const void *y, const void *residual, int M,
                             void *r, void *x, hipStream_t st);

}  // namespace moespec
