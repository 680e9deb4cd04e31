// Attention of drafted tokens over a cache of keys and over their own tree.
//
// The rows of one KV head are its tokens x the G query heads that share it, so a tile of keys that is fetched once serves all
// of them.  One pass over the keys with a running maximum m and sum l per row (in units of log 2):
//   p = 2^(c q.k - m),  l = l 2^(m_old - m) + sum p,  O = O 2^(m_old - m) + p V,   out = O / l.
// A workgroup of WR x WK waves takes 32 WR rows and one part of the keys; wave (wr, wk) multiplies rows 32 wr .. + 31
// with its 32 KB of every stage of 32 KB WK keys.  The products are taken transposed: S^T = K Q^T has a row of scores in one lane
// column (two lanes), so that the softmax needs one exchange between lanes per 32 KB keys, and its weights are already the
// right operand of O^T = V^T P^T: element i of a lane's S^T is key 8 (i / 4) + 4 (lane / 32) + i % 4, and V^T is read from LDS in the same
// order of keys (bf16: transposing reads).
// Keys and values go from memory straight into LDS, one stage ahead of the products.
//
// What bounds it: few rows, the stream of keys and values (16 trees of up to 31 tokens x 4 heads, caches of up to 16381 entries: 175 to
// 182 us, 4.6 to 4.7 TB/s, what a large copy reaches; one token over 65521 entries 30 us, 4.4 TB/s); short caches, launches and trips
// to memory (one token over 1021 entries 9.2 us in two launches, of which the kernels are 5.4 and 3.5 to 4.1).
// Key waves side by side share one stage: for up to 64 rows, workgroups of a stage of 32 keys each with nothing to join took 24.4
// us where these take 19.6 (63 rows x 16 heads, 4093 entries; 72 against 63 with 32768), but win where all keys make one round of
// them (one token over 1021 entries 9.5 us against 11.2).  A third stage ahead, issued behind a second barrier, was slower (25.4 us).
#include <math.h>

#include "attention.h"

namespace moespec {

template <typename T, int D>
struct AttnShape {
  static constexpr int kRow = Rows<T, D>::kBytes;
  static constexpr int kWk1 = 1024 / kRow < 4 ? 1024 / kRow : 4;  // key waves for up to 32 rows: a stage of up to 64 KB
  static constexpr int kWk2 = 1024 / kRow < 2 ? 1024 / kRow : 2;  // ... for up to 64
  static constexpr int kKb4 = sizeof(T) == 2 ? 2 : 1;  // 32-key blocks of a wave with 128 rows a workgroup
};

// Where a lane's operands lie in a tile of keys and one of values: few addresses, everything else is a constant offset (swz
// only touches the last 4 bits of a slot).
template <typename T, int D>
struct TileAddr {
  typedef Rows<T, D> R;
  static constexpr int NB = D / 32, NS = R::kPieces / 2, NK = NS < 8 ? NS : 8, NV = NB < 4 ? NB : 4;
  uint32_t k[NK], v[sizeof(T) == 2 ? NV : 2][sizeof(T) == 2 ? 2 : 1];
  __device__ __forceinline__ TileAddr() {
    const int lane = threadIdx.x & 63, l31 = lane & 31, half = lane >> 5;
#pragma unroll
    for (int i = 0; i < NK; ++i) k[i] = l31 * R::kBytes + (((2 * i + half) ^ R::swz(l31)) << 4);
    if constexpr (sizeof(T) == 2) {
      // lane i of 16 points at 4 elements of row i / 4 and receives element i of 4 rows
      const int i16 = lane & 15, vrow = 4 * half + (i16 >> 2), low = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
#pragma unroll
      for (int b = 0; b < NV; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          v[b][e] = (vrow + 8 * e) * R::kBytes + (((4 * b + low) ^ R::swz(vrow + 8 * e)) << 4) + 8 * (i16 & 1);
    } else {
#pragma unroll
      for (int b = 0; b < 2; ++b) v[b][0] = 4 * half * R::kBytes + (((8 * b + (l31 >> 2)) ^ (8 * half)) << 4) + 4 * (l31 & 3);
    }
  }
  // The addresses in another place.  Opaque to the compiler, which would join the place and the constant offsets and add their sum
  // for every read.
  __device__ __forceinline__ void move(uint32_t keys, uint32_t values) {
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      k[i] += keys;
      asm volatile("" : "+v"(k[i]));
    }
#pragma unroll
    for (auto &x : v)
#pragma unroll
      for (uint32_t &y : x) {
        y += values;
        asm volatile("" : "+v"(y));
      }
  }
  // keys 32 kb .. + 31, step i of the sum over D
  __device__ __forceinline__ typename Frag<T>::type key(uint32_t tile, int kb, int i) const {
    typedef __attribute__((address_space(3))) typename Frag<T>::type lds_frag;
    return *(lds_frag *)(uintptr_t)(k[i % 8] + tile + 32 * kb * R::kBytes + i / 8 * 256);
  }
  // bf16: elements 32 b .. + 31 of keys 32 kb + 16 j .. + 15 in the order of a lane's scores
  __device__ __forceinline__ bf16x8 values(uint32_t tile, int kb, int j, int b) const {
    typedef __attribute__((address_space(3))) bf16x4 lds4;
    const uint32_t at = tile + (32 * kb + 16 * j) * R::kBytes + b / 4 * 256;
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(uintptr_t)(v[b % 4][0] + at));
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(uintptr_t)(v[b % 4][1] + at));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  // fp32: element 32 b + l31 of key 32 kb + acc_row(i, half)
  __device__ __forceinline__ float value(uint32_t tile, int kb, int i, int b) const {
    typedef __attribute__((address_space(3))) float lds1;
    return *(lds1 *)(uintptr_t)(v[b % 2][0] + tile + (32 * kb + acc_row(i, 0)) * R::kBytes + b / 2 * 256);
  }
};

template <typename T>
__device__ __forceinline__ bool not_finite(T bits) {
  return sizeof(T) == 2 ? (bits & 0x7f80u) == 0x7f80u : ((uint32_t)bits & 0x7f800000u) == 0x7f800000u;
}

// A weight of 0 times a NaN or an infinity would reach a token that does not see that key.  So values that not every row sees are
// looked at by the workgroup before they are multiplied: what is not finite becomes 0 in LDS, its key's bit is set in odd (one word per 32
// keys), and add_odd adds it to the rows that see the key.  Those are the values of a tree, and the repetitions of a cache's last entry
// that fill its last tile (only where that entry has such a value: row_not_finite).
template <typename T, int D, int kKeys, int kThreads>
__device__ __forceinline__ void clean_values(unsigned char *tile, uint32_t *odd) {
  typedef Rows<T, D> R;
  static_assert(kKeys * R::kSlots % kThreads == 0, "whole rounds of the workgroup");
#pragma unroll 4
  for (int x = 0; x < kKeys * R::kSlots / kThreads; ++x) {
    const int id = x * kThreads + (int)threadIdx.x, key = id / R::kSlots;
    if (((id % R::kSlots) ^ R::swz_values(key)) >= R::kPieces) continue;
    uint4 *p = reinterpret_cast<uint4 *>(tile + 16 * id);
    uint4 v = *p;
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) {
        const bool lo = not_finite<uint16_t>(w[e] & 0xffffu), hi = not_finite<uint16_t>(w[e] >> 16);
        w[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
        bad |= lo | hi;
      } else {
        const bool is = not_finite<uint32_t>(w[e]);
        w[e] = is ? 0u : w[e];
        bad |= is;
      }
    }
    if (bad) {
      *p = make_uint4(w[0], w[1], w[2], w[3]);
      atomicOr(&odd[key >> 5], 1u << (key & 31));
    }
  }
}
// Whether row r of a tile has a value that is not finite, the same in every lane.
template <typename T, int D>
__device__ __forceinline__ bool row_not_finite(const unsigned char *tile, int r) {
  const uint4 v = *reinterpret_cast<const uint4 *>(tile + r * Rows<T, D>::kBytes + 16 * ((threadIdx.x & 63) % Rows<T, D>::kSlots));
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    bad |= sizeof(T) == 2 ? not_finite<uint16_t>(w[e] & 0xffffu) || not_finite<uint16_t>(w[e] >> 16) : not_finite<uint32_t>(w[e]);
  return __ballot(bad) != 0;
}
// bad: the keys (of 32, the first one's values at vg; each with a row of its own in memory) that have such values; seen: those that this
// row sees.
template <typename T, int D>
__device__ __forceinline__ void add_odd(uint32_t bad, uint32_t seen, const T *vg, int64_t stride, f32x16 (&o)[D / 32]) {
  const int half = (threadIdx.x & 63) >> 5;
  for (; bad != 0; bad &= bad - 1) {
    const int j = __builtin_ctz(bad);
    const bool mine = (seen >> j) & 1u;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 v = Elem<T>::load4(vg + j * stride + 32 * b + acc_row(i, half));
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (mine && not_finite<uint32_t>(__float_as_uint(v[e]))) o[b][i + e] += v[e];
      }
  }
}

// 32 KB keys, base .. of n, that lie in LDS at kt and vt, taken into a wave's 32 rows (row l31 is token t): scores, masks, running
// maximum and sum, values.  whole: every row sees all of them.  odd: see clean_values (NULL: nothing was cleaned); the first key's
// values lie at vg in memory, vstride elements apart.
template <typename T, int D, int KB>
__device__ __forceinline__ void attend_tile(const KeyArgs &a, const SeqGeom &g, TileAddr<T, D> at, bool tree, bool whole,
                                            int base, int n, int t, uint32_t kt, uint32_t vt, const uint32_t *odd, const T *vg, int64_t vstride,
                                            const typename Frag<T>::type (&q)[Rows<T, D>::kPieces / 2], f32x16 (&o)[D / 32],
                                            float &m, float &l) {
  constexpr int NB = D / 32, NS = Rows<T, D>::kPieces / 2;
  const int half = (threadIdx.x & 63) >> 5;
  at.move(kt, vt);
  f32x16 sc[KB];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) sc[kb] = Frag<T>::mma(at.key(0, kb, i), q[i], sc[kb]);
  }
  uint32_t word[KB];
  if (!whole) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      word[kb] = tree ? tree_word(a, g, t, base + 32 * kb) : keys_below(n - base - 32 * kb);
      const uint32_t w = word[kb] >> (4 * half);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!((w >> acc_row(i, 0)) & 1u)) sc[kb][i] = -INFINITY;
    }
  }
  float mx = sc[0][0];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[kb][i]);
  mx = half_swap(mx, true) * a.c;
  // The maximum is only raised when it is passed by more than 2^8: until then the weights stay below 2^8, in fp32 and in bf16
  // as exact as below 1, and O is not rescaled.
  const bool raise = mx > m + 8.f;
  if (__builtin_expect(__ballot(raise) != 0, 0)) {
    const float alpha = raise ? __builtin_amdgcn_exp2f(m - mx) : 1.f;
    m = raise ? mx : m;
    l *= alpha;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] *= alpha;
  }
  const float mu = m == -INFINITY ? 0.f : m;  // nothing seen so far: all weights are 0
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[kb][i] = __builtin_amdgcn_exp2f(fmaf(sc[kb][i], a.c, -mu));
      l += sc[kb][i];
    }
  if constexpr (sizeof(T) == 2) {
    // Weights are rounded to bf16, the type that the matrix instructions take beside bf16 values; l is the sum of the unrounded ones.
    // Half a step a weight, one way or the other from key to key: over long caches outputs are 0.0023 (relative, root of the mean
    // square) from 64 bits, where their own rounding leaves 0.0017.  What the rounding leaves, multiplied as well, would double
    // these instructions.
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        bf16x8 p;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = (__bf16)sc[kb][8 * j + i];
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.values(0, kb, j, b), p, o[b], 0, 0, 0);
      }
  } else {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(at.value(0, kb, i, b), sc[kb][i], o[b], 0, 0, 0);
  }
  if (odd != nullptr && !whole) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const uint32_t bad = keys_there(__builtin_amdgcn_readfirstlane(odd[kb]), n - base - 32 * kb);
      if (__builtin_expect(bad != 0, 0)) add_odd<T, D>(bad, word[kb], vg + 32 * kb * vstride, vstride, o);
    }
  }
}

template <typename T, int D, int WR, int WK, int KB>
__global__ __launch_bounds__(64 * WR * WK, (D <= 128 ? 2 : 1)) void tree_attention_kernel(
    KeyArgs a, int row_tiles, int slots, T *__restrict__ out, float *__restrict__ lse, float *__restrict__ part,
    float2 *__restrict__ part_ml, int32_t *__restrict__ first_of) {
  typedef Rows<T, D> R;
  typedef typename Frag<T>::type frag;
  constexpr int NW = WR * WK, kStageKeys = 32 * KB * WK, kTile = kStageKeys * R::kBytes, kStage = 2 * kTile;
  constexpr int kRowsPerLoad = 64 / R::kSlots, kLoads = kStageKeys / kRowsPerLoad / NW, NB = D / 32, NS = R::kPieces / 2;
  static_assert(kStageKeys % (kRowsPerLoad * NW) == 0, "every wave issues as many loads");
  extern __shared__ __align__(16) unsigned char lds[];
  uint32_t *const odd = reinterpret_cast<uint32_t *>(lds + 2 * kStage);  // [2][kStageKeys / 32], for the stages of both places
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave % WR, wk = wave / WR;
  const int l31 = lane & 31, half = lane >> 5;
  // row tiles that share keys are neighbours on one XCD (workgroup b runs on XCD b mod 8).  The last ones first: in a chain they see the
  // most keys, and what is left for the end of the launch is short (4096 tokens without a cache 154 us, 193 the other way round).
  const int slot = blockIdx.x / 8, group = slot / row_tiles * 8 + (int)(blockIdx.x % 8), tile = row_tiles - 1 - slot % row_tiles;
  const int n_parts = slots == 0 ? a.n_seq : slots, index = group % n_parts, hk = group / n_parts;
  if (hk >= a.Hk) return;
  auto stages = [&](const SeqGeom &g) {
    return g.T == 0 ? 0 : (g.len + kStageKeys - 1) / kStageKeys + (g.T + kStageKeys - 1) / kStageKeys;
  };
  const Share part_of = share_of(a, slots, index, stages, blockIdx.x == 0 ? first_of : nullptr);
  const int s = part_of.s;
  if (s < 0) return;
  const SeqGeom g = seq_geom(a, s);
  const int n_rows = g.T * a.G, r0 = tile * 32 * WR;
  if (r0 >= n_rows) return;

  // stages: those of the cache, then those of the tree (of a chain only up to the last row's token)
  const int ct = (g.len + kStageKeys - 1) / kStageKeys, all = ct + (g.T + kStageKeys - 1) / kStageKeys;
  const int first_t = r0 / a.G, last_t = (min(r0 + 32 * WR, n_rows) - 1) / a.G;
  const int tt = a.tree_mask ? all - ct : last_t / kStageKeys + 1;
  const int st0 = part_of.first(ct + tt), st1 = part_of.last(ct + tt);

  const int row = min(r0 + 32 * wr + l31, n_rows - 1), t = row / a.G, h = hk * a.G + row % a.G;
  const size_t orow = (size_t)(g.row0 + t) * a.H + h;
  const bool row_ok = r0 + 32 * wr + l31 < n_rows;

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds);
  const int64_t head = ((int64_t)s * a.Hk + hk) * a.capacity * D;
  // this lane's share of a stage: slots ld 64 + lane of both tiles.  Padding slots repeat a piece and are not read.
  int rr[kLoads];
  uint32_t kp[kLoads], vp[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    rr[i] = (i * NW + wave) * kRowsPerLoad + lane / R::kSlots;
    kp[i] = 16 * min((lane % R::kSlots) ^ R::swz(rr[i]), R::kPieces - 1);
    vp[i] = 16 * min((lane % R::kSlots) ^ R::swz_values(rr[i]), R::kPieces - 1);
  }
  auto issue = [&](int st, int buf) {
    const bool tree = st >= ct;
    const int base = (tree ? st - ct : st) * kStageKeys, last = (tree ? g.T : g.len) - 1 - base;
    const uint32_t stride = (uint32_t)((tree ? a.kv_stride : D) * sizeof(T));
    const int64_t at = tree ? (g.row0 + base) * a.kv_stride + hk * D : head + (int64_t)base * D;
    const T *kb = static_cast<const T *>(tree ? a.k_tree : a.k_cache) + at;
    const T *vb = static_cast<const T *>(tree ? a.v_tree : a.v_cache) + at;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      // keys past the end repeat the last one: their scores are masked, and their weights of 0 must meet numbers
      const uint32_t off = (uint32_t)min(rr[i], last) * stride;
      dma_to_lds(lds0 + buf * kStage + (i * NW + wave) * 1024, kb, off + kp[i]);
      dma_to_lds(lds0 + buf * kStage + kTile + (i * NW + wave) * 1024, vb, off + vp[i]);
    }
  };

  frag q[NS];
  {
    const T *qp = static_cast<const T *>(a.q) + (g.row0 + t) * a.q_stride + h * D + half * R::kPieceElems;
#pragma unroll
    for (int i = 0; i < NS; ++i) q[i] = *reinterpret_cast<const frag *>(qp + 2 * i * R::kPieceElems);
  }
  if (st0 < st1) issue(st0, 0);
  const TileAddr<T, D> at;
  f32x16 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < NS; ++i) arrived(q[i]);

  for (int st = st0; st < st1; ++st) {
    const int buf = (st - st0) & 1;
    const bool tree = st >= ct;
    const int base0 = (tree ? st - ct : st) * kStageKeys, n = tree ? g.T : g.len, base = base0 + wk * KB * 32;
    // keys inside the cache, or in front of every row's own token in a chain, are seen by all rows
    auto seen_whole = [&](int from, int keys) {
      return from + keys <= n && (!tree || (a.tree_mask == nullptr && from + keys - 1 <= first_t));
    };
    const bool in_part = !seen_whole(base0, kStageKeys);
    uint32_t *const my_odd = odd + buf * (kStageKeys / 32);
    if (in_part && threadIdx.x < kStageKeys / 32) my_odd[threadIdx.x] = 0;  // last read two stages ago
    wait_vm<0>();
    asm volatile("" ::: "memory");
    __syncthreads();  // the stage has arrived, everybody's part of it, and nobody reads the other one any more
    if (st + 1 < st1) issue(st + 1, buf ^ 1);
    const bool clean = in_part && (tree || row_not_finite<T, D>(lds + buf * kStage + kTile, n - 1 - base0));
    if (clean) {
      __syncthreads();  // everybody has looked
      clean_values<T, D, kStageKeys, 64 * NW>(lds + buf * kStage + kTile, my_odd);
      __syncthreads();
    }
    const uint32_t kt = lds0 + buf * kStage + wk * KB * 32 * R::kBytes;
    const int64_t vstride = tree ? a.kv_stride : D;
    const T *vg = static_cast<const T *>(tree ? a.v_tree : a.v_cache) +
                  (tree ? (g.row0 + base) * a.kv_stride + hk * D : head + (int64_t)base * D);
    // (with cleaned values every wave of the stage goes by the masks: a key wave that sees all of its keys may have had some cleaned)
    attend_tile<T, D, KB>(a, g, at, tree, !clean && seen_whole(base, 32 * KB), base, n, t, kt, kt + kTile,
                          clean ? my_odd + wk * KB : nullptr, vg, vstride, q, o, m, l);
  }
  l = half_swap(l, false);
  if (m == -INFINITY && l != 0.f) m = 0.f;  // scores that are all NaN: so is the row

  if constexpr (WK > 1) {  // the waves of a row block joined through LDS, where the stages were
    __syncthreads();
    float2 *ml = reinterpret_cast<float2 *>(lds);                              // [WK][WR][32]
    float *op = reinterpret_cast<float *>(lds + sizeof(float2) * 32 * NW);     // [WK - 1][WR][D / 4][32][4]
    if (half == 0) ml[(wk * WR + wr) * 32 + l31] = make_float2(m, l);
    __syncthreads();
    float mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) mt = fmaxf(mt, ml[(w * WR + wr) * 32 + l31].x);
    const float mu = mt == -INFINITY ? 0.f : mt;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float2 v = ml[(w * WR + wr) * 32 + l31];
      lt += v.y * __builtin_amdgcn_exp2f(v.x - mu);
    }
    const float f = __builtin_amdgcn_exp2f(m - mu);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] *= f;
    if (wk > 0) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4 *>(op + ((((wk - 1) * WR + wr) * (D / 4) + 8 * b + 2 * (i >> 2) + half) * 32 + l31) * 4) =
              f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
    }
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int w = 1; w < WK; ++w)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 v = *reinterpret_cast<const f32x4 *>(
              op + ((((w - 1) * WR + wr) * (D / 4) + 8 * b + 2 * (i >> 2) + half) * 32 + l31) * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[b][i + e] += v[e];
        }
    m = mt;
    l = lt;
  }
  if (row_ok) finish_row<T, D>(a, o, m, l, slots, index, t, h, orow, half, out, lse, part, part_ml);
}

// ---- Many rows per KV head (bf16, D <= 128): bound by arithmetic.
//
// A workgroup of four waves takes 256 rows, a wave 64 of them: every operand that is read from LDS is multiplied twice, which
// halves the LDS traffic that equals the time of the matrix instructions at 32 rows.  One wave per SIMD has all 512 registers and
// overlaps its own work: in one straight line of code the matrix instructions of S(i + 1) = K Q^T run beside the exponentials of
// S(i), those of O += V^T P(i) beside the rest of them and beside the maxima of S(i + 1).  Keys and values of the tiles come
// through two places each, K one tile ahead of V; one barrier per tile.
// Tiles that some row sees in part (the cache's last one, those of the tree) follow one by one.
// 511-token tree x 8 heads over 65521 entries: 510 to 560 us (980 to 1070 TFLOP/s; a library product of 8192^3 reaches 1210 here),
// against 690 us in the form above.  The matrix cores are busy for 46% of the cycles, at 2.0 GHz under this load, and idle for the rest:
// one wave a SIMD issues its instructions one by one, 5.6 of the vector ALU to a matrix instruction (counters).  Heads of 192 and
// 256 have 32 rows a wave (their O and Q fill the accumulation registers): 8 trees of 63 over 8192 entries, heads of 256, 176 us (768
// TFLOP/s) against 250.
template <int D>
struct WideShape {
  static constexpr int RB = D <= 128 ? 2 : 1;  // blocks of 32 rows of a wave
  static constexpr int kRows = 128 * RB, kKeys = 64, kTile = kKeys * Rows<uint16_t, D>::kBytes, kLds = 4 * kTile + 16;
};

// s0 (+)= a b0 and s1 (+)= a b1 with s and a in the registers that other instructions can read, b in the accumulation registers.  Left
// to the compiler, scores land in accumulation registers and cost a copy each.  The compiler keeps no distances to instructions
// that it does not see: a matrix instruction may read a register two wait states after another instruction has written it
// (s_nop 1), and the results are there 16 passes after the last of a chain: whoever reads them does so behind eight other matrix
// instructions or score_wait.
__device__ __forceinline__ void score_mfma(f32x16 &s0, f32x16 &s1, bf16x8 a, bf16x8 b0, bf16x8 b1, bool first) {
  if (first)
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %2, %3, 0\n\tv_mfma_f32_32x32x16_bf16 %1, %2, %4, 0"
                 : "=&v"(s0), "=&v"(s1)
                 : "v"(a), "a"(b0), "a"(b1));
  else
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %2, %3, %0\n\tv_mfma_f32_32x32x16_bf16 %1, %2, %4, %1"
                 : "+v"(s0), "+v"(s1)
                 : "v"(a), "a"(b0), "a"(b1));
}
__device__ __forceinline__ void score_mfma(f32x16 &s, bf16x8 a, bf16x8 b, bool first) {
  if (first)
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "a"(b));
  else
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "a"(b));
}
__device__ __forceinline__ void score_wait(f32x16 &s) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s)); }

template <int D>
__global__ __launch_bounds__(256, 1) void tree_attention_wide_kernel(KeyArgs a, int row_tiles, int slots,
                                                                     uint16_t *__restrict__ out, float *__restrict__ lse,
                                                                     float *__restrict__ part, float2 *__restrict__ part_ml,
                                                                     int32_t *__restrict__ first_of) {
  typedef Rows<uint16_t, D> R;
  typedef WideShape<D> W;
  constexpr int NB = D / 32, NS = R::kPieces / 2, kLoads = W::kTile / 1024 / 4, kRowsPerLoad = 64 / R::kSlots;
  constexpr int RB = W::RB, kScores = 32 * RB;  // scores of a lane in a tile
  constexpr int kSteps1 = 2 * NS, kSteps2 = 4 * NB;  // operands of S and of O, each multiplied RB times
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l31 = lane & 31, half = lane >> 5;
  const int slot = blockIdx.x / 8, group = slot / row_tiles * 8 + (int)(blockIdx.x % 8), tile = row_tiles - 1 - slot % row_tiles;
  const int n_parts = slots == 0 ? a.n_seq : slots, index = group % n_parts, hk = group / n_parts;
  if (hk >= a.Hk) return;
  // a tile that some row sees in part takes as long as kRest others
  constexpr int kRest = 3;
  auto units = [&](const SeqGeom &g) {
    return g.T == 0 ? 0 : g.len / 64 + kRest * ((g.len + 63) / 64 - g.len / 64 + (g.T + 63) / 64);
  };
  const Share part_of = share_of(a, slots, index, units, blockIdx.x == 0 ? first_of : nullptr);
  const int s = part_of.s;
  if (s < 0) return;
  const SeqGeom g = seq_geom(a, s);
  const int n_rows = g.T * a.G, r0 = tile * W::kRows;
  if (r0 >= n_rows) return;
  const int first_t = r0 / a.G, last_t = (min(r0 + W::kRows, n_rows) - 1) / a.G;

  // tiles that every row sees whole: of the cache, then of a chain in front of the first row's token; the others behind them
  const int cache_whole = g.len / 64, whole = cache_whole + (a.tree_mask ? 0 : (first_t + 1) / 64);
  const int cache_rest = (g.len + 63) / 64 - cache_whole;
  const int all = whole + cache_rest + (a.tree_mask ? (g.T + 63) / 64 : last_t / 64 + 1 - (first_t + 1) / 64);
  const int my_units = whole + kRest * (all - whole);
  auto tile_at = [&](int unit) { return unit <= whole ? unit : whole + (unit - whole + kRest - 1) / kRest; };
  const int x0 = tile_at(part_of.first(my_units)), x1 = tile_at(part_of.last(my_units));

  int t[RB], h[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = min(r0 + 32 * RB * wave + 32 * rb + l31, n_rows - 1);
    t[rb] = row / a.G;
    h[rb] = hk * a.G + row % a.G;
  }
  auto load_q = [&](bf16x8(&q)[NS], int rb) {
    const uint16_t *qp = static_cast<const uint16_t *>(a.q) + (g.row0 + t[rb]) * a.q_stride + h[rb] * D + 8 * half;
#pragma unroll
    for (int i = 0; i < NS; ++i) q[i] = *reinterpret_cast<const bf16x8 *>(qp + 16 * i);
#pragma unroll
    for (int i = 0; i < NS; ++i) arrived(q[i]);
  };
  const TileAddr<uint16_t, D> at;
  uint32_t *const odd = reinterpret_cast<uint32_t *>(lds + 4 * W::kTile);
  f32x16 o[RB][NB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[rb][b][i] = 0.f;
  float m[RB], l[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m[rb] = -INFINITY;
    l[rb] = 0.f;
  }

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds);
  const int64_t head = ((int64_t)s * a.Hk + hk) * a.capacity * D;
  // this wave's share of a tile of which n keys are there
  auto fetch = [&](const void *src, int64_t stride, int n, uint32_t dst) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int ld = i * 4 + wave, rr = ld * kRowsPerLoad + lane / R::kSlots;
      const int piece = min((lane % R::kSlots) ^ R::swz(rr), R::kPieces - 1);
      dma_to_lds(dst + ld * 1024, src, (uint32_t)min(rr, n - 1) * (uint32_t)(2 * stride) + 16 * piece);
    }
  };
  auto fetch_whole = [&](const void *cache, const void *tree, int x, uint32_t dst) {
    const bool in_tree = x >= cache_whole;
    const int64_t at = in_tree ? (g.row0 + (x - cache_whole) * 64) * a.kv_stride + hk * D : head + (int64_t)x * 64 * D;
    fetch(static_cast<const uint16_t *>(in_tree ? tree : cache) + at, in_tree ? a.kv_stride : D, 64, dst);
  };
  auto barrier = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  const int n = min(x1, whole) - x0;  // whole tiles of this part
  if (n > 0) {
    auto issue = [&](int i) {  // keys of tile i, values of tile i - 1
      if (i < n) fetch_whole(a.k_cache, a.k_tree, x0 + i, lds0 + (i & 1) * W::kTile);
      if (i >= 1 && i <= n) fetch_whole(a.v_cache, a.v_tree, x0 + i - 1, lds0 + (2 + ((i - 1) & 1)) * W::kTile);
    };
    // the keys of tile i + 1 and the values of tile i are there, and the places of those before them are free
    auto next_tile = [&](int i) {
      wait_vm<0>();
      barrier();
      issue(i + 2);
    };
    issue(0);
    wait_vm<0>();
    barrier();
    issue(1);
    const bool active = r0 + 32 * RB * wave < n_rows;
    if (!active) {  // rows past the end: this wave only carries its share of the tiles
      for (int i = 0; i < n; ++i) next_tile(i);
    } else {
      bf16x8 q[RB][NS];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) load_q(q[rb], rb);
#pragma unroll
      for (int e = 0; e < RB * NS; ++e) asm volatile("" : "+a"(q[e / NS][e % NS]));  // that is where they stay
      f32x16 sa[2][RB], sb[2][RB];  // scores [32-key block][32-row block] of the present and of the next tile
      TileAddr<uint16_t, D> in = at;
      in.move(lds0, lds0 + 2 * W::kTile);
      auto key = [&](int place, int step) { return in.key(place * W::kTile, step / NS, step % NS); };
      auto value = [&](int place, int step) { return in.values(place * W::kTile, step / NB / 2, step / NB % 2, step % NB); };
      float mx[RB];
      auto raise_max = [&]() {
        float top[RB];
        bool raise[RB], any = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          top[rb] = half_swap(mx[rb], true) * a.c;
          raise[rb] = top[rb] > m[rb] + 8.f;
          any |= raise[rb];
        }
        if (__builtin_expect(__ballot(any) != 0, 0)) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            const float alpha = raise[rb] ? __builtin_amdgcn_exp2f(m[rb] - top[rb]) : 1.f;
            m[rb] = raise[rb] ? top[rb] : m[rb];
            l[rb] *= alpha;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int i = 0; i < 16; ++i) o[rb][b][i] *= alpha;
          }
        }
      };
      // the scores `sc` of a tile whose values lie in place `at` into O, and the scores `next` of the tile behind it if there is one
      auto body = [&](f32x16(&sc)[2][RB], f32x16(&next)[2][RB], auto at_, auto has_next_) {
        constexpr int kAt = decltype(at_)::value;
        constexpr bool kNext = decltype(has_next_)::value;
        float mu[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) mu[rb] = m[rb] == -INFINITY ? 0.f : m[rb];
        uint32_t p[4][RB][4];  // weights as operands (rounded as in attend_tile): [16 keys][32-row block], two per word
        // weight e of kScores: keys 16 j .., row block rb
        auto weight = [&](int e) {
          const int j = e / (8 * RB), rb = e / 8 % RB, k = e % 8;
          const float v = __builtin_amdgcn_exp2f(fmaf(sc[j / 2][rb][8 * (j % 2) + k], a.c, -mu[rb]));
          sc[j / 2][rb][8 * (j % 2) + k] = v;
          l[rb] += v;
          if (k % 2 == 1) {
            typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
            typedef __attribute__((ext_vector_type(2))) float f32x2;
            const bf16x2 w = __builtin_convertvector(f32x2{sc[j / 2][rb][8 * (j % 2) + k - 1], v}, bf16x2);
            p[j][rb][k / 2] = __builtin_bit_cast(uint32_t, w);
          }
        };
        constexpr int kEarly = 3 * kScores / 4, kLate = kScores - kEarly;  // weights beside S, and beside the first half of O
        if constexpr (kNext) {
          bf16x8 kf[2] = {key(1 - kAt, 0), key(1 - kAt, 1)};
#pragma unroll
          for (int st = 0; st < kSteps1; ++st) {
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (RB == 2)
              score_mfma(next[st / NS][0], next[st / NS][1], kf[st % 2], q[0][st % NS], q[1][st % NS], st % NS == 0);
            else
              score_mfma(next[st / NS][0], kf[st % 2], q[0][st % NS], st % NS == 0);
            if (st + 2 < kSteps1) kf[st % 2] = key(1 - kAt, st + 2);
#pragma unroll
            for (int e = kEarly * st / kSteps1; e < kEarly * (st + 1) / kSteps1; ++e) weight(e);
          }
        } else {
#pragma unroll
          for (int e = 0; e < kEarly; ++e) weight(e);
        }
        float top[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) top[rb] = -INFINITY;
        bf16x8 vf[2] = {value(kAt, 0), value(kAt, 1)};
#pragma unroll
        for (int st = 0; st < kSteps2; ++st) {
          __builtin_amdgcn_sched_barrier(0);
          constexpr int kHalf = kSteps2 / 2;
          const int j = st / NB;
          if (kNext && st == kHalf) {  // from here on the next scores may be read
#pragma unroll
            for (int e = 0; e < 2 * RB; ++e) asm volatile("" : "+v"(next[e / RB][e % RB]));
          }
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            o[rb][st % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                vf[st % 2], __builtin_bit_cast(bf16x8, uint4{p[j][rb][0], p[j][rb][1], p[j][rb][2], p[j][rb][3]}),
                o[rb][st % NB], 0, 0, 0);
          if (st + 2 < kSteps2) vf[st % 2] = value(kAt, st + 2);
          if (st < kHalf) {
#pragma unroll
            for (int e = kEarly + kLate * st / kHalf; e < kEarly + kLate * (st + 1) / kHalf; ++e) weight(e);
          } else if (kNext) {
#pragma unroll
            for (int e = kScores * (st - kHalf) / kHalf; e < kScores * (st - kHalf + 1) / kHalf; ++e)
              top[e / 32] = fmaxf(top[e / 32], next[e / 16 % 2][e / 32][e % 16]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) mx[rb] = top[rb];
      };
      // scores of the first tile
#pragma unroll
      for (int st = 0; st < kSteps1; ++st) {
        if constexpr (RB == 2) score_mfma(sa[st / NS][0], sa[st / NS][1], key(0, st), q[0][st % NS], q[1][st % NS], st % NS == 0);
        else score_mfma(sa[st / NS][0], key(0, st), q[0][st % NS], st % NS == 0);
      }
#pragma unroll
      for (int e = 0; e < 2 * RB; ++e) score_wait(sa[e / RB][e % RB]);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        mx[rb] = sa[0][rb][0];
#pragma unroll
        for (int e = 1; e < 32; ++e) mx[rb] = fmaxf(mx[rb], sa[e / 16][rb][e % 16]);
      }
      raise_max();
      constexpr std::integral_constant<int, 0> even{};
      constexpr std::integral_constant<int, 1> odd{};
      int i = 0;
      for (; i + 2 < n; i += 2) {
        next_tile(i);
        body(sa, sb, even, std::true_type{});
        raise_max();
        next_tile(i + 1);
        body(sb, sa, odd, std::true_type{});
        raise_max();
      }
      next_tile(i);
      if (i + 1 < n) {
        body(sa, sb, even, std::true_type{});
        raise_max();
        next_tile(i + 1);
        body(sb, sa, odd, std::false_type{});
      } else {
        body(sa, sb, even, std::false_type{});
      }
    }
    barrier();  // all places are free
  }

  auto rest_base = [&](int x) { return 64 * (x >= whole + cache_rest ? x - cache_rest - cache_whole : cache_whole); };
  auto fetch_rest = [&](int x) {
    const bool in_tree = x >= whole + cache_rest;
    const int base = rest_base(x), keys = in_tree ? g.T : g.len;
    const int64_t stride = in_tree ? a.kv_stride : D;
    const int64_t first = in_tree ? (g.row0 + base) * a.kv_stride + hk * D : head + (int64_t)base * D;
    const uint32_t to = lds0 + (x & 1) * W::kTile;
    fetch(static_cast<const uint16_t *>(in_tree ? a.k_tree : a.k_cache) + first, stride, keys - base, to);
    fetch(static_cast<const uint16_t *>(in_tree ? a.v_tree : a.v_cache) + first, stride, keys - base, to + 2 * W::kTile);
  };
  const int y0 = max(x0, whole);
  if (y0 < x1) fetch_rest(y0);
  for (int x = y0; x < x1; ++x) {
    const bool in_tree = x >= whole + cache_rest;
    const int base = rest_base(x), keys = in_tree ? g.T : g.len, at_tile = (x & 1) * W::kTile;
    uint32_t *const my_odd = odd + 2 * (x & 1);
    wait_vm<0>();
    if (threadIdx.x < 2) my_odd[threadIdx.x] = 0;
    __syncthreads();  // the tile is there, and nobody reads the one before it any more
    if (x + 1 < x1) fetch_rest(x + 1);
    const bool clean = in_tree || row_not_finite<uint16_t, D>(lds + 2 * W::kTile + at_tile, keys - 1 - base);
    if (clean) {
      __syncthreads();  // everybody has looked
      clean_values<uint16_t, D, 64, 256>(lds + 2 * W::kTile + at_tile, my_odd);
      __syncthreads();
    }
    const int64_t vstride = in_tree ? a.kv_stride : D;
    const uint16_t *vg = static_cast<const uint16_t *>(in_tree ? a.v_tree : a.v_cache) +
                         (in_tree ? (g.row0 + base) * a.kv_stride + hk * D : head + (int64_t)base * D);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      bf16x8 q[NS];  // loaded again, so that the registers of the walk above are free here
      load_q(q, rb);
      attend_tile<uint16_t, D, 2>(a, g, at, in_tree, false, base, keys, t[rb], lds0 + at_tile, lds0 + 2 * W::kTile + at_tile,
                                  clean ? my_odd : nullptr, vg, vstride, q, o[rb], m[rb], l[rb]);
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    l[rb] = half_swap(l[rb], false);
    if (m[rb] == -INFINITY && l[rb] != 0.f) m[rb] = 0.f;  // scores that are all NaN: so is the row
    if (r0 + 32 * RB * wave + 32 * rb + l31 < n_rows)
      finish_row<uint16_t, D>(a, o[rb], m[rb], l[rb], slots, index, t[rb], h[rb], (size_t)(g.row0 + t[rb]) * a.H + h[rb], half, out,
                              lse, part, part_ml);
  }
}

// The parts of a row's keys joined: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.  D / 4 threads hold four elements each
// of a row; with PG > 1 that many groups of them share a row's parts and meet in LDS.  Nothing that is loaded depends on another
// load: what bounds a small combine is one trip to memory, and every part's statistics come with its values.
constexpr int kJoinGroups = 8;
template <typename T, int D, int PG>
__global__ __launch_bounds__(kJoinGroups *D / 4) void attention_combine_kernel(KeyArgs a, int slots,
                                                                              const float *__restrict__ part,
                                                                              const float2 *__restrict__ part_ml,
                                                                              const int32_t *__restrict__ first_of,
                                                                              T *__restrict__ out, float *__restrict__ lse) {
  constexpr int kCols = D / 4, kRows = kJoinGroups / PG;
  const int col = threadIdx.x % kCols, grp = threadIdx.x / kCols, pg = grp % PG;
  const int64_t r = (int64_t)blockIdx.x * kRows + grp / PG, n = (int64_t)a.max_tree * a.H;
  const int p0 = a.n_seq == 1 ? 0 : first_of[blockIdx.y], n_split = a.n_seq == 1 ? slots : first_of[blockIdx.y + 1] - p0;
  const size_t stride = n, first = (size_t)p0 * n + min(r, n - 1);
  float m = -INFINITY, l = 0.f;
  f32x4 o{0.f, 0.f, 0.f, 0.f};
  for (int i0 = pg; i0 < n_split; i0 += 4 * PG) {
    float2 ml[4];
    f32x4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const size_t at = (size_t)min(i0 + j * PG, n_split - 1) * stride + first;
      ml[j] = part_ml[at];
      v[j] = *reinterpret_cast<const f32x4 *>(part + at * D + 4 * col);
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = fmaxf(top, i0 + j * PG < n_split ? ml[j].x : -INFINITY);
    const float mu = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f(m - mu);
    l *= f0;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + j * PG < n_split && ml[j].x != -INFINITY) {  // a part without keys has left no values
        const float f = __builtin_amdgcn_exp2f(ml[j].x - mu);
        l = fmaf(f, ml[j].y, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[j][e], o[e]);
      }
    }
    m = top;
  }
  if constexpr (PG > 1) {
    __shared__ float2 ml[kJoinGroups];
    __shared__ f32x4 part_o[kJoinGroups][kCols];
    part_o[grp][col] = o;
    if (col == 0) ml[grp] = make_float2(m, l);
    __syncthreads();
    if (pg > 0) return;
    float top = m;
#pragma unroll
    for (int g = 1; g < PG; ++g) top = fmaxf(top, ml[grp + g].x);
    const float mu = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f(m - mu);
    l *= f0;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
    for (int g = 1; g < PG; ++g) {
      const float f = __builtin_amdgcn_exp2f(ml[grp + g].x - mu);
      l = fmaf(f, ml[grp + g].y, l);
      const f32x4 v = part_o[grp + g][col];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[e], o[e]);
    }
    m = top;
  }
  const SeqGeom g = seq_geom(a, blockIdx.y);
  if (r >= (int64_t)g.T * a.H) return;
  const size_t row = (size_t)g.row0 * a.H + r;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  Elem<T>::store4(out + row * D + 4 * col, f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv});
  if (lse && col == 0) lse[row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.69314718055994531f;
}

namespace {

constexpr int kPartRows = 1 << 16;    // most rows (x parts) of a launch whose keys are in parts: workgroups wanted x their rows
constexpr size_t kFirstBytes = 2048;  // first parts of up to kMaxShared sequences
constexpr int kFewStages = 512;       // up to as many stages of 32 keys in all every workgroup has one (both sides: head of this file)
constexpr int kWideSlots = 256;       // workgroups of the straight-line form that run at a time
// Up to here a workgroup of the combine has one row, whose parts its eight groups share (one token over 4000 entries 12.2 us, against 33.5
// with a group per row); above, a row per group (16 trees of 31 tokens x 32 heads, 4 parts: 168 us against 196).
constexpr int kJoinRows = 4096;

// Whether many rows take the straight-line form (heads of up to 128; longer ones always do).  It is ahead over long caches, by up to 17% (one
// tree of 2000 tokens x 32 heads over 128000 entries 3.90 ms against 4.60; 8 chains of 256 over 4800 173 us against 186) and behind where
// tiles that some row sees in part, start and end of a workgroup or an uneven last round weigh more: 16 chains of 256 without a cache 46.5
// us against 32.5, one tree of 2000 without a cache 195 against 113, 8 chains of 300 over 1200 109 against 89 (five row tiles:
// 320 workgroups on 256 compute units).  So it has to have 20 whole tiles of keys a part (511 tokens x 32 heads: even at 16, 79 us
// against 82 at 24), ten times the tiles of the tree (2000 tokens: 3% behind at eight times, 2% ahead at twelve), and the compute units busy:
// rounds at least three quarters full, and in a single round of a chain, whose last rows see the most keys, no less than 6 / 7 of the
// longest part's work on average (2000 tokens: 117 against 128 us with as many entries, equal with three times as many).
bool wide_pays(const KeyArgs &a, int64_t tile_rows) {
  const int64_t tiles = ((int64_t)a.max_tree * a.G + tile_rows - 1) / tile_rows, groups = (int64_t)a.n_seq * a.Hk * tiles;
  const int64_t parts = groups < kWideSlots ? kWideSlots / groups : 1, rounds = (groups + kWideSlots - 1) / kWideSlots;
  const int64_t len = a.max_len, tree = a.max_tree;
  if (a.tree_mask ? len < 10 * tree || len < 20 * 64 * parts : 2 * len + tree < 2 * 20 * 64 * parts) return false;
  if (rounds > 1) return 4 * groups >= 3 * kWideSlots * rounds;
  return a.tree_mask || 7 * (2 * len + tree) >= 6 * 2 * (len + tree);
}

// Parts of the keys (share_of): as many as give `target` workgroups, none without a stage; 0 where every sequence is one part.
int slots_of(const KeyArgs &a, int64_t row_tiles, int64_t target, int64_t stage_keys) {
  const int64_t stages = (a.max_len + stage_keys - 1) / stage_keys + (a.max_tree + stage_keys - 1) / stage_keys;
  int64_t n = target / (a.Hk * row_tiles);
  if (n > a.n_seq * stages) n = a.n_seq * stages;
  if (a.n_seq == 1 && n > kMaxParts) n = kMaxParts;
  return n <= a.n_seq || a.n_seq > kMaxShared ? 0 : (int)n;
}

// A launch of `kern` (rows of a workgroup, workgroups wanted, keys of a stage, threads, LDS) and the combine.
template <typename T, int D, typename Kern>
hipError_t run_kernel(Kern kern, int tile_rows, int target, int stage_keys, int threads, size_t smem, const KeyArgs &a, void *out,
                      float *lse, void *ws, hipStream_t st) {
  const int row_tiles = (int)(((int64_t)a.max_tree * a.G + tile_rows - 1) / tile_rows);
  const int slots = slots_of(a, row_tiles, target, stage_keys);
  if (smem > 64 * 1024) {  // beyond the default limit of a launch
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
  }
  const int64_t rows = (int64_t)a.max_tree * a.H;
  int32_t *first_of = static_cast<int32_t *>(ws);
  float *part = reinterpret_cast<float *>(static_cast<char *>(ws) + kFirstBytes);
  float2 *ml = reinterpret_cast<float2 *>(part + (size_t)slots * rows * D);
  const int64_t groups = (int64_t)a.Hk * (slots == 0 ? a.n_seq : slots);
  kern<<<(unsigned)((groups + 7) / 8 * 8 * row_tiles), threads, smem, st>>>(a, row_tiles, slots, static_cast<T *>(out), lse, part, ml,
                                                                            first_of);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || slots == 0) return e;
  if (rows * a.n_seq <= kJoinRows)
    attention_combine_kernel<T, D, kJoinGroups><<<dim3((unsigned)rows, a.n_seq), kJoinGroups * D / 4, 0, st>>>(
        a, slots, part, ml, first_of, static_cast<T *>(out), lse);
  else
    attention_combine_kernel<T, D, 1><<<dim3((unsigned)((rows + kJoinGroups - 1) / kJoinGroups), a.n_seq), kJoinGroups * D / 4,
                                        0, st>>>(a, slots, part, ml, first_of, static_cast<T *>(out), lse);
  return hipGetLastError();
}

template <typename T, int D, int WR, int WK, int KB>
hipError_t run_attention(const KeyArgs &a, void *out, float *lse, void *ws, hipStream_t st) {
  constexpr size_t stages = (size_t)2 * 2 * 32 * KB * WK * Rows<T, D>::kBytes + 2 * 4 * KB * WK;
  constexpr size_t join = WK > 1 ? sizeof(float2) * 32 * WR * WK + sizeof(float) * (WK - 1) * WR * 32 * D : 0;
  constexpr size_t smem = stages > join ? stages : join;
  static_assert(smem <= 160 * 1024, "LDS of a compute unit");
  static_assert(512 * 32 * WR <= kPartRows, "the workspace has room for the parts");
  return run_kernel<T, D>(tree_attention_kernel<T, D, WR, WK, KB>, 32 * WR, smem <= 80 * 1024 ? 512 : 256, 32 * KB * WK, 64 * WR * WK,
                          smem, a, out, lse, ws, st);
}

template <typename T, int D>
hipError_t run_shape(const KeyArgs &a, void *out, float *lse, void *ws, hipStream_t st) {
  typedef AttnShape<T, D> S;
  const int64_t rows = (int64_t)a.max_tree * a.G;
  // few keys: a stage of 32 keys for every workgroup, whose waves then have nothing to join
  const bool few = (int64_t)a.n_seq * a.Hk * ((a.max_len + 31) / 32 + (a.max_tree + 31) / 32) <= kFewStages;
  if (rows <= 32)
    return few ? run_attention<T, D, 1, 1, 1>(a, out, lse, ws, st) : run_attention<T, D, 1, S::kWk1, 1>(a, out, lse, ws, st);
  if (rows <= 64)
    return few ? run_attention<T, D, 2, 1, 1>(a, out, lse, ws, st) : run_attention<T, D, 2, S::kWk2, 1>(a, out, lse, ws, st);
  if constexpr (sizeof(T) == 2) {
    if (D <= 128 ? rows > 128 && wide_pays(a, WideShape<D>::kRows) : rows > 64)
      return run_kernel<T, D>(tree_attention_wide_kernel<D>, WideShape<D>::kRows, kWideSlots, 64, 256, WideShape<D>::kLds, a, out, lse, ws,
                              st);
  }
  if constexpr (sizeof(T) == 4 || D <= 128) return run_attention<T, D, 4, 1, S::kKb4>(a, out, lse, ws, st);
  return hipErrorInvalidValue;  // not reached: longer bf16 heads have taken one of the forms above
}

template <typename T>
hipError_t run_type(const moespec_attn_desc &ds, const KeyArgs &a, void *out, float *lse, void *ws, hipStream_t st) {
  switch (ds.head_dim) {
    case 64: return run_shape<T, 64>(a, out, lse, ws, st);
    case 96: return run_shape<T, 96>(a, out, lse, ws, st);
    case 128: return run_shape<T, 128>(a, out, lse, ws, st);
    case 192: return run_shape<T, 192>(a, out, lse, ws, st);
    default: return run_shape<T, 256>(a, out, lse, ws, st);
  }
}

}  // namespace

// The parts of every row there may be: no more than stages of 32 keys or more in all sequences, and where there are parts at all at most
// kPartRows rows of workgroups.  Neither bound grows where a call gets smaller.
size_t tree_attention_ws(const moespec_attn_desc &ds, int64_t n_seq, int64_t max_tree, int64_t max_len) {
  const int64_t stages = (max_len + 31) / 32 + (max_tree + 31) / 32, most = kPartRows, seq = n_seq < kMaxShared ? n_seq : kMaxShared;
  int64_t rows = max_tree * ds.n_heads;
  rows = rows > most ? most : rows * (stages * seq < most ? stages * seq : most);
  return kFirstBytes + (size_t)(rows < most ? rows : most) * (sizeof(float) * ds.head_dim + sizeof(float2));
}

hipError_t launch_tree_attention(const moespec_attn_desc &ds, const KeyArgs &a, void *out, float *lse, void *ws,
                                 hipStream_t st) {
  return ds.dtype == MOESPEC_BF16 ? run_type<uint16_t>(ds, a, out, lse, ws, st) : run_type<float>(ds, a, out, lse, ws, st);
}

}  // namespace moespec
