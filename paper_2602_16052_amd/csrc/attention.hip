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
#include <math.h>

#include "attention.h"

namespace moespec {

template <typename T, int D>
struct AttnShape {
  static constexpr int kRow = Rows<T, D>::kBytes;
  static constexpr int kWk1 = 1024 / kRow < 4 ? 1024 / kRow : 4;  // key waves for up to 32 rows: a stage of up to 64 KB
  static constexpr int kWk2 = 1024 / kRow < 2 ? 1024 / kRow : 2;  // ... for up to 64
  static constexpr int kKb4 = kRow <= 256 && sizeof(T) == 2 ? 2 : 1;  // 32-key blocks of a wave with 128 rows a workgroup
};

template <typename T, int D, int WR, int WK, int KB>
__global__ __launch_bounds__(64 * WR * WK, (D <= 128 ? 2 : 1)) void tree_attention_kernel(
    KeyArgs a, int row_tiles, int n_split, T *__restrict__ out, float *__restrict__ lse, float *__restrict__ part,
    float2 *__restrict__ part_ml) {
  typedef Rows<T, D> R;
  typedef typename Frag<T>::type frag;
  constexpr int NW = WR * WK, kStageKeys = 32 * KB * WK, kTile = kStageKeys * R::kBytes, kStage = 2 * kTile;
  constexpr int kRowsPerLoad = 64 / R::kSlots, kLoads = kStageKeys / kRowsPerLoad, NB = D / 32, NS = R::kPieces / 2;
  static_assert(kLoads % NW == 0, "every wave issues as many loads");
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave % WR, wk = wave / WR;
  const int l31 = lane & 31, half = lane >> 5;
  // row tiles that share keys are neighbours on one XCD (workgroup b runs on XCD b mod 8)
  const int slot = blockIdx.x / 8, group = slot / row_tiles * 8 + (int)(blockIdx.x % 8), tile = slot % row_tiles;
  if (group >= a.n_seq * a.Hk * n_split) return;
  const int split = group % n_split, hk = group / n_split % a.Hk, s = group / n_split / a.Hk;
  const SeqGeom g = seq_geom(a, s);
  const int n_rows = g.T * a.G, r0 = tile * 32 * WR;
  if (r0 >= n_rows) return;

  // stages: those of the cache, then those of the tree (of a chain only up to the last row's token)
  const int ct = (g.len + kStageKeys - 1) / kStageKeys, all = ct + (g.T + kStageKeys - 1) / kStageKeys;
  const int last_t = (min(r0 + 32 * WR, n_rows) - 1) / a.G;
  const int tt = a.tree_mask ? all - ct : last_t / kStageKeys + 1;
  const int chunk = (all + n_split - 1) / n_split;
  const int st0 = split * chunk, st1 = min(st0 + chunk, ct + tt);

  const int row = min(r0 + 32 * wr + l31, n_rows - 1), t = row / a.G, h = hk * a.G + row % a.G;
  const size_t orow = (size_t)(g.row0 + t) * a.H + h;
  const bool row_ok = r0 + 32 * wr + l31 < n_rows;

  frag q[NS];
  {
    const T *qp = static_cast<const T *>(a.q) + (g.row0 + t) * a.q_stride + h * D + half * R::kPieceElems;
#pragma unroll
    for (int i = 0; i < NS; ++i) q[i] = *reinterpret_cast<const frag *>(qp + 2 * i * R::kPieceElems);
  }
  f32x16 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds);
  const size_t head = ((size_t)s * a.Hk + hk) * a.capacity * D;
  auto issue = [&](int st, int buf) {
    const bool tree = st >= ct;
    const int base = (tree ? st - ct : st) * kStageKeys, n = tree ? g.T : g.len;
    const int64_t stride = tree ? a.kv_stride : D;
    const int64_t at = tree ? (g.row0 + base) * a.kv_stride + hk * D : (int64_t)head + (int64_t)base * D;
    const T *kp = static_cast<const T *>(tree ? a.k_tree : a.k_cache) + at;
    const T *vp = static_cast<const T *>(tree ? a.v_tree : a.v_cache) + at;
#pragma unroll
    for (int i = 0; i < kLoads / NW; ++i) {
      const int ld = i * NW + wave, rr = ld * kRowsPerLoad + lane / R::kSlots;
      const int piece = min((lane % R::kSlots) ^ R::swz(rr), R::kPieces - 1);  // padding slots repeat a piece, and are not read
      // keys past the end repeat the last one: their scores are masked, and their weights of 0 must meet numbers
      const uint32_t off = (uint32_t)min(rr, n - 1 - base) * (uint32_t)(stride * sizeof(T)) + 16 * piece;
      dma_to_lds(lds0 + buf * kStage + ld * 1024, kp, off);
      dma_to_lds(lds0 + buf * kStage + kTile + ld * 1024, vp, off);
    }
  };

  if (st0 < st1) issue(st0, 0);
  for (int st = st0; st < st1; ++st) {
    const int buf = (st - st0) & 1;
    wait_vm<0>();
    asm volatile("" ::: "memory");
    __syncthreads();  // the stage has arrived, everybody's part of it, and nobody reads the other one any more
    if (st + 1 < st1) issue(st + 1, buf ^ 1);
    const unsigned char *kt = lds + buf * kStage + wk * KB * 32 * R::kBytes, *vt = kt + kTile;
    const bool tree = st >= ct;
    const int base = (tree ? st - ct : st) * kStageKeys + wk * KB * 32, n = tree ? g.T : g.len;

    f32x16 sc[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const frag kf =
            *reinterpret_cast<const frag *>(kt + (32 * kb + l31) * R::kBytes + (((2 * i + half) ^ R::swz(l31)) << 4));
        sc[kb] = Frag<T>::mma(kf, q[i], sc[kb]);
      }
    }
    // A stage inside the cache, or in front of every row's own token in a chain, is seen whole.
    uint32_t word[KB];
    const bool whole = base + 32 * KB <= n && (!tree || (a.tree_mask == nullptr && base + 32 * KB - 1 <= r0 / a.G));
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
    // The maximum is only raised when it is passed by more than 2^8: until then the weights stay below 2^8, in fp32 and in
    // bf16 as exact as below 1, and O is not rescaled.
    const bool raise = mx > m + 8.f;
    if (__ballot(raise) != 0) {
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

    // A weight of 0 times a NaN or an infinity would reach a token that does not see that key.  Keys of the tree with such a
    // value are found first; their values enter the product as 0 and are added to the rows that see them.
    uint32_t odd[KB];
    uint32_t any_odd = 0;
    if (tree && !whole) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        uint32_t bad = 0;
#pragma unroll
        for (int p = 0; p < NS; ++p) {
          const uint4 v = *reinterpret_cast<const uint4 *>(vt + (32 * kb + l31) * R::kBytes + (((2 * p + half) ^ R::swz(l31)) << 4));
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            bad |= (w[e] & 0x7f800000u) == 0x7f800000u;
            if (sizeof(T) == 2) bad |= (w[e] & 0x7f80u) == 0x7f80u;
          }
        }
        const unsigned long long b = __ballot(bad != 0);
        odd[kb] = (uint32_t)b | (uint32_t)(b >> 32);
        any_odd |= odd[kb];
      }
    }
    auto values = [&](auto clean) {
      constexpr bool kClean = decltype(clean)::value;  // non-finite values replaced by 0
      if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) bf16x4 lds4;
        const int i16 = lane & 15, vrow = 4 * half + (i16 >> 2), low = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            bf16x8 p;
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = (__bf16)sc[kb][8 * j + i];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              const int ra = 32 * kb + 16 * j + vrow, rb = ra + 8;
              bf16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                  (lds4 *)(vt + ra * R::kBytes + (((4 * b + low) ^ R::swz(ra)) << 4) + 8 * (i16 & 1)));
              bf16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                  (lds4 *)(vt + rb * R::kBytes + (((4 * b + low) ^ R::swz(rb)) << 4) + 8 * (i16 & 1)));
              bf16x8 v = __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7);
              if constexpr (kClean) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if ((__float_as_uint((float)v[e]) & 0x7f800000u) == 0x7f800000u) v[e] = (__bf16)0.f;
              }
              o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, o[b], 0, 0, 0);
            }
          }
      } else {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int vr = 32 * kb + acc_row(i, half);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              float v = *reinterpret_cast<const float *>(vt + vr * R::kBytes +
                                                         (((8 * b + (l31 >> 2)) ^ R::swz(vr)) << 4) + 4 * (l31 & 3));
              if constexpr (kClean)
                if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) v = 0.f;
              o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, sc[kb][i], o[b], 0, 0, 0);
            }
          }
      }
    };
    if (any_odd == 0) {
      values(std::false_type{});
    } else {
      values(std::true_type{});
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        for (uint32_t left = odd[kb]; left != 0; left &= left - 1) {
          const int j = __builtin_ctz(left), vr = 32 * kb + j;
          const bool seen = (word[kb] >> j) & 1u;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int e = 32 * b + acc_row(i, half);
              const float v = Elem<T>::load(reinterpret_cast<const T *>(
                  vt + vr * R::kBytes + ((e / R::kPieceElems ^ R::swz(vr)) << 4) + sizeof(T) * (e % R::kPieceElems)));
              if (seen && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[b][i] += v;
            }
        }
    }
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
  if (!row_ok) return;
  if (n_split == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        Elem<T>::store4(out + orow * D + 32 * b + acc_row(i, half),
                        f32x4{o[b][i] * inv, o[b][i + 1] * inv, o[b][i + 2] * inv, o[b][i + 3] * inv});
    if (lse && half == 0) lse[orow] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.69314718055994531f;
  } else {
    const size_t at = ((size_t)split * a.n_seq + s) * a.max_tree * a.H + (size_t)t * a.H + h;
    if (half == 0) part_ml[at] = make_float2(m, l);
    if (m == -INFINITY) return;  // the combine passes it over
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4 *>(part + at * D + 32 * b + acc_row(i, half)) =
            f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
  }
}

// The parts of a row's keys joined: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.  One wave per row, lane i has the weight of
// parts i, i + 64, ...
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_combine_kernel(KeyArgs a, int n_split, const float *__restrict__ part,
                                                                const float2 *__restrict__ part_ml, T *__restrict__ out,
                                                                float *__restrict__ lse) {
  constexpr int NC = (D + 63) / 64, NP = kMaxSplits / 64;
  const int lane = threadIdx.x & 63;
  const SeqGeom g = seq_geom(a, blockIdx.y);
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= (int64_t)g.T * a.H) return;
  const size_t row = (size_t)g.row0 * a.H + r, stride = (size_t)a.n_seq * a.max_tree * a.H;
  const size_t first = (size_t)blockIdx.y * a.max_tree * a.H + r;
  float w[NP], m = -INFINITY, l = 0.f;
  float2 ml[NP];
#pragma unroll
  for (int u = 0; u < NP; ++u) {
    const int i = lane + 64 * u;
    ml[u] = i < n_split ? part_ml[i * stride + first] : make_float2(-INFINITY, 0.f);
    m = fmaxf(m, ml[u].x);
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, kWave));
  const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int u = 0; u < NP; ++u) {
    w[u] = __builtin_amdgcn_exp2f(ml[u].x - mu);
    l = fmaf(w[u], ml[u].y, l);
  }
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) l += __shfl_xor(l, x, kWave);
  float o[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) o[c] = 0.f;
#pragma unroll
  for (int u = 0; u < NP; ++u) {
    const uint64_t live = __ballot(ml[u].x != -INFINITY);
    const int top = min(64, n_split - 64 * u);
    for (int i0 = 0; i0 < top; i0 += 8) {  // eight parts in flight
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = min(i0 + j, top - 1);
        const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w[u]), i));
        const bool used = i0 + j < top && ((live >> i) & 1);  // a part without keys has left nothing there
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int e = min(lane + 64 * c, D - 1);
          const float v = part[((64 * u + i) * stride + first) * D + e];
          o[c] = used ? fmaf(f, v, o[c]) : o[c];
        }
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int e = lane + 64 * c;
    if (D % 64 == 0 || e < D) Elem<T>::store(out + row * D + e, o[c] * inv);
  }
  if (lse && lane == 0) lse[row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.69314718055994531f;
}

namespace {

constexpr int kAttnTarget = 512;  // workgroups wanted

// Row tiles and parts of the keys.  stage_keys: keys of a stage.
struct AttnPlan {
  int wr, row_tiles, n_split;
};
int64_t stages_of(int64_t max_tree, int64_t max_len) { return (max_len + 63) / 64 + (max_tree + 63) / 64; }
AttnPlan plan_of(const moespec_attn_desc &ds, int64_t n_seq, int64_t max_tree, int64_t max_len) {
  const int64_t rows = max_tree * (ds.n_heads / ds.n_kv_heads);
  AttnPlan p;
  p.wr = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  p.row_tiles = (int)((rows + 32 * p.wr - 1) / (32 * p.wr));
  const int64_t groups = n_seq * ds.n_kv_heads * p.row_tiles;
  const int64_t stages = stages_of(max_tree, max_len);
  int64_t n = kAttnTarget / groups;
  n = n < stages ? n : stages;
  n = n < kMaxSplits ? n : kMaxSplits;
  p.n_split = (int)(n > 1 ? n : 1);
  return p;
}

template <typename T, int D, int WR, int WK, int KB>
hipError_t run_attention(const KeyArgs &a, const AttnPlan &p, void *out, float *lse, void *ws, hipStream_t st) {
  constexpr size_t stages = (size_t)2 * 2 * 32 * KB * WK * Rows<T, D>::kBytes;
  constexpr size_t join = WK > 1 ? sizeof(float2) * 32 * WR * WK + sizeof(float) * (WK - 1) * WR * 32 * D : 0;
  constexpr size_t smem = stages > join ? stages : join;
  static_assert(smem <= 160 * 1024, "LDS of a compute unit");
  auto kern = tree_attention_kernel<T, D, WR, WK, KB>;
  if (smem > 64 * 1024) {  // beyond the default limit of a launch
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
  }
  float *part = static_cast<float *>(ws);
  float2 *ml = reinterpret_cast<float2 *>(part + (size_t)p.n_split * a.n_seq * a.max_tree * a.H * D);
  const int groups = a.n_seq * a.Hk * p.n_split;
  kern<<<(groups + 7) / 8 * 8 * p.row_tiles, 64 * WR * WK, smem, st>>>(a, p.row_tiles, p.n_split, static_cast<T *>(out), lse,
                                                                       part, ml);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  attention_combine_kernel<T, D><<<dim3((unsigned)(((int64_t)a.max_tree * a.H + 3) / 4), a.n_seq), 256, 0, st>>>(
      a, p.n_split, part, ml, static_cast<T *>(out), lse);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t run_shape(const KeyArgs &a, const AttnPlan &p, void *out, float *lse, void *ws, hipStream_t st) {
  typedef AttnShape<T, D> S;
  if (p.wr == 1) return run_attention<T, D, 1, S::kWk1, 1>(a, p, out, lse, ws, st);
  if (p.wr == 2) return run_attention<T, D, 2, S::kWk2, 1>(a, p, out, lse, ws, st);
  return run_attention<T, D, 4, 1, S::kKb4>(a, p, out, lse, ws, st);
}

template <typename T>
hipError_t run_type(const moespec_attn_desc &ds, const KeyArgs &a, const AttnPlan &p, void *out, float *lse, void *ws,
                    hipStream_t st) {
  switch (ds.head_dim) {
    case 64: return run_shape<T, 64>(a, p, out, lse, ws, st);
    case 96: return run_shape<T, 96>(a, p, out, lse, ws, st);
    case 128: return run_shape<T, 128>(a, p, out, lse, ws, st);
    case 192: return run_shape<T, 192>(a, p, out, lse, ws, st);
    default: return run_shape<T, 256>(a, p, out, lse, ws, st);
  }
}

}  // namespace

// The parts of every row there may be: n_split <= min(kMaxSplits, stages), and where n_split > 1 there are at most
// kAttnTarget workgroups of up to 128 rows.  Neither bound falls where a call gets smaller.
size_t tree_attention_ws(const moespec_attn_desc &ds, int64_t n_seq, int64_t max_tree, int64_t max_len) {
  const int64_t stages = stages_of(max_tree, max_len), most = (int64_t)kAttnTarget * 128;
  int64_t rows = n_seq * max_tree * ds.n_heads;
  rows = rows > most ? most : rows * (stages < kMaxSplits ? stages : kMaxSplits);
  return (size_t)(rows < most ? rows : most) * (sizeof(float) * ds.head_dim + sizeof(float2));
}

hipError_t launch_tree_attention(const moespec_attn_desc &ds, const KeyArgs &a, void *out, float *lse, void *ws,
                                 hipStream_t st) {
  const AttnPlan p = plan_of(ds, a.n_seq, a.max_tree, a.max_len);
  return ds.dtype == MOESPEC_BF16 ? run_type<uint16_t>(ds, a, p, out, lse, ws, st) : run_type<float>(ds, a, p, out, lse, ws, st);
}

}  // namespace moespec
