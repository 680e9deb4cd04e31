// The attention weight that every key received: w_j = sum over rows of row_weight 2^(c q.K_j - lse / ln 2).
//
// The softmax statistics of the rows are known (lse), so a column sum needs nothing from other keys: a wave holds its 32 KB keys
// as matrix operands in registers and walks over the rows, whose tiles of 32 come through a ring of four places in LDS.  S^T = K Q^T has
// a row of queries per lane, and the weights of a key add up in one register per lane; the 32 lanes are summed once at the end.  A
// workgroup is the only writer of its keys, or of its part of the rows, which a second launch adds up in order.
//
// What bounds it: for many rows the exponentials and the two multiply-adds per score, which run beside the next tile's matrix
// instructions: 4 trees of 127 tokens x 8 heads, caches of 32749 down to 20469 entries, 167 to 175 us (530 to 555 TFLOP/s; 193 us with
// the one behind the other).  Over 32749 entries each the VALU is busy for 56% of the cycles, the matrix cores for 32%.  For few rows
// the launch and one trip to memory: 63 tokens x 16 heads over 4093 entries 10 us for 17 MB of keys.
#include <float.h>
#include <math.h>

#include "attention.h"

namespace moespec {

constexpr int kWeightWaves = 4;
constexpr int kNanClass = 0x003, kZeroClass = 0x060, kInfinityClass = 0x204;  // of v_cmp_class

template <typename T, int D>
struct WeightShape {
  // 32-key blocks held by a wave.  Two where the registers allow it: every row operand that is read is multiplied twice (4 trees of
  // 127 tokens, 32749 entries: 172 us against 192; fp32 heads of 64, 63 tokens x 8 over 8192: 37 against 42); one would be faster for one
  // or two tiles of rows (63 tokens over 4093 entries: 8.2 us against 9.3).
  static constexpr int kKb = D * (int)sizeof(T) <= 256 ? 2 : 1;
  static constexpr int kKeys = 32 * kKb * kWeightWaves;
  static constexpr int kRing = 4, kLds = kRing * (32 * Rows<T, D>::kBytes + 512 * kWeightWaves);
};

// 64 lanes x 16 bytes from their own addresses to LDS bytes [lds, lds + 1024) (see dma_to_lds).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma_to_lds_from(uint32_t lds, const void *p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(
                   __builtin_amdgcn_readfirstlane(lds)),
               "v"(p)
               : "m0", "memory");
}
// The same with 4 bytes per lane.
__device__ __forceinline__ void dma_word_to_lds_from(uint32_t lds, const void *p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)),
               "v"(p)
               : "m0", "memory");
}
#pragma clang diagnostic pop

template <typename T, int D>
__global__ __launch_bounds__(64 * kWeightWaves, 2) void cache_weights_kernel(
    KeyArgs a, int tree_tiles, int tiles, int row_splits, const float *__restrict__ lse, const float *__restrict__ row_weight,
    float decay, const float *w_in, float *w_out, float *__restrict__ tree_w, float *__restrict__ part) {
  typedef Rows<T, D> R;
  typedef typename Frag<T>::type frag;
  constexpr int KB = WeightShape<T, D>::kKb, kKeys = WeightShape<T, D>::kKeys, NS = R::kPieces / 2;
  constexpr int kTile = 32 * R::kBytes, kRowsPerLoad = 64 / R::kSlots, kLoads = 32 / kRowsPerLoad;
  constexpr int kRing = WeightShape<T, D>::kRing, kStage = kTile + 512 * kWeightWaves;  // rows, and 128 words for every wave
  static_assert(kLoads % kWeightWaves == 0, "every wave issues as many loads");
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l31 = lane & 31, half = lane >> 5;
  // tiles of the trees, which take longer, first; the heads and sequences of a tile side by side
  const int n_sh = a.n_seq * a.Hk, rs = blockIdx.x % row_splits, sh = blockIdx.x / row_splits % n_sh;
  const int tile = blockIdx.x / row_splits / n_sh, hk = sh % a.Hk, s = sh / a.Hk;
  const SeqGeom g = seq_geom(a, s);
  const bool tree = tile < tree_tiles;
  const int base = (tree ? tile : tile - tree_tiles) * kKeys, n = tree ? g.T : g.len;
  if (base >= n) return;
  const int n_rows = g.T * a.G, blocks = (n_rows + 31) / 32, chunk = (blocks + row_splits - 1) / row_splits;
  const int b0 = rs * chunk, b1 = min(b0 + chunk, blocks);

  frag k[KB][NS];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const int key = min(base + (wave * KB + kb) * 32 + l31, n - 1);  // keys past the end are not written
    const T *kp = static_cast<const T *>(tree ? a.k_tree : a.k_cache) + half * R::kPieceElems +
                  (tree ? (g.row0 + key) * a.kv_stride + hk * D
                        : (((int64_t)s * a.Hk + hk) * a.capacity + key) * (int64_t)D);
#pragma unroll
    for (int i = 0; i < NS; ++i) k[kb][i] = *reinterpret_cast<const frag *>(kp + 2 * i * R::kPieceElems);
  }
  float w[KB][16];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) w[kb][i] = 0.f;

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds);
  // A walk over every 32nd row from `row`, without divisions and products: where something that belongs to the row lies (per_token
  // bytes a token, per_head a query head of it), the last row's place, and the row's place among the G rows of its token.
  const int step_t = 32 / a.G, step_r = 32 % a.G;
  struct Walk {
    const char *p, *last;
    int64_t step, wrap;
    int row, r;
  };
  auto walk = [&](const void *first, int64_t per_token, int64_t per_head, int row) {
    const char *f = static_cast<const char *>(first) + g.row0 * per_token + hk * a.G * per_head;
    return Walk{f + row / a.G * per_token + row % a.G * per_head, f + (g.T - 1) * per_token + (a.G - 1) * per_head,
                step_t * per_token + step_r * per_head, per_token - a.G * per_head, row, row % a.G};
  };
  auto forward = [&](Walk &w) {  // where it was; rows past the end are the last one
    const char *p = w.row < n_rows ? w.p : w.last;
    w.row += 32;
    w.r += step_r;
    const bool wrap = w.r >= a.G;
    w.r -= wrap ? a.G : 0;
    w.p += wrap ? w.step + w.wrap : w.step;
    return p;
  };
  // this lane's share of a tile of 32 rows, and (lanes 0-31) the row's lse or (others) its weight
  Walk src[kLoads / kWeightWaves];
#pragma unroll
  for (int i = 0; i < kLoads / kWeightWaves; ++i) {
    const int rr = (i * kWeightWaves + wave) * kRowsPerLoad + lane / R::kSlots;
    src[i] = walk(a.q, a.q_stride * sizeof(T), D * sizeof(T), 32 * b0 + rr);
    const int piece = 16 * min((lane % R::kSlots) ^ R::swz(rr), R::kPieces - 1);
    src[i].p += piece;
    src[i].last += piece;
  }
  Walk stat = half == 1 && row_weight ? walk(row_weight, 4, 0, 32 * b0 + l31) : walk(lse, 4 * (int64_t)a.H, 4, 32 * b0 + l31);
  // in a tile of a tree the words of its mask with this wave's keys (lanes 0-31 the first, the others the second)
  const bool masks = tree && a.tree_mask != nullptr;
  Walk seen = masks ? walk(a.tree_mask + min(base / 32 + wave * KB + (KB > 1 ? half : 0), a.words - 1), 4 * (int64_t)a.words, 0,
                           32 * b0 + l31)
                    : stat;
  auto issue = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kLoads / kWeightWaves; ++i)
      dma_to_lds_from(lds0 + buf * kStage + (i * kWeightWaves + wave) * 1024, forward(src[i]));
    dma_word_to_lds_from(lds0 + buf * kStage + kTile + wave * 512, forward(stat));
    if (masks) dma_word_to_lds_from(lds0 + buf * kStage + kTile + wave * 512 + 256, forward(seen));
  };
  uint32_t q_at[NS < 8 ? NS : 8];
#pragma unroll
  for (int i = 0; i < (NS < 8 ? NS : 8); ++i) q_at[i] = lds0 + l31 * R::kBytes + (((2 * i + half) ^ R::swz(l31)) << 4);
  constexpr int kCount = kLoads / kWeightWaves + 1;  // fetches of a wave for a tile
  for (int i = 0; i < kRing; ++i)
    if (b0 + i < b1) issue(i);
#pragma unroll
  for (int i = 0; i < KB * NS; ++i) arrived(k[i / NS][i % NS]);
  // Tile b is there (the first time also the one behind it: four have been fetched, two may be on their way), and every wave has read all
  // of tile b - 1, whose place is filled next.
  auto tile_there = [&](int b) {
    const int later = min(b1 - 1 - b, 2);
    if (later <= 0) wait_vm<0>();
    else if (!masks && later == 2) wait_vm<2 * kCount>();
    else if (!masks) wait_vm<kCount>();
    else if (later == 2) wait_vm<2 * kCount + 2>();
    else wait_vm<kCount + 1>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // A step multiplies one operand of the rows by this wave's keys; operands are read in groups, the next one while this one is
  // multiplied.
  typedef __attribute__((address_space(3))) frag lds_frag;
  constexpr int kGroup = 2;
  static_assert(NS % kGroup == 0, "whole groups");
  frag q[2][kGroup];
  auto read = [&](int buf, int n) {
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
      q[n & 1][i] = *(lds_frag *)(uintptr_t)(q_at[(n * kGroup + i) % 8] + buf * kStage + (n * kGroup + i) / 8 * 256);
  };
  // Scores of tile b + 1 (place buf) into next, beside the exponentials of those of the tile before it (sc, with shift and
  // weight of this lane's row), where there are such.
  float shift = 0.f, weight = 0.f;
  auto step = [&](f32x16(&sc)[KB], f32x16(&next)[KB], int buf, auto with_next_, auto with_sc_) {
    constexpr bool kNext = decltype(with_next_)::value, kSc = decltype(with_sc_)::value;
    constexpr int kAll = 16 * KB;
    auto add = [&](int e) {
      w[e / 16][e % 16] = fmaf(weight, __builtin_amdgcn_exp2f(fmaf(sc[e / 16][e % 16], a.c, -shift)), w[e / 16][e % 16]);
      asm volatile("" : "+v"(w[e / 16][e % 16]));  // here, and not behind the matrix instructions where the compiler would move it
    };
    if constexpr (kNext) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) next[kb][i] = 0.f;
      read(buf, 0);
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        if (n % kGroup == 0 && n + kGroup < NS) read(buf, n / kGroup + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) next[kb] = Frag<T>::mma(k[kb][n], q[n / kGroup & 1][n % kGroup], next[kb]);
        if constexpr (kSc)
#pragma unroll
          for (int e = kAll * n / NS; e < kAll * (n + 1) / NS; ++e) add(e);
      }
      __builtin_amdgcn_sched_barrier(0);
    } else {
#pragma unroll
      for (int e = 0; e < kAll; ++e) add(e);
    }
  };
  // this lane's row of tile b, and the masks of its scores
  auto row_of = [&](f32x16(&sc)[KB], int b, int buf) {
    const float *st = reinterpret_cast<const float *>(lds + buf * kStage + kTile + wave * 512);
    const int row = 32 * b + l31;
    const float ls = st[l31], rw = row_weight ? st[32 + l31] : 1.f;
    // The exponent c s - u lse is u (scale s - lse) whatever c was rounded to.  u lse is large where the exponent is small, and rounded
    // to as many bits: what that loses is the same for all keys of the row, and goes into its weight (2^-rest to first order).
    shift = ls * a.u;
    const float rest = fmaf(ls, a.u_rest, fmaf(ls, a.u, -shift));
    weight = rw * fmaf(rest, -0.69314718055994531f, 1.f);
    // few rows are none of the common ones: past the end, of weight 0, not finite (or so large that rest is not small)
    const bool past = row >= n_rows, far = !(fabsf(ls) < 0x1p20f);
    const bool special = __builtin_amdgcn_classf(rw, kNanClass | kInfinityClass | kZeroClass);
    if (__builtin_expect((__ballot(past) | __ballot(far) | __ballot(special)) != 0, 0)) {
      asm volatile("");  // a branch: as selections in the common path they would double its instructions
      const bool common = !past && !far && !special;
      const bool ok = !past && ls != -INFINITY && rw != 0.f;  // others have no part, whatever they hold
      shift = common ? shift : ok ? fmaxf(shift, -FLT_MAX) : 0.f;
      weight = common ? weight : !ok ? 0.f : ls != ls ? NAN : rw;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb][i] = ok ? sc[kb][i] : -INFINITY;
    }
    if (tree) {  // likewise
      asm volatile("");
      // A lse of NaN, or a weight that is not finite, would reach the keys that the row does not see: those come by scores of -inf,
      // which only make 0 of numbers.  So what the row gives to the keys that it sees goes into its scores.
      const bool odd = !(fabsf(weight) < INFINITY);
      if (__builtin_expect(__ballot(odd) != 0, 0)) {
        const bool infinite = weight == weight;  // an infinity, but for scores of -inf (0 times it) and NaN
        shift = odd ? 0.f : shift;
        weight = odd ? copysignf(1.f, weight) : weight;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[kb][i] = !odd ? sc[kb][i] : infinite && sc[kb][i] > -INFINITY ? INFINITY : NAN;
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const int from = base + (wave * KB + kb) * 32;
        uint32_t v = masks ? reinterpret_cast<const uint32_t *>(st)[64 + 32 * kb + l31] : keys_below(row / a.G + 1 - from);
        v = (v & keys_below(g.T - from)) >> (4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!((v >> acc_row(i, 0)) & 1u)) sc[kb][i] = -INFINITY;
      }
    }
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  if (b0 < b1) {
    f32x16 sa[KB], sb[KB];
    tile_there(b0);
    step(sb, sa, 0, yes, no);
    row_of(sa, b0, 0);
    int b = b0, buf = 0;
    auto forward_one = [&](f32x16(&sc)[KB], f32x16(&next)[KB]) {
      tile_there(b + 1);
      if (b + kRing < b1) issue(buf);
      buf = (buf + 1) % kRing;
      step(sc, next, buf, yes, yes);
      row_of(next, b + 1, buf);
      ++b;
    };
    while (b + 2 < b1) {
      forward_one(sa, sb);
      forward_one(sb, sa);
    }
    if (b + 1 < b1) {
      forward_one(sa, sb);
      step(sb, sa, 0, no, yes);
    } else {
      step(sa, sb, 0, no, yes);
    }
  }
  // the 32 lanes of a half summed; lane i < 16 keeps the sum of element i
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float v = row16_sum(w[kb][i]);
      const auto pair = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
      if (l31 == i) mine = __uint_as_float(pair[0]) + __uint_as_float(pair[1]);
    }
    const int key = base + (wave * KB + kb) * 32 + acc_row(l31 & 15, half);
    if (l31 >= 16 || key >= n) continue;
    if (row_splits > 1) {
      part[((size_t)rs * a.n_seq * a.Hk + sh) * tiles * kKeys + (size_t)tile * kKeys + (key - base)] = mine;
    } else if (tree) {
      tree_w[(size_t)(g.row0 + key) * a.Hk + hk] = mine;
    } else {
      const size_t at = (size_t)sh * a.capacity + key;
      w_out[at] = w_in ? fmaf(decay, w_in[at], mine) : mine;
    }
  }
}

// The parts of the rows added up, in order.
__global__ __launch_bounds__(256) void cache_weights_join_kernel(KeyArgs a, int tree_tiles, int tiles, int keys,
                                                                 int row_splits, float decay, const float *w_in, float *w_out,
                                                                 float *__restrict__ tree_w,
                                                                 const float *__restrict__ part) {
  const int sh = blockIdx.y, hk = sh % a.Hk, s = sh / a.Hk;
  const SeqGeom g = seq_geom(a, s);
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= tiles * keys) return;
  const bool tree = i < tree_tiles * keys;
  const int key = tree ? i : i - tree_tiles * keys;
  if (key >= (tree ? g.T : g.len)) return;
  const size_t stride = (size_t)a.n_seq * a.Hk * tiles * keys;
  const float *p = part + (size_t)sh * tiles * keys + i;
  float v = 0.f;
#pragma unroll 4
  for (int r = 0; r < row_splits; ++r) v += p[r * stride];
  if (tree) {
    tree_w[(size_t)(g.row0 + key) * a.Hk + hk] = v;
  } else {
    const size_t at = (size_t)sh * a.capacity + key;
    w_out[at] = w_in ? fmaf(decay, w_in[at], v) : v;
  }
}

namespace {

constexpr int kWeightSlots = 512;   // workgroups that run at a time
constexpr int kWeightParts = 4096;  // most workgroups of a launch whose rows are in parts

// Parts of the rows.  n_seq * Hk * key tiles workgroups run in rounds of kWeightSlots, the last of which may be nearly empty; parts make
// more and shorter rounds, at the price of the keys' loads in each (about four tiles of rows).
int row_splits_of(const KeyArgs &a, int64_t tiles) {
  const int64_t groups = (int64_t)a.n_seq * a.Hk * tiles, blocks = ((int64_t)a.max_tree * a.G + 31) / 32;
  int best = 1;
  int64_t least = INT64_MAX;
  for (int64_t n = 1; n <= blocks && n <= 64 && (n == 1 || n * groups <= kWeightParts); ++n) {
    const int64_t cost = (groups * n + kWeightSlots - 1) / kWeightSlots * ((blocks + n - 1) / n + 4);
    if (cost < least) {
      least = cost;
      best = (int)n;
    }
  }
  return best;
}

template <typename T, int D>
hipError_t run_weights(const KeyArgs &a, const float *lse, const float *row_weight, float decay,
                       const float *w_in, float *w_out, float *tree_w, void *ws, hipStream_t st) {
  constexpr int K = WeightShape<T, D>::kKeys;
  const int tree_tiles = tree_w ? (a.max_tree + K - 1) / K : 0, tiles = tree_tiles + (a.max_len + K - 1) / K;
  if (tiles == 0) return hipSuccess;
  const int rs = row_splits_of(a, tiles);
  float *part = static_cast<float *>(ws);
  auto kern = cache_weights_kernel<T, D>;
  constexpr size_t smem = WeightShape<T, D>::kLds;
  if (smem > 64 * 1024) {  // beyond the default limit of a launch
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
  }
  kern<<<(unsigned)((int64_t)a.n_seq * a.Hk * tiles * rs), 64 * kWeightWaves, smem, st>>>(
      a, tree_tiles, tiles, rs, lse, row_weight, decay, w_in, w_out, tree_w, part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || rs == 1) return e;
  cache_weights_join_kernel<<<dim3((tiles * K + 255) / 256, a.n_seq * a.Hk), 256, 0, st>>>(a, tree_tiles, tiles, K, rs, decay,
                                                                                          w_in, w_out, tree_w, part);
  return hipGetLastError();
}

template <typename T>
hipError_t run_weights_type(const moespec_attn_desc &ds, const KeyArgs &a, const float *lse, const float *row_weight,
                            float decay, const float *w_in, float *w_out, float *tree_w, void *ws, hipStream_t st) {
  switch (ds.head_dim) {
    case 64: return run_weights<T, 64>(a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    case 96: return run_weights<T, 96>(a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    case 128: return run_weights<T, 128>(a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    case 192: return run_weights<T, 192>(a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    default: return run_weights<T, 256>(a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
  }
}

}  // namespace

// With more than one part of the rows there are at most kWeightParts workgroups, each with a sum for every one of up to 256 keys; and
// at most 64 parts of what there is.  Neither bound grows where a call gets smaller.
size_t cache_weights_ws(const moespec_attn_desc &ds, int64_t n_seq, int64_t max_tree, int64_t max_len) {
  const int64_t tiles = (max_tree + 127) / 128 + (max_len + 127) / 128, groups = n_seq * ds.n_kv_heads * tiles;
  return sizeof(float) * 256 * (size_t)(groups < kWeightParts / 64 ? 64 * groups : kWeightParts);
}

hipError_t launch_cache_weights(const moespec_attn_desc &ds, const KeyArgs &a, const float *lse, const float *row_weight,
                                float decay, const float *w_in, float *w_out, float *tree_w, void *ws, hipStream_t st) {
  return ds.dtype == MOESPEC_BF16 ? run_weights_type<uint16_t>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st)
                                  : run_weights_type<float>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
}

}  // namespace moespec
