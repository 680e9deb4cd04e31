// The attention weight that every key received: w_j = sum over rows of row_weight 2^(c q.K_j - lse / ln 2).
//
// The softmax statistics of the rows are known (lse), so a column sum needs nothing from other keys: a wave holds its 32 KB keys
// as matrix operands in registers and walks over the rows, whose tiles of 32 lie in LDS, one ahead.  S^T = K Q^T has a row of
// queries per lane, and the weights of a key add up in one register per lane; the 32 lanes are summed once at the end.  A
// workgroup is the only writer of its keys, or of its part of the rows, which a second launch adds up in order.
#include <math.h>

#include "attention.h"

namespace moespec {

constexpr int kWeightWaves = 4;

template <typename T, int D>
struct WeightShape {
  static constexpr int kKb = D * (int)sizeof(T) <= 384 ? 2 : 1;  // 32-key blocks held by a wave
  static constexpr int kKeys = 32 * kKb * kWeightWaves;
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
#pragma clang diagnostic pop

template <typename T, int D>
__global__ __launch_bounds__(64 * kWeightWaves, 2) void cache_weights_kernel(
    KeyArgs a, int cache_tiles, int tiles, int row_splits, const float *__restrict__ lse, const float *__restrict__ row_weight,
    float decay, const float *w_in, float *w_out, float *__restrict__ tree_w, float *__restrict__ part) {
  typedef Rows<T, D> R;
  typedef typename Frag<T>::type frag;
  constexpr int KB = WeightShape<T, D>::kKb, kKeys = WeightShape<T, D>::kKeys, NS = R::kPieces / 2;
  constexpr int kTile = 32 * R::kBytes, kRowsPerLoad = 64 / R::kSlots, kLoads = 32 / kRowsPerLoad;
  static_assert(kLoads % kWeightWaves == 0, "every wave issues as many loads");
  __shared__ __align__(16) unsigned char lds[2 * kTile];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l31 = lane & 31, half = lane >> 5;
  const int rs = blockIdx.x % row_splits, tile = blockIdx.x / row_splits % tiles, sh = blockIdx.x / row_splits / tiles;
  const int hk = sh % a.Hk, s = sh / a.Hk;
  const SeqGeom g = seq_geom(a, s);
  const bool tree = tile >= cache_tiles;
  const int base = (tree ? tile - cache_tiles : tile) * kKeys, n = tree ? g.T : g.len;
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
  auto issue = [&](int b, int buf) {
#pragma unroll
    for (int i = 0; i < kLoads / kWeightWaves; ++i) {
      const int ld = i * kWeightWaves + wave, rr = ld * kRowsPerLoad + lane / R::kSlots;
      const int piece = min((lane % R::kSlots) ^ R::swz(rr), R::kPieces - 1);
      const int row = min(32 * b + rr, n_rows - 1);
      dma_to_lds_from(lds0 + buf * kTile + ld * 1024,
                      static_cast<const T *>(a.q) + (g.row0 + row / a.G) * a.q_stride + (hk * a.G + row % a.G) * D +
                          piece * R::kPieceElems);
    }
  };
  if (b0 < b1) issue(b0, 0);
  for (int b = b0; b < b1; ++b) {
    const int buf = (b - b0) & 1;
    const int row = min(32 * b + l31, n_rows - 1), t = row / a.G;
    float ls = lse[(size_t)(g.row0 + t) * a.H + hk * a.G + row % a.G];
    const float rw = row_weight ? row_weight[g.row0 + t] : 1.f;
    const bool ok = 32 * b + l31 < n_rows && ls != -INFINITY;
    ls *= 1.4426950408889634f;
    uint32_t word[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      word[kb] = !ok ? 0u : tree ? tree_word(a, g, t, base + (wave * KB + kb) * 32) : ~0u;
    bool all = true;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) all &= word[kb] == ~0u;
    const bool masked = __ballot(!all) != 0;
    wait_vm<0>();
    asm volatile("" ::: "memory");
    __syncthreads();
    if (b + 1 < b1) issue(b + 1, buf ^ 1);
    const unsigned char *qt = lds + buf * kTile;
    f32x16 sc[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const frag q = *reinterpret_cast<const frag *>(qt + l31 * R::kBytes + (((2 * i + half) ^ R::swz(l31)) << 4));
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) sc[kb] = Frag<T>::mma(k[kb][i], q, sc[kb]);
    }
    if (!masked) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) w[kb][i] = fmaf(rw, __builtin_amdgcn_exp2f(fmaf(sc[kb][i], a.c, -ls)), w[kb][i]);
    } else {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const uint32_t v = word[kb] >> (4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float p = fmaf(rw, __builtin_amdgcn_exp2f(fmaf(sc[kb][i], a.c, -ls)), w[kb][i]);
          w[kb][i] = ((v >> acc_row(i, 0)) & 1u) ? p : w[kb][i];
        }
      }
    }
  }
  // the 32 lanes of a half summed; lane i < 16 keeps the sum of element i
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = row16_sum(w[kb][i]);
      v += __shfl_xor(v, 16, kWave);
      if (l31 == i) mine = v;
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
__global__ __launch_bounds__(256) void cache_weights_join_kernel(KeyArgs a, int cache_tiles, int tiles, int keys,
                                                                 int row_splits, float decay, const float *w_in, float *w_out,
                                                                 float *__restrict__ tree_w,
                                                                 const float *__restrict__ part) {
  const int sh = blockIdx.y, hk = sh % a.Hk, s = sh / a.Hk;
  const SeqGeom g = seq_geom(a, s);
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= tiles * keys) return;
  const bool tree = i >= cache_tiles * keys;
  const int key = tree ? i - cache_tiles * keys : i;
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

constexpr int kWeightTarget = 512;  // workgroups wanted

// n_seq * Hk * key tiles workgroups, times the parts of the rows where those are few.
int row_splits_of(const moespec_attn_desc &ds, int64_t n_seq, int64_t tiles, int64_t max_tree) {
  const int64_t groups = n_seq * ds.n_kv_heads * tiles;
  const int64_t blocks = (max_tree * (ds.n_heads / ds.n_kv_heads) + 31) / 32;
  int64_t n = kWeightTarget / groups;
  n = n < blocks ? n : blocks;
  return (int)(n > 1 ? n : 1);
}

template <typename T, int D>
hipError_t run_weights(const moespec_attn_desc &ds, const KeyArgs &a, const float *lse, const float *row_weight, float decay,
                       const float *w_in, float *w_out, float *tree_w, void *ws, hipStream_t st) {
  constexpr int K = WeightShape<T, D>::kKeys;
  const int cache_tiles = (a.max_len + K - 1) / K, tiles = cache_tiles + (tree_w ? (a.max_tree + K - 1) / K : 0);
  if (tiles == 0) return hipSuccess;
  const int rs = row_splits_of(ds, a.n_seq, tiles, a.max_tree);
  float *part = static_cast<float *>(ws);
  cache_weights_kernel<T, D><<<(unsigned)((int64_t)a.n_seq * a.Hk * tiles * rs), 64 * kWeightWaves, 0, st>>>(
      a, cache_tiles, tiles, rs, lse, row_weight, decay, w_in, w_out, tree_w, part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || rs == 1) return e;
  cache_weights_join_kernel<<<dim3((tiles * K + 255) / 256, a.n_seq * a.Hk), 256, 0, st>>>(a, cache_tiles, tiles, K, rs, decay,
                                                                                          w_in, w_out, tree_w, part);
  return hipGetLastError();
}

template <typename T>
hipError_t run_weights_type(const moespec_attn_desc &ds, const KeyArgs &a, const float *lse, const float *row_weight,
                            float decay, const float *w_in, float *w_out, float *tree_w, void *ws, hipStream_t st) {
  switch (ds.head_dim) {
    case 64: return run_weights<T, 64>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    case 96: return run_weights<T, 96>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    case 128: return run_weights<T, 128>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    case 192: return run_weights<T, 192>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
    default: return run_weights<T, 256>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
  }
}

}  // namespace

// With more than one part of the rows there are at most kWeightTarget workgroups, each with a sum for every one of up to 256 keys.
size_t cache_weights_ws(const moespec_attn_desc &, int64_t, int64_t, int64_t) {
  return sizeof(float) * kWeightTarget * 256;
}

hipError_t launch_cache_weights(const moespec_attn_desc &ds, const KeyArgs &a, const float *lse, const float *row_weight,
                                float decay, const float *w_in, float *w_out, float *tree_w, void *ws, hipStream_t st) {
  return ds.dtype == MOESPEC_BF16 ? run_weights_type<uint16_t>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st)
                                  : run_weights_type<float>(ds, a, lse, row_weight, decay, w_in, w_out, tree_w, ws, st);
}

}  // namespace moespec
