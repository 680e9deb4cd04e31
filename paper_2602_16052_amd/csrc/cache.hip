// Writing to a cache of keys and values: the accepted path appended, and a cache cut to its budget.
// Both are bound by memory traffic (and, for few entries, by the launch): every 16 bytes of a kept row are read and written once.
// Commit of 8 tokens for 48 layers x 8 sequences x 4 heads: 5 us.  Eviction, 16 heads 4093 -> 2048 entries: 14 us, selection 7.8 and
// copy 7.2 (4.7 TB/s); 128 heads 32749 -> 4096: 133 us, 27 and 107 (5.0 TB/s).  Selection is bound by the LDS atomics of the first
// histogram and by barriers; it reads 4 bytes an entry where the copy moves 4 D.
#include "attention.h"

namespace moespec {

namespace {
__device__ __forceinline__ int clamp_len(const int32_t *len, int s, int capacity) { return min(max(len[s], 0), capacity); }
}  // namespace

// One thread per 16 bytes of a row, of keys and of values: thread p of (layer, sequence, i, head) appends piece p of token
// path[s, i].
struct CommitArgs {
  const uint4 *k_tree, *v_tree;
  uint4 *k_cache, *v_cache;
  const float *tree_w;
  float *cache_w;
  const int32_t *path, *n_path, *cache_len, *tree_off;
  int32_t *new_len;
  int64_t kv_stride, capacity;  // kv_stride in pieces of 16 bytes
  int n_layers, n_seq, M, max_tree, max_path, Hk, pieces;
};
__global__ __launch_bounds__(256) void cache_commit_kernel(CommitArgs a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (a.new_len && id < a.n_seq)
    a.new_len[id] = (int)min((int64_t)clamp_len(a.cache_len, (int)id, (int)a.capacity) + min(max(a.n_path[id], 0), a.max_path),
                             a.capacity);
  const int p = id % a.pieces;
  int64_t r = id / a.pieces;
  const int hk = r % a.Hk;
  r /= a.Hk;
  const int i = r % a.max_path;
  r /= a.max_path;
  const int s = r % a.n_seq;
  const int layer = (int)(r / a.n_seq);
  if (layer >= a.n_layers || i >= a.n_path[s]) return;
  const int64_t dst = (int64_t)clamp_len(a.cache_len, s, (int)a.capacity) + i;
  if (dst >= a.capacity) return;
  int row0 = 0, T = a.M;
  if (a.tree_off) {
    row0 = min(max(a.tree_off[s], 0), a.M);
    T = min(max(a.tree_off[s + 1], row0), a.M) - row0;
  }
  T = min(T, a.max_tree);
  const int t = a.path[(int64_t)s * a.max_path + i];
  const bool ok = t >= 0 && t < T;
  const int64_t src = ((int64_t)layer * a.M + row0 + (ok ? t : 0)) * a.kv_stride + hk * a.pieces + p;
  const int64_t entry = (((int64_t)layer * a.n_seq + s) * a.Hk + hk) * a.capacity + dst;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 k = zero, v = zero;
  if (ok) {
    k = a.k_tree[src];
    v = a.v_tree[src];
  }
  a.k_cache[entry * a.pieces + p] = k;
  a.v_cache[entry * a.pieces + p] = v;
  if (p == 0 && a.cache_w) a.cache_w[entry] = ok ? a.tree_w[((int64_t)layer * a.M + row0 + t) * a.Hk + hk] : 0.f;
}

hipError_t launch_cache_commit(const moespec_attn_desc &ds, int n_layers, const moespec_tree &tree, const void *k_tree,
                               const void *v_tree, const float *tree_w, const int32_t *path, const int32_t *n_path,
                               int max_path, void *k_cache, void *v_cache, float *cache_w, const int32_t *cache_len,
                               int32_t *new_len, hipStream_t st) {
  const int es = ds.dtype == MOESPEC_BF16 ? 2 : 4, pieces = ds.head_dim * es / 16;
  const int64_t stride = tree.kv_stride ? tree.kv_stride : (int64_t)ds.n_kv_heads * ds.head_dim;
  CommitArgs a{static_cast<const uint4 *>(k_tree), static_cast<const uint4 *>(v_tree), static_cast<uint4 *>(k_cache),
               static_cast<uint4 *>(v_cache), tree_w, cache_w, path, n_path, cache_len, tree.tree_off, new_len,
               stride * es / 16, ds.capacity, n_layers, tree.n_seq, tree.n_tokens, tree.max_tree, max_path, ds.n_kv_heads,
               pieces};
  const int64_t n = (int64_t)n_layers * tree.n_seq * max_path * ds.n_kv_heads * pieces;
  cache_commit_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

// ---- eviction

// A weight as an integer of the same order: NaN behind everything, both zeros alike.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which entries stay, one workgroup per (layer, sequence, head).  The weights are looked at as integers of the same order:
// three histograms (11, 11 and 10 bits from the top) give the value of the last one kept and how many of its equals are kept; then
// every wave places the kept ones of its share, in order.  R > 0: a thread holds the R weights of its places (wave v has 64 R entries in a
// row, lane after lane), which are read once, all loads in flight together; R = 0: longer caches, read in every pass.
// Weights of a cache lie within some ten powers of two, 40 bins of the first histogram: each of kCopies lanes counts into a
// histogram of its own, or most of the 64 lanes would wait for each other.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave, kBins = 2048, kCopies = 4, kMaxHeld = 32, kBatch = 16;
// Sum of v over this lane and those in front of it.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += dpp_or_0<0x111, 0xf>(v);  // one lane on inside of a row of 16, then two, four and eight
  v += dpp_or_0<0x112, 0xf>(v);
  v += dpp_or_0<0x114, 0xf>(v);
  v += dpp_or_0<0x118, 0xf>(v);
  v += dpp_or_0<0x142, 0xa>(v);  // the first row's last lane to the second row, the third's to the fourth
  return v + dpp_or_0<0x143, 0xc>(v);  // the second row's to both rows behind it
}
// Sum of the first `wave` of a workgroup's sums, in every lane.
__device__ __forceinline__ uint32_t sum_before(const uint32_t *sums, int wave) {
  const int l = threadIdx.x & 15;
  static_assert(kSelectWaves == 16, "a row of 16 lanes has them all");
  return (uint32_t)row16_sum(l < wave ? (int)sums[l] : 0);
}

template <int R>
__device__ __forceinline__ void select_entries(const float *__restrict__ w, int n, int want, uint32_t *hist, uint32_t *wave_sum,
                                               uint32_t *wave_eq, uint32_t *found, float *__restrict__ w_out,
                                               int32_t *__restrict__ kept) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int share = R > 0 ? 64 * R : ((n + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64, i0 = wave * share;
  const int rounds = R > 0 ? R : share / 64;
  float held[R > 0 ? R : 1];
  if constexpr (R > 0) {
#pragma unroll
    for (int x = 0; x < R; ++x) held[x] = w[min(i0 + 64 * x + lane, n - 1)];
  }
  // f(entry, weight) for every place of this lane; entries from n on are none
  auto each = [&](auto f) {
    if constexpr (R > 0) {
#pragma unroll
      for (int x = 0; x < R; ++x) f(i0 + 64 * x + lane, held[x]);
    } else {
#pragma unroll 1
      for (int x = 0; x < rounds; x += kBatch) {  // a batch of loads in flight
        float v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int i = i0 + 64 * (x + u) + lane;
          v[u] = w[min(i, n - 1)];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (x + u < rounds) f(i0 + 64 * (x + u) + lane, v[u]);
      }
    }
  };
  uint32_t prefix = 0, left = want;  // the last one kept starts with `prefix`; it is number `left` of those that do
  for (int b = tid; b < kCopies * kBins; b += kSelectThreads) hist[b] = 0;
  __syncthreads();
#pragma unroll 1
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, mask = round == 2 ? 1023 : 2047, known = round == 1 ? 21 : 10;
    each([&](int i, float v) {
      const uint32_t k = weight_key(v);
      if (i < n && (round == 0 || k >> known == prefix)) atomicAdd(&hist[lane % kCopies * kBins + (k >> shift & mask)], 1u);
    });
    __syncthreads();
    // thread i has bins 2 i' and 2 i' + 1 counted from the top, and clears them for the next round; a scan over the workgroup
    // finds the bin of number `left`
    const int top = kBins - 1 - 2 * tid;
    uint32_t h0 = 0, h1 = 0;
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      uint2 *h = reinterpret_cast<uint2 *>(hist + c * kBins + top - 1);
      h0 += h->y;
      h1 += h->x;
      *h = make_uint2(0, 0);
    }
    const uint32_t scan = wave_scan(h0 + h1);
    if (lane == 63) wave_sum[wave] = scan;
    __syncthreads();
    const uint32_t before = sum_before(wave_sum, wave) + scan - h0 - h1;
    if (before < left && before + h0 >= left) {
      found[0] = top;
      found[1] = left - before;
    } else if (before + h0 < left && before + h0 + h1 >= left) {
      found[0] = top - 1;
      found[1] = left - before - h0;
    }
    __syncthreads();
    const uint32_t bin = found[0];
    prefix = round == 2 ? prefix << 10 | bin : round == 1 ? prefix << 11 | bin : bin;
    left = found[1];
  }

  uint32_t gt = 0, eq = 0;  // of this wave's share: above the last one kept, its equals
  each([&](int i, float v) {
    const uint32_t k = weight_key(v);
    gt += __popcll(__ballot(i < n && k > prefix));
    eq += __popcll(__ballot(i < n && k == prefix));
  });
  if (lane == 0) {
    wave_sum[wave] = gt;
    wave_eq[wave] = eq;
  }
  __syncthreads();
  uint32_t eqs = sum_before(wave_eq, wave), at = sum_before(wave_sum, wave);
  at += min(eqs, left);  // of the equals in front of this share the first `left` are kept
  const uint64_t below = (1ull << lane) - 1;
  each([&](int i, float v) {
    const uint32_t k = weight_key(v);
    const uint64_t eq_mask = __ballot(i < n && k == prefix);
    const bool keep = i < n && (k > prefix || (k == prefix && eqs + __popcll(eq_mask & below) < left));
    const uint64_t mask = __ballot(keep);
    if (keep) {
      const uint32_t dst = at + __popcll(mask & below);
      kept[dst] = i;
      w_out[dst] = v;
    }
    at += __popcll(mask);
    eqs += __popcll(eq_mask);
  });
}

template <int R>
__global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(const float *__restrict__ w_all,
                                                                      const int32_t *__restrict__ cache_len, int n_seq,
                                                                      int Hk, int capacity, int budget, int recent,
                                                                      int64_t out_capacity, float *__restrict__ w_out_all,
                                                                      int32_t *__restrict__ kept_all, int32_t *new_len) {
  __shared__ __align__(8) uint32_t hist[kCopies * kBins];
  __shared__ uint32_t wave_sum[kSelectWaves], wave_eq[kSelectWaves], found[2];
  const int hd = blockIdx.x, s = hd / Hk % n_seq, tid = threadIdx.x;
  const int len = clamp_len(cache_len, s, capacity);
  const float *w = w_all + (int64_t)hd * capacity;
  float *w_out = w_out_all + (int64_t)hd * out_capacity;
  int32_t *kept = kept_all + (int64_t)hd * budget;
  if (new_len && hd < n_seq * Hk && hd % Hk == 0 && tid == 0) new_len[s] = min(len, budget);
  for (int i = min(len, budget) + tid; i < budget; i += kSelectThreads) kept[i] = -1;
  if (len <= budget) {
    for (int i = tid; i < len; i += kSelectThreads) {
      kept[i] = i;
      w_out[i] = w[i];
    }
    return;
  }
  const int n = len - recent, want = budget - recent;  // want < n
  for (int i = tid; i < recent; i += kSelectThreads) {
    kept[want + i] = n + i;
    w_out[want + i] = w[n + i];
  }
  if (want == 0) return;

  if (R > 0 && n <= kSelectThreads * R)
    select_entries<R>(w, n, want, hist, wave_sum, wave_eq, found, w_out, kept);
  else
    select_entries<0>(w, n, want, hist, wave_sum, wave_eq, found, w_out, kept);
}

// The rows of the kept entries copied: a workgroup takes 4 kGatherThreads pieces of 16 bytes of each cache, whole rows or not, every
// thread four of each, whose loads are in flight together.
constexpr int kGatherThreads = 256;
__global__ __launch_bounds__(kGatherThreads) void cache_gather_kernel(const uint4 *__restrict__ k_in,
                                                                      const uint4 *__restrict__ v_in,
                                                                      const int32_t *__restrict__ kept, int budget,
                                                                      int64_t capacity, int64_t out_capacity, int pieces,
                                                                      int groups, uint4 *__restrict__ k_out,
                                                                      uint4 *__restrict__ v_out) {
  const int hd = blockIdx.x / groups, grp = blockIdx.x % groups;
  const int32_t *list = kept + (int64_t)hd * budget;
  const int64_t in = (int64_t)hd * capacity * pieces, out = (int64_t)hd * out_capacity * pieces;
  const int64_t total = (int64_t)budget * pieces, i0 = (int64_t)grp * kGatherThreads * 4 + threadIdx.x;
  uint4 k[4], v[4];
  int src[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int64_t i = i0 + u * kGatherThreads;
    src[u] = list[min(i, total - 1) / pieces];
    src[u] = i < total && src[u] < capacity ? src[u] : -1;  // (a list that somebody else wrote to meanwhile)
  }
  if (list[0] < 0) return;  // no entry at all: nothing of this cache is read
#pragma unroll
  for (int u = 0; u < 4; ++u) {  // places that stay empty load the first entry
    const int64_t at = in + (int64_t)max(src[u], 0) * pieces + (i0 + u * kGatherThreads) % pieces;
    k[u] = k_in[at];
    v[u] = v_in[at];
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (src[u] >= 0) {
      k_out[out + i0 + u * kGatherThreads] = k[u];
      v_out[out + i0 + u * kGatherThreads] = v[u];
    }
}

hipError_t launch_cache_evict(const moespec_attn_desc &ds, int n_layers, int n_seq, const void *k_cache,
                              const void *v_cache, const float *cache_w, const int32_t *cache_len, int budget, int recent,
                              int out_capacity, void *k_out, void *v_out, float *w_out, int32_t *kept, int32_t *new_len,
                              hipStream_t st) {
  const int es = ds.dtype == MOESPEC_BF16 ? 2 : 4, pieces = ds.head_dim * es / 16;
  const int64_t heads = (int64_t)n_layers * n_seq * ds.n_kv_heads;
  auto select = [&](auto kern) {
    kern<<<(unsigned)heads, kSelectThreads, 0, st>>>(cache_w, cache_len, n_seq, ds.n_kv_heads, ds.capacity, budget, recent,
                                                     out_capacity, w_out, kept, new_len);
    return hipGetLastError();
  };
  const int each = (ds.capacity + kSelectThreads - 1) / kSelectThreads;  // weights of a thread, at most
  hipError_t e = each <= 6 ? select(cache_select_kernel<6>) : each <= 16 ? select(cache_select_kernel<16>)
                                                                        : select(cache_select_kernel<kMaxHeld>);
  if (e != hipSuccess) return e;
  const int64_t groups = ((int64_t)budget * pieces + 4 * kGatherThreads - 1) / (4 * kGatherThreads);
  cache_gather_kernel<<<(unsigned)(heads * groups), kGatherThreads, 0, st>>>(
      static_cast<const uint4 *>(k_cache), static_cast<const uint4 *>(v_cache), kept, budget, ds.capacity, out_capacity, pieces,
      (int)groups, static_cast<uint4 *>(k_out), static_cast<uint4 *>(v_out));
  return hipGetLastError();
}

}  // namespace moespec
