// Verification of drafted tokens: from the target's logits and given random numbers to the accepted path and the next token.
//
// Two launches.  The first reads every row of logits once, which bounds it: largest logit and sum of exponentials of each chunk of a row
// (which rows lie on the path is known only behind this).  The second, one workgroup a sequence, joins the chunks of its rows, walks
// the tree in LDS, and draws the next token: the chunk in which the running sum passes its target is found from the chunks' sums, and only
// that chunk is read again.  With a drafter's distribution the difference p - q of the last row is summed over chunks there too.
// Probabilities are in fp64: accepting and drawing are decisions, and have to fall the same way whatever the order of the sums.
#include "serving.h"

namespace moespec {

namespace {

constexpr int kChunk = 4096;       // logits of a workgroup's chunk
constexpr int kStatThreads = 256, kWalkThreads = 1024;
constexpr int kEach = kChunk / kStatThreads;

// A chunk of a row: largest logit, its first place, sum of exp((logit - largest) / temperature).
struct ChunkStat {
  double sum;
  float top;
  int arg;
};

struct VerifyArgs {
  const void *logits, *draft;
  const float *temperature;
  const int32_t *tree_off, *tokens;
  const uint32_t *tree_mask;
  const double *u_accept, *u_sample;
  int32_t *path, *n_path, *next_token;
  float *accepted;
  ChunkStat *stats;  // [1 or 2 (draft)][M][chunks]
  int64_t logit_stride, draft_stride;
  int V, chunks, n_seq, M, max_tree, words, max_path;
};

// 1 / temperature of a sequence; 0 where it is greedy.
__device__ __forceinline__ double inverse_heat(const VerifyArgs &a, int s) {
  const float t = a.temperature ? a.temperature[s] : 1.f;
  return t > 0.f ? 1.0 / (double)fminf(fmaxf(t, 0x1p-60f), 0x1p60f) : 0.0;
}

template <typename T>
__device__ __forceinline__ float logit_at(const void *row, int64_t i) {
  return Elem<T>::load(static_cast<const T *>(row) + i);
}

struct Best {
  float top;
  int arg;
};
__device__ __forceinline__ Best better(Best a, Best b) { return b.top > a.top || (b.top == a.top && b.arg < a.arg) ? b : a; }

// exp((x - top) * inverse): 0 for -inf, NaN for NaN and for x = top = +inf.
__device__ __forceinline__ double weight_of(float x, float top, double inverse) {
  return x == -INFINITY ? 0.0 : exp_nonpos(((double)x - (double)top) * inverse);
}

__device__ __forceinline__ double wave_sum64(double v) {
  v = row16_sum(v);
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}

// kVec: rows start at multiples of 16 bytes.
template <typename T, bool kVec>
__global__ __launch_bounds__(kStatThreads) void logit_stats_kernel(VerifyArgs a) {
  constexpr int E = 16 / (int)sizeof(T);
  const int row = blockIdx.y, chunk = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool draft = blockIdx.z == 1;
  const T *x = static_cast<const T *>(draft ? a.draft : a.logits) + (int64_t)row * (draft ? a.draft_stride : a.logit_stride);
  const int base = chunk * kChunk;
  float v[kEach];
  int at[kEach];
  if constexpr (kVec) {
#pragma unroll
    for (int i = 0; i < kEach / E; ++i) {
      const int j = base + (i * kStatThreads + (int)threadIdx.x) * E;
      if (j + E <= a.V) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const f32x4 f = Elem<T>::load4(x + j + e);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[i * E + e + k] = f[k];
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i * E + e] = j + e < a.V ? Elem<T>::load(x + j + e) : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) at[i * E + e] = j + e;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      at[i] = base + i * kStatThreads + (int)threadIdx.x;
      v[i] = at[i] < a.V ? Elem<T>::load(x + at[i]) : -INFINITY;
    }
  }
  const int s = seq_of_row(a.tree_off, a.n_seq, row);
  if (s >= a.n_seq) return;
  const double inverse = inverse_heat(a, s);
  __shared__ Best best_of[kStatThreads / kWave];
  __shared__ double sum_of[kStatThreads / kWave];
  Best b{v[0], at[0]};
#pragma unroll
  for (int i = 1; i < kEach; ++i)
    if (v[i] > b.top) b = Best{v[i], at[i]};  // (places ascend)
  if (!(b.top >= -INFINITY)) {  // the first one is NaN: the comparisons above have all been false
    b.top = -INFINITY;
#pragma unroll
    for (int i = 1; i < kEach; ++i)
      if (v[i] > b.top) b = Best{v[i], at[i]};
  }
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) b = better(b, Best{__shfl_xor(b.top, m, kWave), __shfl_xor(b.arg, m, kWave)});
  if (lane == 0) best_of[wave] = b;
  __syncthreads();
  b = best_of[0];
#pragma unroll
  for (int w = 1; w < kStatThreads / kWave; ++w) b = better(b, best_of[w]);
  double sum = 0.0;
  if (inverse > 0.0) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += weight_of(v[i], b.top, inverse);
  } else {  // greedy: whether the row is a distribution
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += v[i] < INFINITY ? (v[i] == b.top && v[i] > -INFINITY ? 1.0 : 0.0) : __builtin_nan("");
  }
  sum = wave_sum64(sum);
  if (lane == 0) sum_of[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = sum_of[0];
    for (int w = 1; w < kStatThreads / kWave; ++w) total += sum_of[w];
    a.stats[((int64_t)blockIdx.z * a.M + row) * a.chunks + chunk] = ChunkStat{total, b.top, b.arg};
  }
}

// A whole row from its chunks: largest logit, its first place, sum; a row that is no distribution has the sum NaN.  All lanes of a wave
// work on one row and end with the same bits.
struct RowStat {
  double sum;
  float top;
  int arg;
};
__device__ __forceinline__ RowStat join_chunks(const ChunkStat *c, int chunks, double inverse) {
  const int lane = threadIdx.x & 63;
  Best b{-INFINITY, 0x7fffffff};
  for (int i = lane; i < chunks; i += kWave) b = better(b, Best{c[i].top, c[i].arg});
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) b = better(b, Best{__shfl_xor(b.top, m, kWave), __shfl_xor(b.arg, m, kWave)});
  double sum = 0.0;
  for (int i = lane; i < chunks; i += kWave) sum += c[i].sum * weight_of(c[i].top, b.top, inverse);
  sum = wave_sum64(sum);
  return RowStat{sum > 0.0 && sum < INFINITY ? sum : __builtin_nan(""), b.top, b.arg};
}

// What the last row's tokens weigh: p, without the tokens in `gone`; or what p has over q.
template <typename T>
struct Rest {
  const VerifyArgs *a;
  const void *p, *q;  // q NULL: p without the tokens that are gone
  RowStat ps, qs;
  double inverse, p_scale, q_scale;
  const int32_t *gone;  // LDS: tokens that are gone
  int n_gone;
  __device__ __forceinline__ double operator()(int i) const {
    double w = weight_of(logit_at<T>(p, i), ps.top, inverse) * p_scale;
    if (q) w = fmax(w - weight_of(logit_at<T>(q, i), qs.top, inverse) * q_scale, 0.0);
    for (int k = 0; k < n_gone; ++k) w = gone[k] == i ? 0.0 : w;
    return w;
  }
};

template <typename T>
__global__ __launch_bounds__(kWalkThreads) void draft_walk_kernel(VerifyArgs a) {
  constexpr int kWaves = kWalkThreads / kWave;
  extern __shared__ __align__(16) unsigned char lds[];
  // [max_tree] each: probability of the token behind its parent (times q in u's place: see below), token, parent, rejected tokens
  double *const mine = reinterpret_cast<double *>(lds);
  int32_t *const token = reinterpret_cast<int32_t *>(mine + a.max_tree);
  int32_t *const parent = token + a.max_tree;
  int32_t *const gone = parent + a.max_tree;
  double *const chunk_sum = reinterpret_cast<double *>(gone + a.max_tree + (a.max_tree & 1));  // [chunks]
  __shared__ double scan_of[kWaves];
  __shared__ int last_s, n_gone_s, next_s, found_s;
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeqRows g = seq_rows(a.tree_off, s, a.M, a.max_tree);
  int32_t *const path = a.path + (int64_t)s * a.max_path;
  if (a.accepted)
    for (int t = threadIdx.x; t < g.T; t += kWalkThreads) a.accepted[g.row0 + t] = t == 0 ? 1.f : 0.f;
  for (int i = threadIdx.x; i < a.max_path; i += kWalkThreads) path[i] = i == 0 && g.T > 0 ? 0 : -1;
  if (g.T == 0) {
    if (threadIdx.x == 0) {
      a.n_path[s] = 0;
      a.next_token[s] = -1;
    }
    return;
  }
  const double inverse = inverse_heat(a, s);
  const bool greedy = inverse == 0.0, sampled = a.draft != nullptr && !greedy;
  for (int t = threadIdx.x; t < g.T; t += kWalkThreads) {
    int p = t - 1;
    if (a.tree_mask && t > 0) {
      p = -1;
      for (int w = t >> 5; w >= 0 && p < 0; --w) {
        const uint32_t bits = a.tree_mask[(int64_t)(g.row0 + t) * a.words + w] & keys_below(t - 32 * w);
        if (bits) p = 32 * w + 31 - __clz((int)bits);
      }
    }
    parent[t] = p;  // -1: of no token's
    token[t] = a.tokens[g.row0 + t];
  }
  __syncthreads();
  // every token's probability, a wave per token; the rows of the parents are joined where they are needed
  for (int t = 1 + wave; t < g.T; t += kWaves) {
    const int u = parent[t], x = token[t];
    double p = 0.0;
    if (u >= 0 && x >= 0 && x < a.V) {
      const int64_t row = g.row0 + u;
      const RowStat r = join_chunks(a.stats + row * a.chunks, a.chunks, inverse);
      if (greedy) {
        p = r.sum > 0.0 && r.arg == x ? 1.0 : 0.0;
      } else if (r.sum > 0.0) {
        p = weight_of(logit_at<T>(static_cast<const T *>(a.logits) + row * a.logit_stride, x), r.top, inverse) / r.sum;
        if (sampled) {
          const RowStat d = join_chunks(a.stats + (a.M + row) * a.chunks, a.chunks, inverse);
          const double q = weight_of(logit_at<T>(static_cast<const T *>(a.draft) + row * a.draft_stride, x), d.top, inverse) / d.sum;
          p = a.u_accept[row + 1] * q < p ? 2.0 : 0.0;  // (a chain: decided here.  NaN is no)
        }
      }
    }
    if (lane == 0) mine[t] = p;
  }
  __syncthreads();
  // the walk, one wave
  if (wave == 0) {
    int last = 0, length = 1, n_gone = 0, next = -1;
    bool cut = false;
    for (;;) {
      int step = -1;
      double left = 0.0;  // mass of the tokens that are gone
      n_gone = 0;
      for (int base = last + 1; base < g.T && step < 0; base += kWave) {
        const int i = base + lane;
        uint64_t kids = __ballot(i < g.T && parent[min(i, g.T - 1)] == last);
        for (; kids != 0 && step < 0; kids &= kids - 1) {
          const int t = base + __builtin_ctzll(kids), x = token[t];
          bool again = false;  // a token that has been rejected already
          for (int k = lane; k < n_gone; k += kWave) again |= gone[k] == x;
          if (__ballot(again) != 0) continue;
          const double p = mine[t];
          const double u = greedy || sampled ? 0.5 : a.u_accept[g.row0 + t];
          if (u * (1.0 - left) < p) {
            step = t;
          } else {
            left += p;
            if (lane == 0) gone[n_gone] = x;
            ++n_gone;
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
          }
        }
      }
      if (step < 0) break;
      if (length == a.max_path) {
        next = token[step];
        cut = true;
        break;
      }
      last = step;
      if (lane == 0) {
        path[length] = step;
        if (a.accepted) a.accepted[g.row0 + step] = 1.f;
      }
      ++length;
    }
    if (lane == 0) {
      a.n_path[s] = length;
      last_s = last;
      n_gone_s = n_gone;
      next_s = cut ? next : -1;
      found_s = cut;
    }
  }
  __syncthreads();
  const int64_t row = g.row0 + last_s;
  const RowStat ps = join_chunks(a.stats + row * a.chunks, a.chunks, inverse);
  if (found_s || !(ps.sum > 0.0) || greedy) {
    if (threadIdx.x == 0) a.next_token[s] = found_s ? next_s : ps.sum > 0.0 ? ps.arg : -1;
    return;
  }
  Rest<T> rest{&a, static_cast<const T *>(a.logits) + row * a.logit_stride, nullptr, ps, RowStat{}, inverse, 1.0, 0.0, gone, n_gone_s};
  if (sampled) {
    rest.n_gone = 0;
    if (n_gone_s > 0) {
      rest.qs = join_chunks(a.stats + (a.M + row) * a.chunks, a.chunks, inverse);
      if (rest.qs.sum > 0.0) {
        rest.q = static_cast<const T *>(a.draft) + row * a.draft_stride;
        rest.p_scale = 1.0 / ps.sum;
        rest.q_scale = 1.0 / rest.qs.sum;
      }
    }
  }
  // sums of the chunks of what is left; where there is nothing, of p itself
  auto whole_chunks = [&]() {
    for (int c = threadIdx.x; c < a.chunks; c += kWalkThreads) {
      const ChunkStat st = a.stats[row * a.chunks + c];
      chunk_sum[c] = st.sum * weight_of(st.top, ps.top, inverse);
    }
  };
  auto some_left = [&]() {
    bool any = false;
    for (int c = lane; c < a.chunks; c += kWave) any |= chunk_sum[c] > 0.0;
    return __ballot(any) != 0;
  };
  if (rest.q || rest.n_gone > 0) {
    for (int c = wave; c < a.chunks; c += kWaves) {
      double sum = 0.0;
      for (int i = c * kChunk + lane; i < min((c + 1) * kChunk, a.V); i += kWave) sum += rest(i);
      sum = wave_sum64(sum);
      if (lane == 0) chunk_sum[c] = sum;
    }
    __syncthreads();
    if (!some_left()) {
      __syncthreads();
      rest.q = nullptr;
      rest.n_gone = 0;
      rest.p_scale = 1.0;
      whole_chunks();
    }
  } else {
    whole_chunks();
  }
  __syncthreads();
  // the running sum over chunks, by every wave for itself
  double total = 0.0;
  for (int c = 0; c < a.chunks; c += kWave) {
    double v = c + lane < a.chunks ? chunk_sum[c + lane] : 0.0;
    total += wave_sum64(v);
  }
  const double u = a.u_sample[s];
  const double goal = (u > 0.0 ? fmin(u, 1.0) : 0.0) * total;  // (NaN: 0)
  double before = 0.0;
  int chunk = -1, most = -1;  // most: the last chunk with anything
  for (int c = 0; c < a.chunks && chunk < 0; c += kWave) {
    const double v = c + lane < a.chunks ? chunk_sum[c + lane] : 0.0;
    double sum = v;
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
      const double up = __shfl_up(sum, m, kWave);
      if (lane >= m) sum += up;
    }
    const uint64_t hit = __ballot(before + sum > goal && v > 0.0), some = __ballot(v > 0.0);
    if (hit != 0) {
      const int f = __builtin_ctzll(hit);
      chunk = c + f;
      before += __shfl(sum, f, kWave) - __shfl(v, f, kWave);
    } else {
      before += __shfl(sum, 63, kWave);
    }
    if (some != 0) most = c + 63 - __clzll((long long)some);
  }
  const bool past = chunk < 0;  // lost to rounding: the last token with a weight
  if (past) chunk = most;
  // the chunk's tokens: kChunk / kWalkThreads in a row to a thread
  constexpr int N = kChunk / kWalkThreads;
  double w[N], sum = 0.0;
  const int first = chunk * kChunk + (int)threadIdx.x * N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    w[i] = chunk >= 0 && first + i < a.V ? rest(first + i) : 0.0;
    sum += w[i];
  }
  double scan = sum;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const double up = __shfl_up(scan, m, kWave);
    if (lane >= m) scan += up;
  }
  if (lane == 63) scan_of[wave] = scan;
  if (threadIdx.x == 0) {
    found_s = 0x7fffffff;
    next_s = -1;
  }
  __syncthreads();
  for (int k = 0; k < wave; ++k) before += scan_of[k];
  double run = before + scan - sum;
  int mine_is = 0x7fffffff, positive = -1;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    run += w[i];
    if (w[i] > 0.0) {
      positive = first + i;
      if (!past && run > goal && mine_is == 0x7fffffff) mine_is = first + i;
    }
  }
  if (mine_is != 0x7fffffff) atomicMin(&found_s, mine_is);
  if (positive >= 0) atomicMax(&next_s, positive);
  __syncthreads();
  if (threadIdx.x == 0) a.next_token[s] = found_s != 0x7fffffff ? found_s : next_s;
}

int chunks_of(const moespec_verify &v) { return (v.vocab + kChunk - 1) / kChunk; }

template <typename T>
hipError_t run_verify(const VerifyArgs &a, hipStream_t st) {
  const bool vec = a.logit_stride * sizeof(T) % 16 == 0 && (!a.draft || a.draft_stride * sizeof(T) % 16 == 0);
  const dim3 grid(a.chunks, a.M, a.draft ? 2 : 1);
  if (vec) logit_stats_kernel<T, true><<<grid, kStatThreads, 0, st>>>(a);
  else logit_stats_kernel<T, false><<<grid, kStatThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t smem = (size_t)a.max_tree * 20 + 4 + (size_t)a.chunks * 8;
  auto kern = draft_walk_kernel<T>;
  if (smem > 60 * 1024) {
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != hipSuccess) return e;
  }
  kern<<<a.n_seq, kWalkThreads, smem, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t draft_verify_ws(const moespec_verify &v, int, int M) {
  return sizeof(ChunkStat) * (size_t)M * chunks_of(v) * (v.draft_logits ? 2 : 1);
}

hipError_t launch_draft_verify(const moespec_verify &v, const moespec_tree &tree, const int32_t *tokens, const double *u_accept,
                               const double *u_sample, int32_t *path, int32_t *n_path, int max_path, int32_t *next_token,
                               float *accepted, void *ws, hipStream_t st) {
  VerifyArgs a{};
  a.logits = v.logits;
  a.draft = v.draft_logits;
  a.temperature = v.temperature;
  a.tree_off = tree.tree_off;
  a.tokens = tokens;
  a.tree_mask = tree.tree_mask;
  a.u_accept = u_accept;
  a.u_sample = u_sample;
  a.path = path;
  a.n_path = n_path;
  a.next_token = next_token;
  a.accepted = accepted;
  a.stats = static_cast<ChunkStat *>(ws);
  a.logit_stride = v.logit_stride ? v.logit_stride : v.vocab;
  a.draft_stride = v.draft_stride ? v.draft_stride : v.vocab;
  a.V = v.vocab;
  a.chunks = chunks_of(v);
  a.n_seq = tree.n_seq;
  a.M = tree.n_tokens;
  a.max_tree = tree.max_tree;
  a.words = (tree.max_tree + 31) / 32;
  a.max_path = max_path;
  return v.dtype == MOESPEC_BF16 ? run_verify<uint16_t>(a, st) : run_verify<float>(a, st);
}

}  // namespace moespec
