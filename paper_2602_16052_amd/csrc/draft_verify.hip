// Verification of drafted tokens: from the target's logits and given random numbers to the accepted path and the next token.
//
// The first launch reads every row of logits once: largest logit and sum of exponentials of each chunk of a row (which rows lie on the
// path is known only behind it).  The second, one workgroup a sequence, joins the chunks of its rows, walks the tree in LDS, and draws the
// next token: the chunk in which the running sum passes its target is found from the chunks' sums, and only that chunk is read again.  With
// a drafter's distribution the difference p - q of the last row is summed over its chunks by workgroups side by side, and a third
// launch draws from it.
// Probabilities are in fp64: accepting and drawing are decisions, and have to fall the same way whatever the order of the sums.  So the
// exponentials, 20 instructions each, bound the first launch (16 trees of 63 x 50001 bf16 logits: 41 us of 52, where the bytes take 16; one tree
// x 131071: 10 of 20) and trips to memory the second (9 to 15 us).  A table of 2^x for bf16 logits in LDS was tried: 34 us for the 41, nothing
// for one tree, for a hundred lines more.
#include "serving.h"

namespace moespec {

namespace {

constexpr int kChunk = kVerifyChunk;  // logits of a wave
constexpr int kStatThreads = 256, kWalkThreads = 1024;
constexpr int kEach = kChunk / kWave;

// A chunk of a row: largest logit, its first place (greedy), sum of 2^((logit - largest) k).
struct ChunkStat {
  double sum;
  float top;
  int arg;
};

// What the walk leaves for the draw from p - q: the path's last row, 0 where nothing is to be drawn.
struct WalkEnd {
  int row, draw;
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
  double *rest;      // [n_seq][chunks] sums of p - q (draft)
  WalkEnd *ends;     // [n_seq] (draft)
  int64_t logit_stride, draft_stride;
  int V, chunks, n_seq, M, max_tree, words, max_path;
};

// log2(e) / temperature of a sequence: probabilities are 2^((logit - largest) k) over their sum.  0 where it is greedy.
__device__ __forceinline__ double heat_of(const VerifyArgs &a, int s) {
  const float t = a.temperature ? a.temperature[s] : 1.f;
  return t > 0.f ? 1.4426950408889634 / (double)fminf(fmaxf(t, 0x1p-60f), 0x1p60f) : 0.0;
}

// N sums' terms 2^t side by side, t <= 0 (or just above): t = n + r with |r| <= 1/2 (the sum with 1.5 * 2^52 rounds, and holds n in its
// low word), the polynomial of degree 10 through 2^r at the Chebyshev nodes (off by 3.2e-16 relative at most), n added to the
// exponent.  Below -1020: 2^-1020.  Drops a NaN.
template <int N>
__device__ __forceinline__ void exp2_of(double (&t)[N]) {
  constexpr double kCoef[] = {7.072585949269223e-09, 1.0208690299958306e-07, 1.321544258792169e-06, 1.5252657260200837e-05,
                              0.0001540353044173605, 0.0013333558230164974, 0.009618129107606888, 0.05550410866444772,
                              0.24022650695910097, 0.69314718055995, 1.0};
  double r[N];
  int n[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double c = fmax(t[i], -1020.0), shifted = c + 6755399441055744.0;
    n[i] = __double2loint(shifted);
    r[i] = c - (shifted - 6755399441055744.0);
    t[i] = kCoef[0];
  }
#pragma unroll
  for (int d = 1; d <= 10; ++d)
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = fma(t[i], r[i], kCoef[d]);
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = __hiloint2double(__double2hiint(t[i]) + (n[i] << 20), __double2loint(t[i]));
}
__device__ __forceinline__ double exp2_sum(double t) {
  double v[1] = {t};
  exp2_of(v);
  return v[0];
}

// The same for a single token: 0 below 2^-1022 and for -inf.  (Rows with NaN or +inf are told by their sums.)
__device__ __forceinline__ double weight_of(float x, float top, double k) {
  const double t = ((double)x - (double)top) * k;
  return t < -1022.0 ? 0.0 : exp2_sum(t);
}

template <typename T>
__device__ __forceinline__ float logit_at(const void *row, int64_t i) {
  return Elem<T>::load(static_cast<const T *>(row) + i);
}

// Lane `l`'s value in every lane.
__device__ __forceinline__ double from_lane(double v, int l) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), l), __builtin_amdgcn_readlane(__double2loint(v), l));
}
__device__ __forceinline__ double wave_sum64(double v) {
  v = row16_sum(v);
  return (from_lane(v, 0) + from_lane(v, 16)) + (from_lane(v, 32) + from_lane(v, 48));
}
__device__ __forceinline__ float row16_top(float v) {
  auto step = [&](auto ctrl) {
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false)));
  };
  step(std::integral_constant<int, kDppXor1>{});
  step(std::integral_constant<int, kDppXor2>{});
  step(std::integral_constant<int, kDppHalfMirror>{});
  step(std::integral_constant<int, kDppMirror>{});
  return v;
}
__device__ __forceinline__ float wave_top(float v) {
  v = row16_top(v);
  auto of = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return fmaxf(fmaxf(of(0), of(16)), fmaxf(of(32), of(48)));
}
// Sum of the lanes up to this one: rows of 16 by shifts, then the rows in front.
template <int N>
__device__ __forceinline__ double add_from_below(double v) {  // v of lane - N of the same row of 16, 0 where there is none
  constexpr int kShift = 0x110 + N;
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), kShift, 0xf, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), kShift, 0xf, 0xf, false);
  return v + __hiloint2double(hi, lo);
}
__device__ __forceinline__ double wave_scan64(double v) {
  v = add_from_below<1>(v);
  v = add_from_below<2>(v);
  v = add_from_below<4>(v);
  v = add_from_below<8>(v);
  const double r0 = from_lane(v, 15), r1 = r0 + from_lane(v, 31), r2 = r1 + from_lane(v, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return v + (row == 0 ? 0.0 : row == 1 ? r0 : row == 2 ? r1 : r2);
}

// A wave takes a chunk.  kVec: rows start at multiples of 16 bytes.
template <typename T, bool kVec>
__global__ __launch_bounds__(kStatThreads) void logit_stats_kernel(VerifyArgs a) {
  constexpr int E = 16 / (int)sizeof(T);
  const int row = blockIdx.y, lane = threadIdx.x & 63;
  const int chunk = __builtin_amdgcn_readfirstlane(blockIdx.x * (kStatThreads / kWave) + (int)(threadIdx.x >> 6));
  if (chunk >= a.chunks) return;
  const bool draft = blockIdx.z == 1;
  const T *x = static_cast<const T *>(draft ? a.draft : a.logits) + (int64_t)row * (draft ? a.draft_stride : a.logit_stride);
  float v[kEach];
  auto place = [&](int i) {  // of this lane's value i
    return chunk * kChunk + (kVec ? (i / E * kWave + lane) * E + i % E : i * kWave + lane);
  };
  if constexpr (kVec) {
#pragma unroll
    for (int i = 0; i < kEach; i += E) {
      const int j = place(i);
      if (j + E <= a.V) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const f32x4 f = Elem<T>::load4(x + j + e);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[i + e + k] = f[k];
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i + e] = j + e < a.V ? Elem<T>::load(x + j + e) : -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = place(i) < a.V ? Elem<T>::load(x + place(i)) : -INFINITY;
  }
  const int s = seq_of_row(a.tree_off, a.n_seq, row);
  if (s >= a.n_seq) return;
  const double k = heat_of(a, s);
  float top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kEach; i += 2) {
    top = fmaxf(fmaxf(top, v[i]), v[i + 1]);
    nan |= __builtin_isunordered(v[i], v[i + 1]);
  }
  top = wave_top(top);
  double sum = 0.0;
  int arg = 0x7fffffff;
  if (k > 0.0) {
    if (top > -INFINITY && top < INFINITY) {
      // 2^(x k - c) with c = top k rounded, one instruction less than from x - top; what c has lost is the same for all.  From |c| = 2^40 on
      // (a row of the type's lowest value) that could be anything, and the floats next to top are 2^16 away: only top itself weighs.
      const double c = (double)top * k;
      if (fabs(c) < 0x1p40) {
        constexpr int kSide = 4;  // in flight at a time; more of them, and their registers cost waves
#pragma unroll
        for (int i = 0; i < kEach; i += kSide) {
          double w[kSide];
#pragma unroll
          for (int j = 0; j < kSide; ++j) w[j] = fma((double)v[i + j], k, -c);
          exp2_of(w);
          sum += (w[0] + w[1]) + (w[2] + w[3]);
          __builtin_amdgcn_sched_barrier(0);
        }
        sum *= exp2_sum(-fma((double)top, k, -c));
      } else {
        int n = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) n += v[i] == top ? 1 : 0;
        sum = n;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (v[i] == top) arg = min(arg, place(i));
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) arg = min(arg, __shfl_xor(arg, m, kWave));
    sum = top > -INFINITY ? 1.0 : 0.0;
  }
  if (nan || top == INFINITY) sum = __builtin_nan("");
  sum = wave_sum64(sum);
  if (lane == 0) a.stats[((int64_t)blockIdx.z * a.M + row) * a.chunks + chunk] = ChunkStat{sum, top, arg};
}

// A whole row from its chunks, by the 16 lanes of a row of lanes (kWide: by a wave); all of them end with the same bits.  A lane holds its
// first four chunks, so that rows of up to 64 (256) chunks take one trip to memory.  A row of logits that is no distribution has the sum
// NaN.
struct RowStat {
  double sum;
  float top;
  int arg;
};
template <bool kWide>
__device__ __forceinline__ RowStat join_chunks(const ChunkStat *c, int chunks, double k) {
  constexpr int kLanes = kWide ? kWave : 16, kHeld = 4;
  const int first = threadIdx.x & (kLanes - 1);
  ChunkStat held[kHeld];
  float top = -INFINITY;
  int arg = 0x7fffffff;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = first + j * kLanes;
    held[j] = c[min(i, chunks - 1)];
    if (i >= chunks) held[j] = ChunkStat{0.0, -INFINITY, 0x7fffffff};
  }
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (held[j].top > top) {  // (places ascend)
      top = held[j].top;
      arg = held[j].arg;
    }
  for (int i = first + kHeld * kLanes; i < chunks; i += kLanes) {
    const ChunkStat x = c[i];
    if (x.top > top) {
      top = x.top;
      arg = x.arg;
    }
  }
  const float mine_top = top;
  top = kWide ? wave_top(top) : row16_top(top);
  if (k == 0.0) {
    arg = mine_top == top ? arg : 0x7fffffff;
#pragma unroll
    for (int m = 1; m < kLanes; m <<= 1) arg = min(arg, __shfl_xor(arg, m, kWave));
  }
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) sum += held[j].sum * weight_of(held[j].top, top, k);
  for (int i = first + kHeld * kLanes; i < chunks; i += kLanes) sum += c[i].sum * weight_of(c[i].top, top, k);
  sum = kWide ? wave_sum64(sum) : row16_sum(sum);
  return RowStat{sum > 0.0 && sum < INFINITY ? sum : __builtin_nan(""), top, arg};
}

// What the last row's tokens weigh: p, or what p has over q.
template <typename T>
struct Rest {
  const void *p, *q;  // q NULL: p
  RowStat ps, qs;
  double k, p_scale, q_scale;
  const int32_t *gone;  // LDS: tokens that weigh nothing
  int n_gone;
  __device__ __forceinline__ double of(float x, float y) const {
    const double w = weight_of(x, ps.top, k);
    return q ? fmax(w * p_scale - weight_of(y, qs.top, k) * q_scale, 0.0) : w;
  }
  __device__ __forceinline__ double operator()(int i) const {
    double w = of(logit_at<T>(p, i), q ? logit_at<T>(q, i) : 0.f);
    for (int j = 0; j < n_gone; ++j) w = gone[j] == i ? 0.0 : w;
    return w;
  }
};

struct WalkShared {
  double scan[kWalkThreads / kWave];
  int hit[kWalkThreads / kWave], some[kWalkThreads / kWave];
  int last, n_gone, next, found;
};

// Sum of v over the workgroup, the same bits in every thread.
__device__ __forceinline__ double group_sum64(double v, double *scan) {
  v = wave_sum64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) scan[threadIdx.x >> 6] = v;
  __syncthreads();
  return wave_sum64((threadIdx.x & 63) < kWalkThreads / kWave ? scan[threadIdx.x & (kWalkThreads / kWave - 1)] : 0.0);
}

// The next token of sequence s from its chunks' sums (LDS) of what is left.
template <typename T>
__device__ __forceinline__ void draw_token(const VerifyArgs &a, int s, const Rest<T> &rest, const double *chunk_sum, WalkShared &sh) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int kWaves = kWalkThreads / kWave;
  const double u = a.u_sample[s];
  double total = 0.0;
  for (int c = 0; c < a.chunks; c += kWave) total += wave_sum64(c + lane < a.chunks ? chunk_sum[c + lane] : 0.0);
  const double goal = (u > 0.0 ? fmin(u, 1.0) : 0.0) * total;  // (NaN: 0)
  double before = 0.0;
  int chunk = -1, most = 0;  // most: the last chunk with anything
  for (int c = 0; c < a.chunks && chunk < 0; c += kWave) {
    const double v = c + lane < a.chunks ? chunk_sum[c + lane] : 0.0, sum = wave_scan64(v);
    const uint64_t hit = __ballot(before + sum > goal && v > 0.0), some = __ballot(v > 0.0);
    if (hit != 0) {
      const int f = __builtin_ctzll(hit);
      chunk = c + f;
      before += f > 0 ? from_lane(sum, f - 1) : 0.0;
    } else {
      before += from_lane(sum, 63);
    }
    if (some != 0) most = c + 63 - __clzll((long long)some);
  }
  const bool past = chunk < 0;  // lost to rounding: the last token with a weight
  if (past) chunk = most;
  // the chunk's tokens: kChunk / kWalkThreads in a row to a thread
  constexpr int N = kChunk / kWalkThreads;
  double w[N], sum = 0.0;
  float x[N], y[N] = {};
  const int first = chunk * kChunk + (int)threadIdx.x * N;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = logit_at<T>(rest.p, min(first + i, a.V - 1));
  if (rest.q) {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = logit_at<T>(rest.q, min(first + i, a.V - 1));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = first + i < a.V ? rest.of(x[i], y[i]) : 0.0;
  for (int j = 0; j < rest.n_gone; ++j) {
    const int at = rest.gone[j] - first;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = at == i ? 0.0 : w[i];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) sum += w[i];
  const double scan = wave_scan64(sum);
  __syncthreads();
  if (lane == 63) sh.scan[wave] = scan;
  __syncthreads();
  const double waves = wave_scan64(lane < kWaves ? sh.scan[min(lane, kWaves - 1)] : 0.0);
  if (wave > 0) before += from_lane(waves, wave - 1);
  double run = before + scan - sum;
  int mine = -1, positive = -1;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    run += w[i];
    if (w[i] > 0.0) {
      positive = first + i;
      if (mine < 0 && run > goal) mine = first + i;
    }
  }
  // threads hold ascending places: the first hit, and the last token with a weight
  const uint64_t hits = __ballot(mine >= 0 && !past), some = __ballot(positive >= 0);
  if (lane == 0) {
    sh.hit[wave] = hits ? __builtin_amdgcn_readlane(mine, __builtin_ctzll(hits)) : -1;
    sh.some[wave] = some ? __builtin_amdgcn_readlane(positive, 63 - __clzll((long long)some)) : -1;
  }
  __syncthreads();
  if (wave == 0) {
    const int h = lane < kWaves ? sh.hit[lane] : -1, p = lane < kWaves ? sh.some[lane] : -1;
    const uint64_t hb = __ballot(h >= 0), pb = __ballot(p >= 0);
    const int token = hb ? __builtin_amdgcn_readlane(h, __builtin_ctzll(hb)) : pb ? __builtin_amdgcn_readlane(p, 63 - __clzll((long long)pb)) : -1;
    if (lane == 0) a.next_token[s] = token;
  }
}

// The walk of sequence blockIdx.y.  kSampled: with a drafter's distribution; the workgroups of a sequence then all walk its chain, and
// sum p - q over chunks of the last row between them; the draw follows in draft_draw_kernel.
template <typename T, bool kSampled, bool kWide>
__global__ __launch_bounds__(kWalkThreads) void draft_walk_kernel(VerifyArgs a) {
  constexpr int lanes = kWide ? kWave : 16;
  extern __shared__ __align__(16) unsigned char lds[];
  // [max_tree] each: probability of a token behind its parent, its random number, the row's sum, its largest logit, token, parent, and
  // the place of the largest logit (greedy) or the list of tokens that are gone (else); sampled: sum and largest logit of the drafter's
  // row.  [chunks]: sums
  double *const mine = reinterpret_cast<double *>(lds), *const number = mine + a.max_tree, *const row_sum = number + a.max_tree;
  float *const row_top = reinterpret_cast<float *>(row_sum + a.max_tree);
  int32_t *const token = reinterpret_cast<int32_t *>(row_top + a.max_tree), *const parent = token + a.max_tree;
  int32_t *const gone = parent + a.max_tree, *const row_arg = gone;
  double *const chunk_sum = reinterpret_cast<double *>(gone + a.max_tree), *const draft_sum = chunk_sum;  // (one or the other)
  float *const draft_top = reinterpret_cast<float *>(draft_sum + a.max_tree);
  __shared__ WalkShared sh;
  const int s = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool first_group = blockIdx.x == 0;
  const SeqRows g = seq_rows(a.tree_off, s, a.M, a.max_tree);
  const double k = heat_of(a, s);
  const bool greedy = k == 0.0, sampled = kSampled && !greedy;
  int32_t *const path = a.path + (int64_t)s * a.max_path;
  if (g.T == 0) {
    if (first_group) {
      for (int i = threadIdx.x; i < a.max_path; i += kWalkThreads) path[i] = -1;
      if (threadIdx.x == 0) {
        a.n_path[s] = 0;
        a.next_token[s] = -1;
        if (kSampled) a.ends[s] = WalkEnd{0, 0};
      }
    }
    return;
  }
  // tokens, their parents and logits (of a sampled chain the drafter's too), before the rows are joined: loads that wait for none of that
  for (int t0 = 0; t0 < g.T; t0 += kWalkThreads) {
    const int t = t0 + (int)threadIdx.x;
    if (t < g.T) {
      int p = t - 1;
      if (!kSampled && a.tree_mask && t > 0) {
        p = -1;
        const uint32_t *words = a.tree_mask + (int64_t)(g.row0 + t) * a.words;
        for (int w = (t - 1) >> 5; w >= 0 && p < 0; w -= 2) {
          const uint32_t high = words[w] & keys_below(t - 32 * w), low = w > 0 ? words[w - 1] : 0;
          if (high) p = 32 * w + 31 - __clz((int)high);
          else if (low) p = 32 * (w - 1) + 31 - __clz((int)low);
        }
      }
      const int x = a.tokens[g.row0 + t];
      const bool ok = p >= 0 && x >= 0 && x < a.V;
      parent[t] = p;  // -1: of no token's
      token[t] = x;
      number[t] = greedy ? 0.5 : a.u_accept[g.row0 + t];
      float l[2] = {-INFINITY, -INFINITY};
      if (ok && !greedy) {
        l[0] = logit_at<T>(static_cast<const T *>(a.logits) + (int64_t)(g.row0 + p) * a.logit_stride, x);
        if (kSampled) l[1] = logit_at<T>(static_cast<const T *>(a.draft) + (int64_t)(g.row0 + p) * a.draft_stride, x);
      }
      mine[t] = __hiloint2double(__float_as_int(l[0]), __float_as_int(l[1]));  // until the rows are there
      if (first_group && a.accepted) a.accepted[g.row0 + t] = t == 0 ? 1.f : 0.f;
    }
  }
  if (first_group)
    for (int i = threadIdx.x; i < a.max_path; i += kWalkThreads) path[i] = i == 0 ? 0 : -1;
  for (int u = threadIdx.x / lanes; u < g.T; u += kWalkThreads / lanes) {
    const RowStat r = join_chunks<kWide>(a.stats + (int64_t)(g.row0 + u) * a.chunks, a.chunks, k);
    if ((threadIdx.x & (lanes - 1)) == 0) {
      row_sum[u] = r.sum;
      row_top[u] = r.top;
      if (greedy) row_arg[u] = r.arg;
    }
    if (sampled) {
      const RowStat d = join_chunks<kWide>(a.stats + (int64_t)(a.M + g.row0 + u) * a.chunks, a.chunks, k);
      if ((threadIdx.x & (lanes - 1)) == 0) {
        draft_sum[u] = d.sum;
        draft_top[u] = d.top;
      }
    }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < g.T; t += kWalkThreads) {
    const int u = parent[t];
    double p = 0.0;
    if (u >= 0 && row_sum[u] > 0.0)
      p = greedy ? (row_arg[u] == token[t] ? 1.0 : 0.0) : weight_of(__int_as_float(__double2hiint(mine[t])), row_top[u], k) / row_sum[u];
    if (sampled) {  // a chain: decided here (NaN is no)
      const double q = u >= 0 ? weight_of(__int_as_float(__double2loint(mine[t])), draft_top[u], k) / draft_sum[u] : 0.0;
      p = number[t] * q < p ? INFINITY : 0.0;
    }
    mine[t] = p;
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
          for (int i = lane; i < n_gone; i += kWave) again |= gone[i] == x;
          if (__ballot(again) != 0) continue;
          const double p = mine[t];
          if (p > 0.0 && number[t] * (1.0 - left) < p) {
            step = t;
          } else {
            if (greedy || x < 0 || x >= a.V) continue;  // (a token of no vocabulary leaves p as it is)
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
      if (lane == 0 && first_group) {
        path[length] = step;
        if (a.accepted) a.accepted[g.row0 + step] = 1.f;
      }
      ++length;
    }
    if (lane == 0) {
      if (first_group) a.n_path[s] = length;
      sh.last = last;
      sh.n_gone = n_gone;
      sh.next = next;
      sh.found = cut;
    }
  }
  __syncthreads();
  const int64_t row = g.row0 + sh.last;
  const RowStat ps{row_sum[sh.last], row_top[sh.last], greedy ? row_arg[sh.last] : 0};
  const bool done = sh.found || !(ps.sum > 0.0) || greedy;
  if (first_group && threadIdx.x == 0) {
    if (done) a.next_token[s] = sh.found ? sh.next : ps.sum > 0.0 ? ps.arg : -1;
    if (kSampled) a.ends[s] = WalkEnd{(int)row, done ? 0 : sh.n_gone > 0 ? 2 : 1};
  }
  if (done) return;
  Rest<T> rest{static_cast<const T *>(a.logits) + row * a.logit_stride, nullptr, ps, RowStat{}, k, 1.0, 0.0, gone, 0};
  if constexpr (kSampled) {
    if (sh.n_gone == 0) return;
    rest.qs = RowStat{draft_sum[sh.last], draft_top[sh.last], 0};
    const bool some = rest.qs.sum > 0.0;  // else: p as it is
    rest.q = static_cast<const T *>(a.draft) + row * a.draft_stride;
    rest.p_scale = 1.0 / ps.sum;
    rest.q_scale = 1.0 / rest.qs.sum;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
      double sum = 0.0;
      if (some)
        for (int i = c * kChunk + (int)threadIdx.x; i < min((c + 1) * kChunk, a.V); i += kWalkThreads) sum += rest(i);
      sum = group_sum64(sum, sh.scan);
      if (threadIdx.x == 0) a.rest[(int64_t)s * a.chunks + c] = sum;
    }
  } else {
    const int n_gone = rest.n_gone = sh.n_gone;
    auto whole = [&](int c) {
      const ChunkStat st = a.stats[row * a.chunks + c];
      return st.sum * weight_of(st.top, ps.top, k);
    };
    // The sums of the chunks without the tokens that are gone.  Where these leave less than 2^-10 of a chunk, it is summed again: the
    // difference would have lost ten bits.
    uint64_t again = 0;
    for (int c0 = 0; c0 < a.chunks; c0 += kWalkThreads) {
      const int c = c0 + (int)threadIdx.x;
      if (c < a.chunks) {
        const double all = whole(c);
        double sum = all;
        for (int j = 0; j < n_gone; ++j)
          if (gone[j] >= 0 && gone[j] < a.V && gone[j] / kChunk == c)
            sum -= weight_of(logit_at<T>(rest.p, gone[j]), ps.top, k);
        const bool lost = sum < all * 0x1p-10;
        chunk_sum[c] = lost ? -1.0 : sum;
      }
    }
    __syncthreads();
    for (int c0 = 0; c0 < a.chunks && n_gone > 0; c0 += kWave) {
      again = __ballot(c0 + lane < a.chunks && chunk_sum[min(c0 + lane, a.chunks - 1)] < 0.0);
      __syncthreads();
      for (; again != 0; again &= again - 1) {
        const int c = c0 + __builtin_ctzll(again);
        double sum = 0.0;
        for (int i = c * kChunk + (int)threadIdx.x; i < min((c + 1) * kChunk, a.V); i += kWalkThreads) sum += rest(i);
        sum = group_sum64(sum, sh.scan);
        if (threadIdx.x == 0) chunk_sum[c] = sum;
      }
    }
    __syncthreads();
    bool any = false;
    for (int c = lane; c < a.chunks; c += kWave) any |= chunk_sum[c] > 0.0;
    if (__ballot(any) == 0) {  // nothing: p as it is
      __syncthreads();
      rest.n_gone = 0;
      for (int c = threadIdx.x; c < a.chunks; c += kWalkThreads) chunk_sum[c] = whole(c);
      __syncthreads();
    }
    draw_token(a, s, rest, chunk_sum, sh);
  }
}

// Sampled drafts: the next token of sequence blockIdx.x where the path ended, from p - q or, where no token was rejected or p has nothing over
// q, from p.
template <typename T>
__global__ __launch_bounds__(kWalkThreads) void draft_draw_kernel(VerifyArgs a) {
  extern __shared__ __align__(16) double chunk_sums[];
  __shared__ WalkShared sh;
  const int s = blockIdx.x, lane = threadIdx.x & 63;
  const WalkEnd end = a.ends[s];
  if (end.draw == 0) return;
  const double k = heat_of(a, s);
  const int64_t row = end.row;
  Rest<T> rest{static_cast<const T *>(a.logits) + row * a.logit_stride, nullptr, RowStat{}, RowStat{}, k, 1.0, 0.0, nullptr, 0};
  rest.ps = join_chunks<true>(a.stats + row * a.chunks, a.chunks, k);
  bool any = false;
  if (end.draw == 2) {
    for (int c = threadIdx.x; c < a.chunks; c += kWalkThreads) chunk_sums[c] = a.rest[(int64_t)s * a.chunks + c];
    __syncthreads();
    for (int c = lane; c < a.chunks; c += kWave) any |= chunk_sums[c] > 0.0;
  }
  if (__ballot(any) != 0) {
    rest.qs = join_chunks<true>(a.stats + (a.M + row) * a.chunks, a.chunks, k);
    rest.q = static_cast<const T *>(a.draft) + row * a.draft_stride;
    rest.p_scale = 1.0 / rest.ps.sum;
    rest.q_scale = 1.0 / rest.qs.sum;
  } else {
    __syncthreads();
    for (int c = threadIdx.x; c < a.chunks; c += kWalkThreads) {
      const ChunkStat st = a.stats[row * a.chunks + c];
      chunk_sums[c] = st.sum * weight_of(st.top, rest.ps.top, k);
    }
    __syncthreads();
  }
  draw_token(a, s, rest, chunk_sums, sh);
}

int chunks_of(const moespec_verify &v) { return (v.vocab + kChunk - 1) / kChunk; }

template <typename T>
hipError_t run_verify(const VerifyArgs &a, hipStream_t st) {
  const bool vec = a.logit_stride * sizeof(T) % 16 == 0 && (!a.draft || a.draft_stride * sizeof(T) % 16 == 0);
  constexpr int kWaves = kStatThreads / kWave;
  const dim3 grid((a.chunks + kWaves - 1) / kWaves, a.M, a.draft ? 2 : 1);
  if (vec) logit_stats_kernel<T, true><<<grid, kStatThreads, 0, st>>>(a);
  else logit_stats_kernel<T, false><<<grid, kStatThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int groups = a.chunks < kVerifyGroups ? a.chunks : kVerifyGroups;
  const size_t sums = (size_t)a.chunks * sizeof(double), smem = (size_t)a.max_tree * 40 + (a.draft ? (size_t)a.max_tree * 12 : sums);
  const bool wide = a.chunks > 64;
  auto walk = a.draft ? (wide ? draft_walk_kernel<T, true, true> : draft_walk_kernel<T, true, false>)
                      : (wide ? draft_walk_kernel<T, false, true> : draft_walk_kernel<T, false, false>);
  if (smem > 60 * 1024) {
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(walk), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != hipSuccess) return e;
  }
  walk<<<dim3(a.draft ? groups : 1, a.n_seq), kWalkThreads, smem, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || !a.draft) return e;
  auto draw = draft_draw_kernel<T>;
  if (sums > 60 * 1024) {
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(draw), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sums);
    if (e != hipSuccess) return e;
  }
  draw<<<a.n_seq, kWalkThreads, sums, st>>>(a);
  return hipGetLastError();
}

size_t stats_bytes(const moespec_verify &v, int M) {
  return align_up(sizeof(ChunkStat) * (size_t)M * chunks_of(v) * (v.draft_logits ? 2 : 1), 256);
}

}  // namespace

size_t draft_verify_ws(const moespec_verify &v, int n_seq, int M) {
  return stats_bytes(v, M) + (v.draft_logits ? (sizeof(double) * chunks_of(v) + sizeof(WalkEnd)) * (size_t)n_seq : 0);
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
  a.rest = reinterpret_cast<double *>(static_cast<char *>(ws) + stats_bytes(v, tree.n_tokens));
  a.ends = reinterpret_cast<WalkEnd *>(a.rest + (size_t)tree.n_seq * chunks_of(v));
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
