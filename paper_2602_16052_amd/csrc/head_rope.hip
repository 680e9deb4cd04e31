// Queries and keys made ready for attention: norm of every head, rotation to the token's place, one pass.  Bound by traffic: each row
// is read and written once.  A lane holds two pieces of 16 bytes of a head, chosen so that both elements of every rotated pair
// are its own: nothing is exchanged between lanes but the sum of squares.  The angles of a token are the same for all of its heads:
// a workgroup takes one token, and its first rot_dim / 2 threads leave sine and cosine in LDS.
// 2044 rows of 32/8 heads of 128, bf16, out of a projection: 10.0 us, 4.2 TB/s (a workgroup makes one trip to memory for what says
// where the token stands, one for its row, and the write); one token of 32/4 heads: 4.0 to 4.8 us, the launch.
#include "serving.h"

namespace moespec {

namespace {

struct RopeArgs {
  const int32_t *tree_off;
  const uint32_t *tree_mask;
  const int32_t *positions, *cache_len;
  const float *freq;
  const void *q, *k, *w_q, *w_k;
  void *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  int n_seq, M, max_tree, words, H, Hk, rot, interleaved, norm;
  float eps;
};

// Cosine and sine of place * freq.  The angle is reduced to a quarter turn in 64 bits, with what the products round off carried along (a
// product rounded once is off by 2.4e-7 at place 2^31): what is left is at most pi / 4 and rounded to fp32 once (2.4e-8 at
// most), up to 2^50 quarter turns.
__device__ __forceinline__ float2 turn(double place, float freq) {
#pragma clang fp contract(off)  // (a difference that took the place of its rounded product would count the rest twice)
  constexpr double kQuarters = 0.63661977236758134, kQuartersRest = -3.935735335036497e-17;  // 2 / pi
  const double x = place * (double)freq, x_rest = fma(place, (double)freq, -x);
  const double quarters = x * kQuarters, rest = fma(x, kQuarters, -quarters) + fma(x, kQuartersRest, x_rest * kQuarters);
  const double n = rint(quarters);
  float s, c;
  sincospif(0.5f * (float)((quarters - n) + rest), &s, &c);
  const int k = (int)(n - 4.0 * floor(0.25 * n));
  if (k & 1) {
    const float x = s;
    s = c;
    c = -x;
  }
  return (k & 2) ? make_float2(-c, -s) : make_float2(c, s);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void head_rope_kernel(RopeArgs a) {
  typedef Piece<T> P;
  constexpr int E = P::kElems, kPieces = D / E, kLanes = kPieces / 2, W = pow2_ceil(kLanes), kHeads = 256 / W;
  __shared__ float2 cs[D / 2];
  const int row = blockIdx.x, lane = threadIdx.x & 63, j = threadIdx.x % W;
  const int s = seq_of_row(a.tree_off, a.n_seq, row);
  if (s >= a.n_seq) return;
  const SeqRows g = seq_rows(a.tree_off, s, a.M, a.max_tree);
  const int t = row - g.row0;
  if (t < 0 || t >= g.T) return;
  if (a.rot > 0) {
    double place;
    if (a.positions) {
      place = a.positions[row];
    } else {
      int seen = t + 1;
      if (a.tree_mask) {
        seen = 0;
        for (int w = lane; 32 * w < g.T; w += kWave)
          seen += __popc(a.tree_mask[(size_t)row * a.words + w] & keys_below(g.T - 32 * w));
        seen = wave_sum(seen);
      }
      place = (double)(a.cache_len ? max(a.cache_len[s], 0) : 0) + (seen - 1);
    }
    if ((int)threadIdx.x < a.rot / 2) cs[threadIdx.x] = turn(place, a.freq[threadIdx.x]);
  }
  __syncthreads();
  const int rp = a.rot / E;  // rotated pieces
  int p0 = 2 * j, p1 = 2 * j + 1;
  if (!a.interleaved && j < rp / 2) {
    p0 = j;
    p1 = j + rp / 2;
  }
  const bool there = j < kLanes;
  for (int h = threadIdx.x / W; h < a.H + a.Hk; h += kHeads) {
    const bool is_q = h < a.H;
    if ((is_q ? a.q : a.k) == nullptr) continue;
    const int hh = is_q ? h : h - a.H;
    const T *x = static_cast<const T *>(is_q ? a.q : a.k) + (int64_t)row * (is_q ? a.q_stride : a.k_stride) + hh * D;
    T *y = static_cast<T *>(is_q ? a.q_out : a.k_out) + (int64_t)row * (is_q ? a.q_out_stride : a.k_out_stride) + hh * D;
    float v0[E], v1[E];
    if (there) {
      P::load(x + p0 * E, v0);
      P::load(x + p1 * E, v1);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v0[e] = v1[e] = 0.f;
    }
    if (a.norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(v0[e], v0[e], fmaf(v1[e], v1[e], ss));
#pragma unroll
      for (int m = 1; m < W; m <<= 1) ss += __shfl_xor(ss, m, kWave);
      const float f = 1.f / sqrtf(ss / (float)D + a.eps);
      const T *w = static_cast<const T *>(is_q ? a.w_q : a.w_k);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v0[e] *= f;
        v1[e] *= f;
      }
      if (w && there) {
        float w0[E], w1[E];
        P::load(w + p0 * E, w0);
        P::load(w + p1 * E, w1);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          v0[e] *= w0[e];
          v1[e] *= w1[e];
        }
      }
    }
    if (2 * j < rp) {
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 r0 = cs[(p0 * E + e) / 2], r1 = cs[(p1 * E + e) / 2];
          const float a0 = v0[e], a1 = v1[e];
          v0[e] = a0 * r0.x - v0[e + 1] * r0.y;
          v0[e + 1] = v0[e + 1] * r0.x + a0 * r0.y;
          v1[e] = a1 * r1.x - v1[e + 1] * r1.y;
          v1[e + 1] = v1[e + 1] * r1.x + a1 * r1.y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 r = cs[j * E + e];
          const float a0 = v0[e];
          v0[e] = a0 * r.x - v1[e] * r.y;
          v1[e] = v1[e] * r.x + a0 * r.y;
        }
      }
    }
    if (there) {
      P::store(y + p0 * E, v0);
      P::store(y + p1 * E, v1);
    }
  }
}

template <typename T>
hipError_t run_rope(int D, const RopeArgs &a, hipStream_t st) {
  auto run = [&](auto kern) {
    kern<<<a.M, 256, 0, st>>>(a);
    return hipGetLastError();
  };
  switch (D) {
    case 64: return run(head_rope_kernel<T, 64>);
    case 96: return run(head_rope_kernel<T, 96>);
    case 128: return run(head_rope_kernel<T, 128>);
    case 192: return run(head_rope_kernel<T, 192>);
    default: return run(head_rope_kernel<T, 256>);
  }
}

}  // namespace

hipError_t launch_head_rope(const moespec_attn_desc &ds, const moespec_rope &r, const moespec_tree &tree, const void *q,
                            const void *k, void *q_out, void *k_out, hipStream_t st) {
  const int64_t qs = (int64_t)ds.n_heads * ds.head_dim, ks = (int64_t)ds.n_kv_heads * ds.head_dim;
  RopeArgs a{};
  a.tree_off = tree.tree_off;
  a.tree_mask = tree.tree_mask;
  a.positions = r.positions;
  a.cache_len = r.cache_len;
  a.freq = r.freq;
  a.q = q;
  a.k = k;
  a.w_q = r.w_q;
  a.w_k = r.w_k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_stride = tree.q_stride ? tree.q_stride : qs;
  a.k_stride = tree.kv_stride ? tree.kv_stride : ks;
  a.q_out_stride = r.q_out_stride ? r.q_out_stride : qs;
  a.k_out_stride = r.k_out_stride ? r.k_out_stride : ks;
  a.n_seq = tree.n_seq;
  a.M = tree.n_tokens;
  a.max_tree = tree.max_tree;
  a.words = (tree.max_tree + 31) / 32;
  a.H = ds.n_heads;
  a.Hk = ds.n_kv_heads;
  a.rot = r.rot_dim;
  a.interleaved = r.interleaved;
  a.norm = r.norm;
  a.eps = r.eps;
  return ds.dtype == MOESPEC_BF16 ? run_rope<uint16_t>(ds.head_dim, a, st) : run_rope<float>(ds.head_dim, a, st);
}

}  // namespace moespec
