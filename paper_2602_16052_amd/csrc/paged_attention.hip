// Attention of one new token of every sequence over its pages of keys and values, which may be held in 8 bits.
//
// Bound by the stream of keys and values: each is read once for all query heads that share it.  One pass with a running maximum m and
// sum l for each head: p = 2^(c (q.k - m)), l += p, O += p V, out = O / l; the scale of a key's row multiplies its
// score, that of a value's row its weight.  The keys are split into parts (few sequences) that a second kernel joins.
//
// The query heads of a KV head are the 16 columns of matrix instructions (unused ones repeat a head and are not written).  S = K Q^T
// takes keys as they come from memory: lane l holds 16 bytes of key l % 16, piece l / 16, and queries are loaded in the
// same order of elements.  A lane's scores, key 4 (l / 16) + i of head l % 16, are already the right operand of O^T = V^T P^T.
// Values lie in rows and are needed in columns: a wave lays its own through LDS (rows of D elements and a pad that keeps the
// transposing reads off each other's banks).  Waves share nothing until their results are joined at the end.
// A wave requests the next tile's keys when the products have used up their registers, and its values when these lie in LDS, so that
// one of the two is always under way.
// 64 requests x 8 heads of 128, up to 8189 bf16 entries: 263 us, 6.2 TB/s (a read-only stream reaches 6.4); int8, 48 x 4 heads, up to 16381: 117
// us, 5.4 TB/s (the vector ALU, which widens the codes, is busy for over 40 % of the cycles, and 38 % of the LDS cycles are bank conflicts: the stores of
// widened values, pieces of 16 bytes 32 apart); e4m3, one request over 131071: 29 us, 4.7 TB/s (2 us of start, 5.5 of joining 128 parts); one
// over 1021 bf16 entries: 8.7 us, two launches.
// fp32 layers over codes with heads of 128 keep 60 bytes a lane in scratch (168 registers, for three workgroups a compute unit).
#include "serving.h"

namespace moespec {

namespace {

struct PagedAttnArgs {
  KeyArgs keys;  // q, cache_len, lengths and heads (one token of every sequence)
  Pages pages;
  int head_tiles, slots;  // tiles of 16 query heads; parts of all sequences together, 0: every sequence is one part
  // 2^-8 / 2^k with 2^k >= max_len: what weights of 1 enter the products as (exactly).  Weights are up to 2^8 before the maximum is raised, and so the
  // sum over a sequence's keys is no larger than the largest value: finite wherever that is, as the result is.  (Without it values from 2^-8
  // of the largest number on, or many keys of the same score, are infinities.)  us without and with it: 48 requests over int8 rows of 128 117.9 and 117.5, 30 over ones of
  // 192 61.0 and 63.2, 64 over bf16 ones 263.6 and 263.5, four of fp32 12.2 and 12.3; by each sequence's own length, which joining then has to
  // load, 118.2, 61.3, 263.9 and 12.6.
  float unit;
};

template <typename T, int CODE, int D>
struct PagedShape {
  static constexpr bool kCodes = CODE != MOESPEC_CACHE_PLAIN;
  // Codes are exact in bf16, and so an fp32 layer over codes takes bf16 products too, with queries and weights in three parts (24 bits):
  // fp32 products of 16 requests, 8 heads of 96 over up to 3000 entries took 35.8 us, these 22.3.
  static constexpr bool kBf16 = sizeof(T) == 2 || kCodes;
  static constexpr int kQParts = sizeof(T) == 2 || !kBf16 ? 1 : 3, kPParts = sizeof(T) == 2 ? 2 : 3;
  static constexpr int kWaves = 4;
  static constexpr int kHalves = kBf16 ? 2 : 1, kKeys = 16 * kHalves;  // keys of a wave's tile
  static constexpr int kUnit = kKeys * kWaves;                         // ... of a workgroup's
  static constexpr int kHeld = kCodes ? 1 : (int)sizeof(T);            // bytes of an element in a page
  static constexpr int kRowBytes = D * kHeld;
  static constexpr int kLoads = (kRowBytes + 63) / 64;     // loads of 64 bytes of 16 keys; the last one may be of 32
  static constexpr bool kTail = kRowBytes % 64 != 0;       // (8-bit rows of 96: 8 bytes a lane)
  static constexpr int kPiece = 16 / kHeld;                // elements of a lane's 16 bytes
  static constexpr int kStride = kBf16 ? 2 * D + 32 : 4 * D + 16;  // bytes of a value's row in LDS
  static constexpr int kTileLds = kKeys * kStride;
  static constexpr int kValueLanes = kRowBytes / 16;       // lanes that hold a row of values
  static constexpr int kValueRows = 64 / pow2_ceil(kValueLanes) < kKeys ? 64 / pow2_ceil(kValueLanes) : kKeys;  // rows of a load
  static constexpr int kValueLoads = kKeys / kValueRows;
  // Workgroups wanted: one round of what the compute units hold by registers (up to three each, or one with long rows), two each where
  // parts are short, which then have as many again to join.  us with 512 and with 768: 48 requests over int8 rows of 128 123 and 116, 64
  // over bf16 ones 266 and 263, one over 131071 e4m3 rows 29.2 and 31.9; with 512 and with 256: bf16 rows of 192 46.5 and 41.5, fp32
  // ones of 256 36.5 and 30.9, int8 ones of 256 56.2 and 51.6.  8-bit rows of 192 in bf16 layers, of which two fit, are the exception: 30 requests x 4
  // heads over 5000 int8 entries 51.6 and 62.5, e4m3 48.8 and 56.4.
  static constexpr bool kLong = D >= 192 || kRowBytes >= 512;
  static int target(int64_t all_units) { return kLong ? 256 : all_units >= 16 * 768 ? 768 : 512; }
  static constexpr int kJoinRow = D + 4;  // floats; the pad keeps the 16 heads of a store off each other's banks
  static constexpr int kJoin = kWaves * 16 * (kJoinRow + 2) * (int)sizeof(float);
  static constexpr int kLds = kWaves * kTileLds > kJoin ? kWaves * kTileLds : kJoin;
};

// Eight codes as bf16 (exact: bf16 has no fewer bits).
template <int CODE>
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t a, uint32_t b) {
  bf16x8 v;
  if constexpr (CODE == MOESPEC_CACHE_I8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = (__bf16)(float)(int8_t)(a >> (8 * e));
      v[4 + e] = (__bf16)(float)(int8_t)(b >> (8 * e));
    }
  } else {  // two at a time
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true)};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p[e / 2][e % 2];
  }
  return v;
}

// Eight numbers as the sum of N bf16 ones: each is the rounding of what those before it leave.
template <int N>
__device__ __forceinline__ void split(float (&v)[8], bf16x8 (&part)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      part[j][i] = (__bf16)v[i];
      v[i] -= (float)part[j][i];
    }
}

// Eight weights in two parts that are both above 0 where the weight is, so that a value of infinity stays one: cut off, and the rest, which is
// 2^-16 of the weight at least (off by 2^-15 of it at most).
__device__ __forceinline__ void split_above_zero(const float (&v)[8], bf16x8 (&part)[2]) {
  uint32_t cut[4];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    cut[i / 2] = __builtin_amdgcn_perm(__float_as_uint(v[i + 1]), __float_as_uint(v[i]), 0x07060302u);
#pragma unroll
    for (int j = i; j < i + 2; ++j) part[1][j] = (__bf16)fmaxf(v[j] - __uint_as_float(__float_as_uint(v[j]) & 0xffff0000u), v[j] * 0x1p-16f);
  }
  part[0] = __builtin_bit_cast(bf16x8, cut);
}

// 16 bytes that nobody reads again soon.  Values come in whole lines and are requested so: 64 requests 293 -> 266 us (6.1 TB/s), int8 130 ->
// 123, one over 131071 e4m3 entries 33.1 -> 29.3.  A load of keys takes half a line of every row, and the other half has to stay until
// the next one: with keys requested so too, 284, 122 and 30.8.
__device__ __forceinline__ uint4 stream_load(const unsigned char *p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p)));
}

// v of the lanes that hold the same head, l ^ 16 and l ^ 32, combined.
__device__ __forceinline__ float head_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  return half_swap(v, true);
}
__device__ __forceinline__ float head_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  return half_swap(v, false);
}

// log sum exp of a row from its largest score, the sum of 2^(c (score - largest)), and c.  (c and the logarithm are brought to natural units
// first: finite wherever the result is.)
__device__ __forceinline__ float lse_of(float m, float l, float c) {
  constexpr float kLn2 = 0.69314718055994531f;
  return l == 0.f ? -INFINITY : fmaf(m, c * kLn2, __log2f(l) * kLn2);
}

template <typename T, int CODE, int D>
__global__ __launch_bounds__(256, (D <= 128 ? 3 : 1)) void paged_attention_kernel(PagedAttnArgs a, T *__restrict__ out, float *__restrict__ lse,
                                                              float *__restrict__ part, float2 *__restrict__ part_ml,
                                                              int32_t *__restrict__ first_of) {
  typedef PagedShape<T, CODE, D> P;
  constexpr int NB = D / 16;
  extern __shared__ __align__(16) unsigned char lds[];
  const KeyArgs &ka = a.keys;
  const Pages &pg = a.pages;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g4 = lane >> 4;
  // head tiles that share keys are neighbours on one XCD (workgroup b runs on XCD b mod 8)
  const int slot = blockIdx.x / 8, group = slot / a.head_tiles * 8 + (int)(blockIdx.x % 8), tile = slot % a.head_tiles;
  const int n_parts = a.slots == 0 ? ka.n_seq : a.slots, index = group % n_parts, hk = group / n_parts;
  if (hk >= ka.Hk) return;
  auto units = [&](const SeqGeom &g) { return (g.len + P::kUnit - 1) / P::kUnit; };
  const Share share = share_of(ka, a.slots, index, units, blockIdx.x == 0 ? first_of : nullptr);
  const int s = share.s;
  if (s < 0) return;
  const int len = seq_geom(ka, s).len, all = (len + P::kUnit - 1) / P::kUnit;
  const int u0 = share.first(all), u1 = share.last(all);
  const int h = hk * ka.G + min(tile * 16 + n16, ka.G - 1);

  // queries, in the order of a lane's keys
  typename std::conditional<P::kBf16, bf16x8, f32x4>::type q[P::kQParts][P::kBf16 ? D / 32 : D / 16];
  {
    const T *qp = static_cast<const T *>(ka.q) + (int64_t)s * ka.q_stride + h * D;
    if constexpr (!P::kBf16) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) q[0][i] = *reinterpret_cast<const f32x4 *>(qp + 16 * i + 4 * g4);
    } else {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const int at = !P::kCodes || (P::kTail && i == D / 32 - 1) ? 32 * i + 8 * g4 : i / 2 * 64 + 16 * g4 + 8 * (i % 2);
        if constexpr (sizeof(T) == 2) {
          q[0][i] = *reinterpret_cast<const bf16x8 *>(qp + at);
        } else {
          const f32x4 lo = *reinterpret_cast<const f32x4 *>(qp + at), hi = *reinterpret_cast<const f32x4 *>(qp + at + 4);
          float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          bf16x8 part[P::kQParts];
          split<P::kQParts>(v, part);
#pragma unroll
          for (int j = 0; j < P::kQParts; ++j) q[j][i] = part[j];
        }
      }
    }
  }

  f32x4 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  unsigned char *const my = lds + wave * P::kTileLds;
  const uint32_t my_lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)my);

  uint4 kr[P::kHalves][P::kLoads], vr[P::kValueLoads];
  f32x4 ks[P::kHalves], vs[P::kHalves];
  const int vrow = lane / pow2_ceil(P::kValueLanes), vpiece = lane % pow2_ceil(P::kValueLanes);
  const uint32_t kat = n16 * P::kRowBytes, vat = vrow * P::kRowBytes + 16 * min(vpiece, P::kValueLanes - 1);
  // Pages of this wave's next tiles, one half of a tile to a lane: the table is read once every 64 / kHalves tiles.
  int ids = 0;
  auto page_ids = [&](int u) {
    const int64_t e = (int64_t)(u + lane / P::kHalves) * P::kUnit + wave * P::kKeys + 16 * (lane % P::kHalves);
    ids = pg.table[(int64_t)s * pg.max_pages + ((int)min(e, (int64_t)len - 1) >> pg.log_page)];
  };
  // First row (of D elements) of 16 entries from e on in the pool; of some page that is there where theirs is not.
  auto page_there = [&](int u, int x) {
    const int p = __builtin_amdgcn_readlane(ids, ((u - u0) * P::kHalves + x) & 63);
    return p >= 0 && p < pg.n_pages;
  };
  auto row_of = [&](int u, int x) {
    const int p = __builtin_amdgcn_readlane(ids, ((u - u0) * P::kHalves + x) & 63);
    const int e = u * P::kUnit + wave * P::kKeys + 16 * x;
    return pg.row(0, p >= 0 && p < pg.n_pages ? p : 0, hk, e);
  };
  auto load_keys = [&](int u) {
#pragma unroll
    for (int x = 0; x < P::kHalves; ++x) {
      const int64_t row = row_of(u, x);
      const unsigned char *at = pg.k + row * P::kRowBytes;
#pragma unroll
      for (int i = 0; i < P::kLoads; ++i) {
        if (P::kTail && i == P::kLoads - 1) {
          const uint2 two = *reinterpret_cast<const uint2 *>(at + (kat + 8 * g4) + 64 * i);
          kr[x][i] = make_uint4(two.x, two.y, 0, 0);
        } else {
          kr[x][i] = *reinterpret_cast<const uint4 *>(at + (kat + 16 * g4) + 64 * i);
        }
      }
      if (P::kCodes) ks[x] = *reinterpret_cast<const f32x4 *>(pg.k_scale + row + 4 * g4);
    }
  };
  auto load_values = [&](int u) {
#pragma unroll
    for (int x = 0; x < P::kHalves; ++x) {
      const int64_t row = row_of(u, x);
      const unsigned char *at = pg.v + row * P::kRowBytes;
#pragma unroll
      for (int j = 0; j < P::kValueLoads / P::kHalves; ++j)
        vr[x * (P::kValueLoads / P::kHalves) + j] = stream_load(at + vat + j * P::kValueRows * P::kRowBytes);
      if (P::kCodes) vs[x] = *reinterpret_cast<const f32x4 *>(pg.v_scale + row + 4 * g4);
    }
  };

  const int mine = min(u1, (len - wave * P::kKeys + P::kUnit - 1) / P::kUnit);  // units in which this wave has a key
  if (u0 < mine) {
    page_ids(u0);
    load_keys(u0);
    load_values(u0);
  }
  for (int u = u0; u < mine; ++u) {
    const int e0 = u * P::kUnit + wave * P::kKeys;
    bool there[P::kHalves], whole = e0 + P::kKeys <= len;
#pragma unroll
    for (int x = 0; x < P::kHalves; ++x) {
      there[x] = page_there(u, x);
      whole &= there[x];
    }
    // (the table's next pages, behind the last use of these)
    const bool more = u + 1 < mine;
    if (more && (u + 1 - u0) % (64 / P::kHalves) == 0) page_ids(u + 1);
    f32x4 sc[P::kHalves];
#pragma unroll
    for (int x = 0; x < P::kHalves; ++x) {
      sc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
      const uint32_t *w = reinterpret_cast<const uint32_t *>(kr[x]);
      if constexpr (P::kBf16) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          bf16x8 k;
          if constexpr (P::kCodes) k = codes_bf16<CODE>(w[2 * i], w[2 * i + 1]);
          else k = __builtin_bit_cast(bf16x8, kr[x][i]);
#pragma unroll
          for (int j = 0; j < P::kQParts; ++j) sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[j][i], sc[x], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < D / 4; ++i) {
          sc[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), q[0][i / 4][i % 4], sc[x], 0, 0, 0);
        }
      }
      if (P::kCodes)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[x][i] *= ks[x][i];
    }
    if (more) load_keys(u + 1);  // into the registers that the products have left
    f32x4 vscale[P::kHalves];
#pragma unroll
    for (int x = 0; x < P::kHalves; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) vscale[x][i] = P::kCodes ? vs[x][i] * a.unit : 0.f;
    if (!whole) {  // what is not seen has no score, and must meet weights of 0 as numbers
#pragma unroll
      for (int x = 0; x < P::kHalves; ++x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool seen = there[x] && e0 + 16 * x + 4 * g4 + i < len;
          sc[x][i] = seen ? sc[x][i] : -INFINITY;
          vscale[x][i] = seen ? vscale[x][i] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < P::kValueLoads / P::kHalves; ++j) {
          const bool seen = there[x] && e0 + 16 * x + j * P::kValueRows + vrow < len;
          uint4 &v = vr[x * (P::kValueLoads / P::kHalves) + j];
          v = make_uint4(seen ? v.x : 0u, seen ? v.y : 0u, seen ? v.z : 0u, seen ? v.w : 0u);
        }
      }
    }
    // values to LDS
    if (vpiece < P::kValueLanes) {
#pragma unroll
      for (int i = 0; i < P::kValueLoads; ++i) {
        unsigned char *to = my + (i * P::kValueRows + vrow) * P::kStride;
        const uint32_t w[4] = {vr[i].x, vr[i].y, vr[i].z, vr[i].w};
        if constexpr (!P::kCodes) {
          *reinterpret_cast<uint4 *>(to + 16 * vpiece) = vr[i];
        } else {
          *reinterpret_cast<bf16x8 *>(to + 32 * vpiece) = codes_bf16<CODE>(w[0], w[1]);
          *reinterpret_cast<bf16x8 *>(to + 32 * vpiece + 16) = codes_bf16<CODE>(w[2], w[3]);
        }
      }
    }
    if (more) load_values(u + 1);
    float mx = -INFINITY;
#pragma unroll
    for (int x = 0; x < P::kHalves; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[x][i]);
    mx = head_max(mx);
    // raised only when it is passed by more than 2^8: until then weights stay below 2^8, as exact as below 1, and O is not rescaled (raised every time:
    // int8 rows of 128 118.9 us for 118.1, of 192 62.1 for 61.2).  Scores are subtracted before they are scaled, so that the largest weighs 1 (up
    // to 2^8) however large it is.
    const bool raise = (mx - m) * ka.c > 8.f;
    if (__ballot(raise) != 0) {
      const float alpha = raise ? __builtin_amdgcn_exp2f((m - mx) * ka.c) : 1.f;
      m = raise ? mx : m;
      l *= alpha;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[b][i] *= alpha;
    }
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int x = 0; x < P::kHalves; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[x][i] = __builtin_amdgcn_exp2f((sc[x][i] - mu) * ka.c);
        l += sc[x][i];
        sc[x][i] *= P::kCodes ? vscale[x][i] : a.unit;
      }
    asm volatile("" ::: "memory");  // the wave's own rows: LDS keeps their order
    if constexpr (P::kBf16) {
      // The matrix instructions take bf16 weights beside bf16 values: a weight goes in as its rounding and what that leaves (off by 2^-16 of
      // it at most; fp32 layers: in three parts, 2^-24), so that outputs are as exact as their own rounding.  With the rounding alone
      // they are 0.0023 off (root of the mean square, relative) where that leaves 0.0017; the other products are hidden behind the
      // stream of keys and values.
      bf16x8 p[P::kPParts];
      float weights[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) weights[i] = sc[i / 4][i % 4];
      if constexpr (P::kCodes) split<P::kPParts>(weights, p);
      else split_above_zero(weights, p);
      // lane i of 16 points at 4 elements of row i / 4 and receives element i of 4 rows
      typedef __attribute__((address_space(3))) bf16x4 lds4;
      const uint32_t at = my_lds + (4 * g4 + (n16 >> 2)) * P::kStride + 8 * (n16 & 3);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(uintptr_t)(at + 32 * b));
        const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4 *)(uintptr_t)(at + 16 * P::kStride + 32 * b));
        const bf16x8 v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int j = 0; j < P::kPParts; ++j) o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[j], o[b], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = *reinterpret_cast<const float *>(my + (4 * g4 + i) * P::kStride + 64 * b + 4 * n16);
          o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, sc[0][i], o[b], 0, 0, 0);
        }
    }
    asm volatile("" ::: "memory");
  }
  l = head_sum(l);
  if (m == -INFINITY && l != 0.f) m = 0.f;  // scores that are all NaN: so is the row

  // the waves' results joined: [wave][head]{m, l}, then [wave][head][D].  Here and between parts m stays a score: maxima are subtracted before they are
  // scaled, so that a key weighs the same whichever wave or part it falls to.  (Scaled ones, rounded, would be off by half a unit of log 2 at 2^23.)
  __syncthreads();
  float2 *ml = reinterpret_cast<float2 *>(lds);
  float *op = reinterpret_cast<float *>(lds + P::kWaves * 16 * sizeof(float2));
  if (g4 == 0) ml[wave * 16 + n16] = make_float2(m, l);
#pragma unroll
  for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4 *>(op + (wave * 16 + n16) * P::kJoinRow + 16 * b + 4 * g4) = o[b];
  __syncthreads();
  const int heads = min(16, ka.G - tile * 16);
  for (int id = threadIdx.x; id < heads * (D / 4); id += 256) {
    const int n = id / (D / 4), d = 4 * (id % (D / 4));
    float mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int w = 0; w < P::kWaves; ++w) mt = fmaxf(mt, ml[w * 16 + n].x);
    const float mu = mt == -INFINITY ? 0.f : mt;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < P::kWaves; ++w) {
      const float2 x = ml[w * 16 + n];
      const float f = __builtin_amdgcn_exp2f((x.x - mu) * ka.c);
      lt = fmaf(x.y, f, lt);
      const f32x4 y = *reinterpret_cast<const f32x4 *>(op + (w * 16 + n) * P::kJoinRow + d);
      if (x.x != -INFINITY) {  // a wave without keys has no values
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(y[e], f, v[e]);
      }
    }
    const int head = hk * ka.G + tile * 16 + n;
    if (a.slots == 0) {
      const size_t row = (size_t)s * ka.H + head;
      const float inv = lt == 0.f ? 0.f : 1.f / (lt * a.unit);
      Elem<T>::store4(out + row * D + d, lt == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv});
      if (lse && d == 0) lse[row] = lse_of(mt, lt, ka.c);
    } else {
      const size_t row = (size_t)index * ka.H + head;
      *reinterpret_cast<f32x4 *>(part + row * D + d) = v;
      if (d == 0) part_ml[row] = make_float2(mt, lt);
    }
  }
}

// The parts of a token's keys joined: a workgroup of D / 4 x kGroups threads per head, the parts shared out to the groups.
constexpr int kGroups = 8;
template <typename T, int D>
__global__ __launch_bounds__(kGroups *D / 4) void paged_join_kernel(KeyArgs a, int slots, float unit, const float *__restrict__ part,
                                                                   const float2 *__restrict__ part_ml,
                                                                   const int32_t *__restrict__ first_of, T *__restrict__ out,
                                                                   float *__restrict__ lse) {
  constexpr int kCols = D / 4;
  __shared__ float2 ml[kGroups];
  __shared__ f32x4 po[kGroups][kCols];
  const int col = threadIdx.x % kCols, grp = threadIdx.x / kCols, head = blockIdx.x, s = blockIdx.y;
  const int p0 = a.n_seq == 1 ? 0 : first_of[s], n = a.n_seq == 1 ? slots : first_of[s + 1] - p0;
  float m = -INFINITY, l = 0.f;
  f32x4 o{0.f, 0.f, 0.f, 0.f};
  for (int i0 = grp; i0 < n; i0 += 4 * kGroups) {
    float2 x[4];
    f32x4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const size_t row = (size_t)(p0 + min(i0 + j * kGroups, n - 1)) * a.H + head;
      x[j] = part_ml[row];
      v[j] = *reinterpret_cast<const f32x4 *>(part + row * D + 4 * col);
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = fmaxf(top, i0 + j * kGroups < n ? x[j].x : -INFINITY);
    const float mu = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f((m - mu) * a.c);
    l *= f0;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + j * kGroups >= n || x[j].x == -INFINITY) continue;
      const float f = __builtin_amdgcn_exp2f((x[j].x - mu) * a.c);
      l = fmaf(f, x[j].y, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[j][e], o[e]);
    }
    m = top;
  }
  po[grp][col] = o;
  if (col == 0) ml[grp] = make_float2(m, l);
  __syncthreads();
  if (grp > 0) return;
  float top = m;
#pragma unroll
  for (int g = 1; g < kGroups; ++g) top = fmaxf(top, ml[g].x);
  const float mu = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f((m - mu) * a.c);
  l *= f0;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
  for (int g = 1; g < kGroups; ++g) {
    const float f = __builtin_amdgcn_exp2f((ml[g].x - mu) * a.c);
    l = fmaf(f, ml[g].y, l);
    const f32x4 v = po[g][col];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(f, v[e], o[e]);
  }
  const size_t row = (size_t)s * a.H + head;
  const float inv = l == 0.f ? 0.f : 1.f / (l * unit);
  Elem<T>::store4(out + row * D + 4 * col, l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv});
  if (lse && col == 0) lse[row] = lse_of(top, l, a.c);
}

constexpr int kMostGroups = 768;      // workgroups wanted, at most
constexpr size_t kFirstBytes = 2048;  // first parts of up to kMaxShared sequences

// Short caches and many sequences are not split: a unit of keys takes a workgroup 1.2 us, the launch that joins parts 2.5 to 6.  us whole and
// in parts, heads of 128 (of 256 where it says so), bf16, with int8 behind them: 4 heads of one sequence (workgroups), 250 entries (2 units) 6.9 and 8.4, 500
// entries 9.7 and 8.5; 64 of them, 500 10.7 and 11.4, 1000 17.0 and 13.9; 160, 1000 19.8 and 23.1 (19.8 and 19.2), 2000 34.1 and 36.4 (34.3 and
// 26.6), 4000 62.1 and 59.3 (63.2 and 39.4); 400, 2000 69.9 and 74.2 (44.6 and 52.6), 4000 132 and 141 (82 and 89); rows of 256, 64
// workgroups, 250 entries 12.7 and 14.1, 500 18.9 and 16.5.  The rule counts rows of 128 and of 256 bytes alike, which suits int8 at 160
// workgroups and costs bf16 7 % there (2000 entries), and it takes the parts, 6 to 9 % slower, at 400 workgroups and 4000 entries.
// Parts are what cuts a sequence that is much longer than the others: as many sequences as target / (Hk * head_tiles), or more, have none
// to spare.  A request of 131071 bf16 entries (8 KV heads; alone 87 us) among 63 of 100 entries takes 93 us, among 94 834, among 95 1635,
// among 127 4250 (its eight workgroups are then on one XCD).
// Parts of all sequences together: enough for `target` workgroups, none without a unit of keys; 0 where every sequence is one part.
int slots_of(int64_t target, int64_t n_seq, int64_t Hk, int64_t head_tiles, int64_t max_len, int64_t unit, int64_t row_bytes) {
  const int64_t units = (max_len + unit - 1) / unit, groups = n_seq * Hk * head_tiles;
  if (units * (row_bytes > 256 ? row_bytes : 256) <= (2 + groups / 26) * 256) return 0;
  int64_t n = target / (Hk * head_tiles);
  if (n > n_seq * units) n = n_seq * units;
  if (n_seq == 1 && n > kMaxParts) n = kMaxParts;
  return n <= n_seq || n_seq > kMaxShared ? 0 : (int)n;
}

template <typename T, int CODE, int D>
hipError_t run_paged(const PagedAttnArgs &args, void *out, float *lse, void *ws, hipStream_t st) {
  typedef PagedShape<T, CODE, D> P;
  PagedAttnArgs a = args;
  const KeyArgs &k = a.keys;
  const int64_t units = ((int64_t)k.max_len + P::kUnit - 1) / P::kUnit * k.n_seq * k.Hk * a.head_tiles;
  a.slots = slots_of(P::target(units), k.n_seq, k.Hk, a.head_tiles, k.max_len, P::kUnit, P::kRowBytes);
  auto kern = paged_attention_kernel<T, CODE, D>;
  static_assert(P::kLds <= 160 * 1024, "LDS of a compute unit");
  if (P::kLds > 64 * 1024) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, P::kLds);
    if (e != hipSuccess) return e;
  }
  int32_t *first_of = static_cast<int32_t *>(ws);
  float *part = reinterpret_cast<float *>(static_cast<char *>(ws) + kFirstBytes);
  float2 *ml = reinterpret_cast<float2 *>(part + (size_t)a.slots * k.H * D);
  const int64_t groups = (int64_t)k.Hk * (a.slots == 0 ? k.n_seq : a.slots);
  kern<<<(unsigned)((groups + 7) / 8 * 8 * a.head_tiles), 256, P::kLds, st>>>(a, static_cast<T *>(out), lse, part, ml, first_of);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.slots == 0) return e;
  paged_join_kernel<T, D>
      <<<dim3(k.H, k.n_seq), kGroups * D / 4, 0, st>>>(k, a.slots, a.unit, part, ml, first_of, static_cast<T *>(out), lse);
  return hipGetLastError();
}

template <typename T, int CODE>
hipError_t run_head(int D, const PagedAttnArgs &a, void *out, float *lse, void *ws, hipStream_t st) {
  switch (D) {
    case 64: return run_paged<T, CODE, 64>(a, out, lse, ws, st);
    case 96: return run_paged<T, CODE, 96>(a, out, lse, ws, st);
    case 128: return run_paged<T, CODE, 128>(a, out, lse, ws, st);
    case 192: return run_paged<T, CODE, 192>(a, out, lse, ws, st);
    default: return run_paged<T, CODE, 256>(a, out, lse, ws, st);
  }
}
template <typename T>
hipError_t run_code(int code, int D, const PagedAttnArgs &a, void *out, float *lse, void *ws, hipStream_t st) {
  return code == MOESPEC_CACHE_PLAIN ? run_head<T, MOESPEC_CACHE_PLAIN>(D, a, out, lse, ws, st)
         : code == MOESPEC_CACHE_I8  ? run_head<T, MOESPEC_CACHE_I8>(D, a, out, lse, ws, st)
                                     : run_head<T, MOESPEC_CACHE_E4M3>(D, a, out, lse, ws, st);
}

}  // namespace

// Room for the parts: no more workgroups than kMostGroups, and no more than units of 64 keys.  Neither bound grows where a call gets smaller.
size_t paged_attention_ws(const moespec_attn_desc &ds, const moespec_paged_cache &, int n_seq, int max_len) {
  const int64_t G = ds.n_heads / ds.n_kv_heads, units = (max_len + 63) / 64 * (int64_t)(n_seq < kMaxShared ? n_seq : kMaxShared);
  const int64_t most = kMostGroups / (ds.n_kv_heads * ((G + 15) / 16)), slots = units < most ? units : most;
  return kFirstBytes + (size_t)slots * ds.n_heads * (sizeof(float) * ds.head_dim + sizeof(float2));
}

hipError_t launch_paged_attention(const moespec_attn_desc &ds, const moespec_paged_cache &cache, int n_seq, const void *q,
                                  int64_t q_stride, const int32_t *cache_len, int max_len, void *out, float *lse, void *ws,
                                  hipStream_t st) {
  PagedAttnArgs a{};
  a.keys.q = q;
  a.keys.cache_len = cache_len;
  a.keys.q_stride = q_stride ? q_stride : (int64_t)ds.n_heads * ds.head_dim;
  a.keys.n_seq = n_seq;
  a.keys.M = n_seq;
  a.keys.max_tree = 1;
  a.keys.max_len = max_len;
  a.keys.H = ds.n_heads;
  a.keys.Hk = ds.n_kv_heads;
  a.keys.G = ds.n_heads / ds.n_kv_heads;
  a.keys.c = (float)((double)ds.scale * 1.4426950408889634);
  a.pages = pages_of(ds, cache);
  a.head_tiles = (a.keys.G + 15) / 16;
  a.unit = 0x1p-8f;
  for (int64_t n = 1; n < max_len; n *= 2) a.unit *= 0.5f;
  return ds.dtype == MOESPEC_BF16 ? run_code<uint16_t>(cache.code, ds.head_dim, a, out, lse, ws, st)
                                  : run_code<float>(cache.code, ds.head_dim, a, out, lse, ws, st);
}

}  // namespace moespec
