// A cache in pages: rows of keys and values written as they are or in 8 bits, and read back.  Bound by traffic; few rows, by the launch.
// A row belongs to a group of lanes that hold 16 bytes of it each (of keys and of values), so that its largest magnitude is found
// without LDS.  The groups of a workgroup take neighbouring entries of one head, whose rows and scales are neighbours in a page.
// 4 prompts of 8190 rows x 8 heads of 128, bf16 to e4m3: written 40.8 us (4.9 TB/s, a large copy's rate), read back 25.8 (7.8 TB/s: out of the
// last-level cache); 48 layers x 8 sequences x up to 8 rows in int8: 5 us each, the launch and two or three trips to memory.
#include "serving.h"

namespace moespec {

namespace {

struct PagedArgs {
  Pages pages;
  const void *k_tree, *v_tree;  // write: sources
  void *k, *v;                  // read: destinations
  const int32_t *path, *n_path, *cache_len, *first, *tree_off;
  int32_t *new_len;
  int64_t kv_stride, capacity;
  int n_layers, n_seq, M, max_tree, max_path, max_len;
};

// 16 bytes of a row as four words; a bf16 word holds two elements.
template <typename T>
__device__ __forceinline__ float elem_of(const uint4 &b, int e) {
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
  if (sizeof(T) == 4) return __uint_as_float(w[e]);
  return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
}

struct RowCode {
  float scale, inv;
};
// Scale of a row by the bits of its largest magnitude (as integers they are in the order of the values, infinities and NaN behind).
template <int CODE>
__device__ __forceinline__ RowCode row_code(uint32_t amax) {
  if (amax >= 0x7f800000u) return RowCode{__uint_as_float(0x7fc00000u), 0.f};
  if (CODE == MOESPEC_CACHE_I8) {
    const float m = __uint_as_float(amax);
    return RowCode{m / 127.f, fminf(127.f / m, FLT_MAX)};  // (a row of zeros: codes 0)
  }
  // 448 = 1.75 * 2^8: the power of two 8 below, or 7 where the mantissa is beyond 1.75
  const int e = max((int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
  return RowCode{__uint_as_float((uint32_t)(e + 127) << 23), __uint_as_float((uint32_t)(127 - e) << 23)};
}

// Four elements' codes in a word.  I8: the sum with 1.5 * 2^23 rounds the unrounded product to an integer, ties to even, which is then
// its last byte.  E4M3: the product with a power of two is exact, the conversion rounds to the nearest.
template <int CODE>
__device__ __forceinline__ uint32_t codes4(const float (&x)[4], const RowCode &c, bool odd) {
  if (odd) return 0;
  if (CODE == MOESPEC_CACHE_I8) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= (__float_as_uint(fmaf(x[e], c.inv, 12582912.f)) & 0xffu) << (8 * e);
    return w;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * c.inv, x[1] * c.inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * c.inv, x[3] * c.inv, w, true);
}

template <int CODE>
__device__ __forceinline__ float value_of(uint32_t codes, int e) {
  if (CODE == MOESPEC_CACHE_I8) return (float)(int8_t)(codes >> (8 * e));
  switch (e) {
    case 0: return __builtin_amdgcn_cvt_f32_fp8(codes, 0);
    case 1: return __builtin_amdgcn_cvt_f32_fp8(codes, 1);
    case 2: return __builtin_amdgcn_cvt_f32_fp8(codes, 2);
    default: return __builtin_amdgcn_cvt_f32_fp8(codes, 3);
  }
}

template <typename T, int D>
struct RowShape {
  static constexpr int E = 16 / (int)sizeof(T), kPieces = D / E, W = pow2_ceil(kPieces), kRows = 256 / W;
};

template <typename T, int CODE, int D>
__global__ __launch_bounds__(256) void paged_write_kernel(PagedArgs a) {
  typedef RowShape<T, D> R;
  const Pages &pg = a.pages;
  const int hk = blockIdx.x % pg.Hk, s = blockIdx.y, layer = blockIdx.z, p = threadIdx.x % R::W;
  const int i = (int)(blockIdx.x / pg.Hk) * R::kRows + (int)threadIdx.x / R::W;
  // two trips to memory: what says where the row comes from and goes to, then the row beside its page
  const int t = a.path ? a.path[(int64_t)s * a.max_path + min(i, a.max_path - 1)] : i;
  const SeqRows g = seq_rows(a.tree_off, s, a.M, a.max_tree);
  const int n = a.n_path ? min(max(a.n_path[s], 0), a.max_path) : g.T;
  const int64_t len = min((int64_t)max(a.cache_len[s], 0), pg.entries());
  if (a.new_len && blockIdx.x == 0 && layer == 0 && threadIdx.x == 0) a.new_len[s] = (int)min(len + n, pg.entries());
  const int64_t e = len + i;
  if (i >= n || e >= pg.entries()) return;
  uint4 kv[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  if (t >= 0 && t < g.T && p < R::kPieces) {
    const int64_t src = ((int64_t)layer * a.M + g.row0 + t) * a.kv_stride + hk * D + p * R::E;
    kv[0] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.k_tree) + src);
    kv[1] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.v_tree) + src);
  }
  const int page = pg.page_of(s, e);
  if (page < 0) return;
  const int64_t row = pg.row(layer, page, hk, e);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    unsigned char *to = const_cast<unsigned char *>(x == 0 ? pg.k : pg.v);
    if constexpr (CODE == MOESPEC_CACHE_PLAIN) {
      if (p < R::kPieces) reinterpret_cast<uint4 *>(to)[row * R::kPieces + p] = kv[x];
    } else {
      float v[R::E];
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < R::E; ++i) {
        v[i] = elem_of<T>(kv[x], i);
        amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
      }
#pragma unroll
      for (int m = 1; m < R::W; m <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, m, kWave));
      const RowCode c = row_code<CODE>(amax);
      const bool odd = amax >= 0x7f800000u;
      if (p < R::kPieces) {
        uint32_t w[R::E / 4];
#pragma unroll
        for (int i = 0; i < R::E / 4; ++i) {
          const float four[4] = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
          w[i] = codes4<CODE>(four, c, odd);
        }
        unsigned char *at = to + row * D + p * R::E;
        if constexpr (R::E == 8) *reinterpret_cast<uint2 *>(at) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(at) = w[0];
      }
      if (p == 0) const_cast<float *>(x == 0 ? pg.k_scale : pg.v_scale)[row] = c.scale;
    }
  }
}

constexpr int kReadGroups = 4096;

template <typename T, int CODE, int D>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedArgs a, int blocks) {
  typedef RowShape<T, D> R;
  const Pages &pg = a.pages;
  const int hk = blockIdx.x % pg.Hk, s = blockIdx.y, layer = blockIdx.z, p = threadIdx.x % R::W;
  const int len = min(max(a.cache_len[s], 0), a.max_len), from = a.first ? max(a.first[s], 0) : 0;
  if (p >= R::kPieces) return;
  for (int64_t e = (int64_t)from + (int64_t)(blockIdx.x / pg.Hk) * R::kRows + threadIdx.x / R::W; e < len;
       e += (int64_t)blocks * R::kRows) {
    const int page = pg.page_of(s, e);
    const int64_t row = pg.row(layer, max(page, 0), hk, e);
    const int64_t dst = ((((int64_t)layer * a.n_seq + s) * pg.Hk + hk) * a.capacity + e) * R::kPieces + p;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const unsigned char *src = x == 0 ? pg.k : pg.v;
      uint4 *to = static_cast<uint4 *>(x == 0 ? a.k : a.v) + dst;
      if constexpr (CODE == MOESPEC_CACHE_PLAIN) {
        *to = page < 0 ? make_uint4(0, 0, 0, 0) : reinterpret_cast<const uint4 *>(src)[row * R::kPieces + p];
      } else {
        const unsigned char *at = src + row * D + p * R::E;
        uint32_t w[2] = {0, 0};
        if constexpr (R::E == 8) {
          const uint2 two = *reinterpret_cast<const uint2 *>(at);
          w[0] = two.x;
          w[1] = two.y;
        } else {
          w[0] = *reinterpret_cast<const uint32_t *>(at);
        }
        const float scale = (x == 0 ? pg.k_scale : pg.v_scale)[row];
        float v[R::E];
#pragma unroll
        for (int i = 0; i < R::E; ++i) v[i] = page < 0 ? 0.f : value_of<CODE>(w[i / 4], i % 4) * scale;
        Elem<T>::store4(reinterpret_cast<T *>(to), f32x4{v[0], v[1], v[2], v[3]});
        if constexpr (R::E == 8) Elem<T>::store4(reinterpret_cast<T *>(to) + 4, f32x4{v[4], v[5], v[6], v[7]});
      }
    }
  }
}

// run(type, code, head size) with what the descriptor and the cache say, as constants.
template <typename T, int CODE, typename Run>
hipError_t by_head(int D, Run run) {
  switch (D) {
    case 64: return run(T{}, std::integral_constant<int, CODE>{}, std::integral_constant<int, 64>{});
    case 96: return run(T{}, std::integral_constant<int, CODE>{}, std::integral_constant<int, 96>{});
    case 128: return run(T{}, std::integral_constant<int, CODE>{}, std::integral_constant<int, 128>{});
    case 192: return run(T{}, std::integral_constant<int, CODE>{}, std::integral_constant<int, 192>{});
    default: return run(T{}, std::integral_constant<int, CODE>{}, std::integral_constant<int, 256>{});
  }
}
template <typename T, typename Run>
hipError_t by_code(int code, int D, Run run) {
  return code == MOESPEC_CACHE_PLAIN ? by_head<T, MOESPEC_CACHE_PLAIN>(D, run)
         : code == MOESPEC_CACHE_I8  ? by_head<T, MOESPEC_CACHE_I8>(D, run)
                                     : by_head<T, MOESPEC_CACHE_E4M3>(D, run);
}
template <typename Run>
hipError_t by_kind(const moespec_attn_desc &ds, int code, Run run) {
  return ds.dtype == MOESPEC_BF16 ? by_code<uint16_t>(code, ds.head_dim, run) : by_code<float>(code, ds.head_dim, run);
}

}  // namespace

hipError_t launch_paged_write(const moespec_attn_desc &ds, int n_layers, const moespec_paged_cache &cache, const moespec_tree &tree,
                              const void *k_tree, const void *v_tree, const int32_t *path, const int32_t *n_path, int max_path,
                              const int32_t *cache_len, int32_t *new_len, hipStream_t st) {
  PagedArgs a{};
  a.pages = pages_of(ds, cache);
  a.k_tree = k_tree;
  a.v_tree = v_tree;
  a.path = path;
  a.n_path = n_path;
  a.cache_len = cache_len;
  a.tree_off = tree.tree_off;
  a.new_len = new_len;
  a.kv_stride = tree.kv_stride ? tree.kv_stride : (int64_t)ds.n_kv_heads * ds.head_dim;
  a.n_layers = n_layers;
  a.n_seq = tree.n_seq;
  a.M = tree.n_tokens;
  a.max_tree = tree.max_tree;
  a.max_path = path ? max_path : tree.max_tree;
  return by_kind(ds, cache.code, [&](auto type, auto code, auto dim) {
    typedef RowShape<decltype(type), decltype(dim)::value> R;
    const dim3 grid((unsigned)((a.max_path + R::kRows - 1) / R::kRows * ds.n_kv_heads), a.n_seq, n_layers);
    paged_write_kernel<decltype(type), decltype(code)::value, decltype(dim)::value><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_paged_read(const moespec_attn_desc &ds, int n_layers, int n_seq, const moespec_paged_cache &cache,
                             const int32_t *first, const int32_t *cache_len, int max_len, void *k_cache, void *v_cache,
                             hipStream_t st) {
  if (max_len == 0) return hipSuccess;
  PagedArgs a{};
  a.pages = pages_of(ds, cache);
  a.k = k_cache;
  a.v = v_cache;
  a.first = first;
  a.cache_len = cache_len;
  a.capacity = ds.capacity;
  a.n_layers = n_layers;
  a.n_seq = n_seq;
  a.max_len = max_len;
  return by_kind(ds, cache.code, [&](auto type, auto code, auto dim) {
    typedef RowShape<decltype(type), decltype(dim)::value> R;
    // as many workgroups a head as there may be rows for, and no more than fill the card: new entries of long caches are few, and a
    // workgroup without any costs as much as one with some (8 sequences of 48 layers, up to 8 entries of 127, write and read: 10.0 us, 14.6 with a workgroup for every 16 entries)
    const int64_t heads = (int64_t)ds.n_kv_heads * n_seq * n_layers, most = std::max<int64_t>(kReadGroups / heads, 1);
    const int blocks = (int)std::min<int64_t>((max_len + R::kRows - 1) / R::kRows, most);
    const dim3 grid((unsigned)(blocks * ds.n_kv_heads), n_seq, n_layers);
    paged_read_kernel<decltype(type), decltype(code)::value, decltype(dim)::value><<<grid, 256, 0, st>>>(a, blocks);
    return hipGetLastError();
  });
}

}  // namespace moespec
