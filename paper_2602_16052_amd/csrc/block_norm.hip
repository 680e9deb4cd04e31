// Between two blocks: the norm of a block's output, its gate and scale, the residual stream and the norm of the next input in one
// pass.  Bound by memory traffic: y, residual and an element gate are read once, r and x written once.  A workgroup holds a
// row in registers, so that nothing is read again for the second norm.  2044 rows of 4096, bf16, gate for every element: 13.4 us, 6.3
// TB/s (the 84 MB stay in the last-level cache between calls); one row of 2048: 2.5 us, the launch and its two reductions.
#include <math.h>

#include "attention.h"

namespace moespec {

constexpr int kNormThreads = 256;

// Sum over the workgroup, the same bits in every thread.  part: one float per wave.
__device__ __forceinline__ float group_sum(float v, float *part) {
  v = row16_sum(v);
  v += __shfl_xor(v, 16, kWave);
  v += __shfl_xor(v, 32, kWave);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  float a = part[0];
#pragma unroll
  for (int i = 1; i < kNormThreads / kWave; ++i) a += part[i];
  return a;
}

template <typename T, int NC>
__global__ __launch_bounds__(kNormThreads) void block_norm_kernel(moespec_block b, const T *y, const T *residual, int d, T *r,
                                                                  T *x) {
  constexpr int E = Piece<T>::kElems;
  __shared__ float part[2][kNormThreads / kWave];
  const size_t at = (size_t)blockIdx.x * d;
  const T *gate = static_cast<const T *>(b.gate), *w_post = static_cast<const T *>(b.w_post);
  const T *w_pre = static_cast<const T *>(b.w_pre);
  const float eps = b.eps;
  float z[NC][E], res[NC][E], ss = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int j = (c * kNormThreads + (int)threadIdx.x) * E;
#pragma unroll
    for (int e = 0; e < E; ++e) z[c][e] = res[c][e] = 0.f;
    if (j < d) {
      Piece<T>::load(y + at + j, z[c]);
      if (residual) Piece<T>::load(residual + at + j, res[c]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(z[c][e], z[c][e], ss);
  }
  auto gated = [&](float v) { return b.gate_sigmoid ? 1.f / (1.f + __expf(-v)) : v; };
  float f = b.scale;
  if (b.post_norm) f *= 1.f / sqrtf(group_sum(ss, part[0]) / (float)d + eps);
  if (b.gate_kind == MOESPEC_BLOCK_GATE_TOKEN) f *= gated(Elem<T>::load(gate + blockIdx.x));
  ss = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int j = (c * kNormThreads + (int)threadIdx.x) * E;
    if (j < d) {
      if (b.post_norm && w_post) {
        float w[E];
        Piece<T>::load(w_post + j, w);
#pragma unroll
        for (int e = 0; e < E; ++e) z[c][e] *= w[e];
      }
      if (b.gate_kind == MOESPEC_BLOCK_GATE_CHANNEL || b.gate_kind == MOESPEC_BLOCK_GATE_ELEMENT) {
        float w[E];
        Piece<T>::load(gate + (b.gate_kind == MOESPEC_BLOCK_GATE_ELEMENT ? at : 0) + j, w);
#pragma unroll
        for (int e = 0; e < E; ++e) z[c][e] *= gated(w[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      z[c][e] = fmaf(f, z[c][e], res[c][e]);
      if (j < d) ss = fmaf(z[c][e], z[c][e], ss);
    }
    if (r && j < d) Piece<T>::store(r + at + j, z[c]);
  }
  if (!x) return;
  const float n = 1.f / sqrtf(group_sum(ss, part[1]) / (float)d + eps);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int j = (c * kNormThreads + (int)threadIdx.x) * E;
    if (j >= d) continue;
    float w[E];
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = 1.f;
    if (w_pre) Piece<T>::load(w_pre + j, w);
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] *= n * z[c][e];
    Piece<T>::store(x + at + j, w);
  }
}

hipError_t launch_block_norm(const moespec_desc &ds, const moespec_block &b, const void *y, const void *residual, int M,
                             void *r, void *x, hipStream_t st) {
  auto run = [&](auto kern, auto *type) -> hipError_t {
    typedef decltype(type) P;
    kern<<<M, kNormThreads, 0, st>>>(b, static_cast<const std::remove_pointer_t<P> *>(y),
                                     static_cast<const std::remove_pointer_t<P> *>(residual), ds.d, static_cast<P>(r),
                                     static_cast<P>(x));
    return hipGetLastError();
  };
  if (ds.dtype == MOESPEC_BF16) {
    uint16_t *t = nullptr;
    const int n = (ds.d + 8 * kNormThreads - 1) / (8 * kNormThreads);  // d <= 8192
    return n <= 1 ? run(block_norm_kernel<uint16_t, 1>, t) : n <= 2 ? run(block_norm_kernel<uint16_t, 2>, t)
                                                                    : run(block_norm_kernel<uint16_t, 4>, t);
  }
  float *t = nullptr;
  const int n = (ds.d + 4 * kNormThreads - 1) / (4 * kNormThreads);
  return n <= 1 ? run(block_norm_kernel<float, 1>, t) : n <= 2 ? run(block_norm_kernel<float, 2>, t)
         : n <= 4 ? run(block_norm_kernel<float, 4>, t) : run(block_norm_kernel<float, 8>, t);
}

}  // namespace moespec
