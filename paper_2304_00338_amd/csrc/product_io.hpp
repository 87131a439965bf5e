// What the products of scaled low-precision matrices (matmul8.hip, matmul4.hip) do
// with their sums: the epilogue, four consecutive columns at a time, and the join of
// sums that several blocks share.  A job is a struct with the call p (a, b, ep, c_type,
// c, ldc, part) and the number of splits.
#pragma once

#include "dev_common.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// What a load takes for what lies beyond a matrix's columns.
static __device__ const uint4 zero16 = {0, 0, 0, 0};

__device__ __forceinline__ f32x4 load4(const float* p, int n) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (n >= 4) {
    __builtin_memcpy(&v, p, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) v[e] = p[e];
  }
  return v;
}
__device__ __forceinline__ f32x4 load4(const bf16* p, int n) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (n >= 4) {
    uint32_t w[2];
    __builtin_memcpy(w, p, 8);
    v = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16),
              __uint_as_float(w[1] & 0xffff0000u)};
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) v[e] = tof(p[e]);
  }
  return v;
}
template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v, int n) {
  if (n >= 4) {
    const T w[4] = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    __builtin_memcpy(p, w, sizeof(w));
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = (T)v[e];
  }
}

// Four sums of row m, columns n .. n + 3 (those inside c), become c.
template <typename P>
__device__ __forceinline__ void finish(const P& p, int64_t m, int64_t n, f32x4 v) {
  const int k = (int)min(p.b.rows - n, (int64_t)4);
  if (p.ep.bias != nullptr) v += load4(p.ep.bias + n, k);
  if (p.ep.act == MGN_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];  // a NaN stays
  } else if (p.ep.act == MGN_ACT_RELU_GRAD) {
    const int64_t i = m * p.ep.ldaux + n;
    const f32x4 h = p.ep.aux_type == MGN_FP32 ? load4((const float*)p.ep.aux + i, k) : load4((const bf16*)p.ep.aux + i, k);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = h[e] > 0.f ? v[e] : 0.f;
  }
  const int64_t i = m * p.ldc + n;
  if (p.c_type == MGN_FP32) {
    float* c = (float*)p.c + i;
    if (p.ep.accumulate) v += load4(c, k);
    store4(c, v, k);
  } else {
    bf16* c = (bf16*)p.c + i;
    if (p.ep.accumulate) v += load4(c, k);
    store4(c, v, k);
  }
}

// Four sums of a split, or of the whole.
template <typename J_>
__device__ __forceinline__ void put4(const J_& J, int split, int64_t m, int64_t n, f32x4 v) {
  if (J.splits == 1)
    finish(J.p, m, n, v);
  else
    store4(J.p.part + ((int64_t)split * J.p.a.rows + m) * J.p.b.rows + n, v, (int)min(J.p.b.rows - n, (int64_t)4));
}

// Sums of the splits, 4 columns a thread: G threads for each, thread g the splits
// g, g + G, ..., then the G sums in order.
template <int G, typename J_>
__global__ void __launch_bounds__(256) k_product_join(J_ J) {
  __shared__ f32x4 sums[G][256 / G];
  const int g = threadIdx.x / (256 / G), q = threadIdx.x % (256 / G);
  const int64_t M = J.p.a.rows, N = J.p.b.rows, n4 = ceil_div(N, 4), t = (int64_t)blockIdx.x * (256 / G) + q;
  const bool in = t < M * n4;
  const int64_t m = in ? t / n4 : 0, n = in ? t % n4 * 4 : 0;
  const int k = (int)min(N - n, (int64_t)4);
  const float* p = J.p.part + m * N + n;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = g; s < J.splits; s += G) v += load4(p + (int64_t)s * M * N, k);
  if constexpr (G > 1) {
    sums[g][q] = v;
    __syncthreads();
    if (g > 0) return;
#pragma unroll
    for (int i = 1; i < G; ++i) v += sums[i][q];
  }
  if (in) finish(J.p, m, n, v);
}

}  // namespace dev
}  // namespace mgn
