// The norm over a list of gradients and its clipping (see include/mgn.h).
//
// Squares are summed in 64 bits, where no float32 and no number of them overflows or
// vanishes; an element costs a conversion and a multiply-add there, which memory hides.
// The list comes as pieces of at most 16,384 elements; a block takes every
// gridDim.x-th.  Blocks' sums are added in a fixed order, by every block of the second
// launch for itself, so that there is no third.
//
// Bound by memory: a gradient is read twice (the second time from the caches if the list
// fits them) and written once.
#include "dev_common.hpp"
#include "row_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

constexpr int kClipBlocks = 2048;  // at most, and partial sums

// The sum over the lanes of a block, for all of them.
__device__ __forceinline__ double block_sum(double v, double* buf) {
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) v += __shfl_xor(v, k);
  const int w = threadIdx.x >> 6, n = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) buf[w] = v;
  __syncthreads();
  v = buf[0];
  for (int i = 1; i < n; ++i) v += buf[i];
  return v;
}

template <typename T>
__device__ __forceinline__ double squares(const mgn_piece& p) {
  const T* x = (const T*)p.in;
  double s[2] = {0.0, 0.0};
#pragma unroll 4
  for (int i = threadIdx.x * 8; i < p.n; i += 256 * 8) {
    const Raw8<T> v = load8(x + i, p.n - i);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double d = (double)v.get(e);
      s[e & 1] = __builtin_fma(d, d, s[e & 1]);
    }
  }
  return s[0] + s[1];
}

__global__ void __launch_bounds__(256) k_grad_squares(GradClip a) {
  __shared__ double buf[4];
  double s = 0.0;
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const mgn_piece p = a.pieces[i];
    s += (p.types & 1) ? squares<bf16>(p) : squares<float>(p);
  }
  s = block_sum(s, buf);
  if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}

template <typename TI, typename TO>
__device__ __forceinline__ void scaled(const mgn_piece& p, double k) {
  const TI* x = (const TI*)p.in;
  TO* y = (TO*)p.out;
#pragma unroll 4
  for (int i = threadIdx.x * 8; i < p.n; i += 256 * 8) {
    const Raw8<TI> v = load8(x + i, p.n - i);
    float f[8];
    // in 64 bits: the factor may be smaller than float32 numbers are
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)((double)v.get(e) * k);
    store8(y + i, 0, min(p.n - i, 8), f);
  }
}

__global__ void __launch_bounds__(256) k_grad_clip(GradClip a, int parts) {
  __shared__ double buf[4];
  double norm;
  if (a.given) {
    norm = (double)*a.norm;
  } else {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += a.part[i];
    norm = __builtin_sqrt(block_sum(s, buf));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  }
  if (!a.clip) return;
  const double k = norm > a.max_norm && norm < __builtin_inf() ? a.max_norm / norm : 1.0;
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const mgn_piece p = a.pieces[i];
    if (k == 1.0 && p.in == p.out) continue;  // nothing changes
    switch (p.types & 3) {
      case 0: scaled<float, float>(p, k); break;
      case 1: scaled<bf16, float>(p, k); break;
      case 2: scaled<float, bf16>(p, k); break;
      default: scaled<bf16, bf16>(p, k); break;
    }
  }
}

}  // namespace dev

using namespace dev;

size_t grad_norm_workspace(int64_t n) { return n > 0 ? (size_t)std::min<int64_t>(n, kClipBlocks) * 8 : 0; }

hipError_t launch_grad_clip(const GradClip& a, hipStream_t s) {
  const int blocks = (int)std::min<int64_t>(a.n, kClipBlocks);
  if (!a.given && blocks > 0) {
    hipLaunchKernelGGL(k_grad_squares, dim3(blocks), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_grad_clip, dim3(a.clip ? std::max(blocks, 1) : 1), dim3(256), 0, s, a, blocks);
  return hipGetLastError();
}

}  // namespace mgn
