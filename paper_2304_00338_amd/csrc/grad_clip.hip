// The norm over a list of gradients and its clipping (see include/mgn.h).
//
// Squares are summed in 64 bits, where no float32 and no number of them overflows or
// vanishes; an element costs a conversion and a multiply-add there, which memory hides.
// The list comes as pieces of at most 16,384 elements; a thread takes four neighbouring
// ones at a time, so that a wave's loads and stores are of whole lines.  A block takes
// every gridDim.x-th piece.  Blocks' sums are added in a fixed order, by every block of
// the second launch for itself, so that there is no third; that launch goes through the
// pieces from the last one on, whose gradients the last-level cache still holds.  Up to
// two pieces are one block's, in one launch, with the gradients kept in registers.
//
// Bound by memory: a gradient is read twice and written once.  Measured: 300 M bf16 to fp32
// squares 121 us (5.0 TB/s), clipping 405 (4.4).
#include "dev_common.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kClipBlocks = 2048;  // at most, and partial sums
constexpr int kClipSmall = 2;      // pieces that one block takes
constexpr int kBatch = 8;          // times four elements that a thread loads at once

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

__device__ __forceinline__ f32x4 load_four(const float* p) { return *(const f32x4u*)p; }
__device__ __forceinline__ f32x4 load_four(const bf16* p) {
  const u16x4 v = *(const u16x4*)p;
  return f32x4{__uint_as_float((uint32_t)v[0] << 16), __uint_as_float((uint32_t)v[1] << 16),
               __uint_as_float((uint32_t)v[2] << 16), __uint_as_float((uint32_t)v[3] << 16)};
}
// Elements i .. i + 3 of a piece; 0 behind its end.
template <typename T>
__device__ __forceinline__ f32x4 four_of(const mgn_piece& p, int i) {
  const T* x = (const T*)p.in;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (i + 4 <= p.n) {
    v = load_four(x + i);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (i + e < p.n) v[e] = tof(x[i + e]);
  }
  return v;
}
__device__ __forceinline__ f32x4 four_of(const mgn_piece& p, int i) {
  return (p.types & 1) ? four_of<bf16>(p, i) : four_of<float>(p, i);
}
// v times k becomes elements i .. i + 3 of the piece's place.  The product is of 64 bits: the
// factor may be smaller than float32 numbers are.  Whole runs go out past the caches.
__device__ __forceinline__ void put_four(const mgn_piece& p, int i, f32x4 v, double k) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)((double)v[e] * k);
  if (p.types & 2) {
    bf16* y = (bf16*)p.out + i;
    const bf16 w[4] = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    if (i + 4 <= p.n) {
      __builtin_nontemporal_store(__builtin_bit_cast(u16x4, w), (u16x4*)y);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (i + e < p.n) y[e] = w[e];
    }
  } else {
    float* y = (float*)p.out + i;
    if (i + 4 <= p.n) {
      __builtin_nontemporal_store((f32x4u)v, (f32x4u*)y);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (i + e < p.n) y[e] = v[e];
    }
  }
}
__device__ __forceinline__ void add_squares(double (&s)[2], f32x4 v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double d = (double)v[e];
    s[e & 1] = __builtin_fma(d, d, s[e & 1]);
  }
}
__device__ __forceinline__ double factor(double norm, double most) {
  return norm > most && norm < __builtin_inf() ? most / norm : 1.0;
}

template <typename T>
__device__ __forceinline__ void squares(double (&s)[2], const mgn_piece& p) {
  for (int i = threadIdx.x * 4; i < p.n; i += 1024 * kBatch) {
    f32x4 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = four_of<T>(p, i + 1024 * u);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) add_squares(s, v[u]);
  }
}

__global__ void __launch_bounds__(256) k_grad_squares(GradClip a) {
  __shared__ double buf[4];
  double s[2] = {0.0, 0.0};
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const mgn_piece p = a.pieces[i];
    if (p.types & 1)
      squares<bf16>(s, p);
    else
      squares<float>(s, p);
  }
  const double t = block_sum(s[0] + s[1], buf);
  if (threadIdx.x == 0) a.part[blockIdx.x] = t;
}

__global__ void __launch_bounds__(256) k_grad_clip(GradClip a, int parts) {
  __shared__ double buf[4];
  const int t = threadIdx.x * 4;
  // the first elements are on their way while the sums are added
  mgn_piece p = {};
  f32x4 v[kBatch] = {};
  const int64_t first = a.n - 1 - (int64_t)blockIdx.x;
  if (a.clip && first >= 0) {
    p = a.pieces[first];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = four_of(p, t + 1024 * u);
  }
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
  const double k = factor(norm, a.max_norm);
  for (int64_t i = first; i >= 0;) {
    if (p.out != nullptr && (k != 1.0 || p.in != p.out)) {  // else nothing changes
      for (int at = t; at < p.n; at += 1024 * kBatch) {
        if (at != t) {
#pragma unroll
          for (int u = 0; u < kBatch; ++u) v[u] = four_of(p, at + 1024 * u);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (at + 1024 * u < p.n) put_four(p, at + 1024 * u, v[u], k);
      }
    }
    i -= gridDim.x;
    if (i < 0) break;
    p = a.pieces[i];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = four_of(p, t + 1024 * u);
  }
}

// The whole of a short list, kept in registers: fours one after the other through the
// pieces, a thread every 1024th.
__global__ void __launch_bounds__(1024) k_grad_clip_small(GradClip a) {
  constexpr int H = kClipSmall * kPiece / 4096;
  __shared__ double buf[16];
  mgn_piece p[kClipSmall] = {};
#pragma unroll
  for (int q = 0; q < kClipSmall; ++q)
    if (q < a.n) p[q] = a.pieces[q];
  const int t = threadIdx.x, end = (p[0].n + 3) / 4;  // the second piece's first four
  f32x4 v[H];
#pragma unroll
  for (int k = 0; k < H; ++k) {
    const int u = k * 1024 + t;
    v[k] = u < end ? four_of(p[0], u * 4) : four_of(p[1], (u - end) * 4);
  }
  double norm;
  if (a.given) {
    norm = (double)*a.norm;
  } else {
    double s[2] = {0.0, 0.0};
#pragma unroll
    for (int k = 0; k < H; ++k) add_squares(s, v[k]);
    norm = __builtin_sqrt(block_sum(s[0] + s[1], buf));
    if (t == 0) *a.norm = (float)norm;
  }
  if (!a.clip) return;
  const double f = factor(norm, a.max_norm);
#pragma unroll
  for (int k = 0; k < H; ++k) {
    const int u = k * 1024 + t, q = u >= end, at = (u - (q ? end : 0)) * 4;
    const mgn_piece& o = p[q];
    if (at < o.n && o.out != nullptr && (f != 1.0 || o.in != o.out)) put_four(o, at, v[k], f);
  }
}

}  // namespace dev

using namespace dev;

namespace {
// As many blocks as take the same number of pieces each.
int clip_blocks(int64_t n) {
  if (n <= 0) return 0;
  return (int)ceil_div(n, ceil_div(n, (int64_t)kClipBlocks));
}
}  // namespace

size_t grad_norm_workspace(int64_t n) { return (size_t)clip_blocks(n) * 8; }

hipError_t launch_grad_clip(const GradClip& a, hipStream_t s) {
  if (a.n <= kClipSmall) {
    hipLaunchKernelGGL(k_grad_clip_small, dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  const int blocks = clip_blocks(a.n);
  if (!a.given) {
    hipLaunchKernelGGL(k_grad_squares, dim3(blocks), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_grad_clip, dim3(a.clip ? blocks : 1), dim3(256), 0, s, a, blocks);
  return hipGetLastError();
}

}  // namespace mgn
