// 4-bit quantisation with one power of two for each 32 columns of a row, and the
// way back (see include/mgn.h).
//
// With u the bits of the largest magnitude, X = 2^(b - 127), b = max(0, ((u + 2^21) >>
// 23) - 2): the exponent of u less 2, one more where its mantissa is 1.75 or more. x / X
// is exact, and the conversion instruction, which takes X as a float's exponent, rounds
// it to the nearest number, ties to even (checked for every bf16 below 7 X and for the
// float neighbours of the middles, at X from 2^-127 to 2^126).
//
// Bound by memory: an element is read once (2 or 4 bytes) and written as half a
// byte a copy.  k_quant4_rows (rows only) gives 16 lanes to 128 columns, four to a
// block; k_quant4_tile takes 128 x 128, a thread 8 rows x 8 columns, so that a wave
// has the 32 rows of a column's block and the column maxima stay in it; the
// transpose and the scales go through LDS to be stored in whole pieces.
// Measured: 852,640 x 256 fp32 to both copies 239 us (4.6 TB/s of reads and writes), 852,640
// x 128 fp32 to rows 88 (5.6) and with sums 127 and 9 for these, 5120 x 4999 bf16 to both 26
// (3.1; rows of odd alignment), 852,640 x 256 back to fp32 139 (7.1).
#include "dev_common.hpp"
#include "row_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

// The kernels that go through rows take them in units of some rows x 128 columns, one row of
// units after the other, kUnits of them a block.
constexpr int kUnits = 4;

// Magnitudes as bits: their order is that of the values, a NaN is the largest.
__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7fffffffu; }
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, false);
}
// The largest of the four lanes 4 i .. 4 i + 3.
__device__ __forceinline__ uint32_t max_quad(uint32_t v) {
  v = max(v, dpp_u<0xb1>(v));  // lanes 1 0 3 2
  return max(v, dpp_u<0x4e>(v));  // lanes 2 3 0 1
}
// The largest of the lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ uint32_t max_rows(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const uint32_t u = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return max(b[0], b[1]);
}

// The scale's byte for a largest magnitude.
__device__ __forceinline__ uint32_t scale4(uint32_t u) {
  return u >= 0x7f800000u ? 255u : (uint32_t)max((int)((u + 0x200000u) >> 23) - 2, 0);
}
// 2^(b - 127) as a float.
__device__ __forceinline__ float power(uint32_t b) { return __uint_as_float(max(b << 23, 0x400000u)); }

// Eight numbers, the first in the lowest half byte.
__device__ __forceinline__ uint32_t numbers4(const float (&v)[8], uint32_t b) {
  const float s = power(b);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
  return b == 255u ? 0u : w;
}

template <typename XT>
__global__ void __launch_bounds__(256) k_quant4_rows(Quant4 a) {
  const int l = threadIdx.x & 15;
  const int64_t end = (a.cols + 31) & ~31LL;
  const uint32_t cbs = (uint32_t)ceil_div(a.cols, 128);
  const int64_t u0 = (blockIdx.y * (int64_t)kGridRow + blockIdx.x) * kUnits;
  // unit k: a row of 16, the first column of 128
  auto place = [&](int k, int64_t& r, int64_t& cb) {
    const int64_t g = (u0 + k) / cbs;
    cb = u0 + k - g * cbs;
    r = g * 16 + (threadIdx.x >> 4);
  };
  Raw8<XT> raw[kUnits];
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    int64_t r, cb;
    place(k, r, cb);
    const int64_t c = cb * 128 + l * 8;
    raw[k] = load8((const XT*)a.x + r * a.ldx + c, r < a.rows ? (int)min(a.cols - c, (int64_t)8) : 0);
  }
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    int64_t r, cb;
    place(k, r, cb);
    const int64_t c = cb * 128 + l * 8;
    if (r >= a.rows) break;  // all 16 lanes of the row
    float v[8];
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = raw[k].get(e);
      m = max(m, magnitude(v[e]));
    }
    const uint32_t b = scale4(max_quad(m));
    if (c < end) *(uint32_t*)(a.q + r * a.ldq + c / 2) = numbers4(v, b);
    // the four bytes meet in lane 0
    uint32_t w = b << (8 * (l >> 2));
    w |= dpp_u<0x128>(w);
    w |= dpp_u<0x124>(w);
    if (l == 0) ((uint32_t*)a.scale)[cb * a.rows + r] = w;
  }
}

// Eight elements past the caches.
template <typename XT>
__device__ __forceinline__ Raw8<XT> load8_once(const XT* p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
  u32x4 w[sizeof(Raw8<XT>) / 16];
#pragma unroll
  for (int i = 0; i < (int)(sizeof(Raw8<XT>) / 16); ++i) w[i] = __builtin_nontemporal_load((const u32x4*)p + i);
  Raw8<XT> r;
  __builtin_memcpy(&r, w, sizeof(r));
  return r;
}

// LARGE: x is larger than the caches.
template <typename XT, bool SUMS, bool LARGE>
__global__ void __launch_bounds__(256) k_quant4_tile(Quant4 a) {
  constexpr int CLD = 68;  // bytes of a column in LDS
  __shared__ __align__(16) uint8_t turned[128 * CLD];
  __shared__ __align__(16) uint8_t cscale[128][4];
  __shared__ uint32_t rscale[128];
  __shared__ float csum[SUMS ? 4 : 1][128];
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, w = threadIdx.x >> 6;
  const int64_t cbs = ceil_div(a.cols, 128), rbs = ceil_div(a.rows, 128);
  const uint32_t block = blockIdx.y * (uint32_t)kGridRow + blockIdx.x;
  const int64_t rb = block / (uint32_t)cbs, cb = block - rb * cbs;
  if (rb >= rbs) return;  // behind the last block
  const int64_t up_cols = (a.cols + 31) & ~31LL, up_rows = (a.rows + 31) & ~31LL;
  const int64_t c0 = cb * 128 + l * 8;
  const int n = (int)min(max(a.cols - c0, (int64_t)0), (int64_t)8);
  const bool turn = a.qt != nullptr;
  float cs[8] = {};
  const int64_t r0 = rb * 128 + g * 8;
  Raw8<XT> raw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = min(r0 + i, a.rows - 1);
    const XT* x = (const XT*)a.x + r * a.ldx + c0;
    const int k = r0 + i < a.rows ? n : 0;
    raw[i] = LARGE && k >= 8 ? load8_once(x) : load8(x, k);
  }
  uint32_t cm[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = raw[i].get(e);
      const uint32_t u = magnitude(v[e]);
      m = max(m, u);
      cm[e] = max(cm[e], u);
      if (SUMS) cs[e] += v[e];
    }
    if (a.q != nullptr) {
      const uint32_t b = scale4(max_quad(m));
      if (r0 + i < a.rows && c0 < up_cols) *(uint32_t*)(a.q + (r0 + i) * a.ldq + c0 / 2) = numbers4(v, b);
      uint32_t s = b << (8 * (l >> 2));
      s |= dpp_u<0x128>(s);
      s |= dpp_u<0x124>(s);
      if (l == 0) rscale[g * 8 + i] = s;
    }
  }
  if (turn) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t b = scale4(max_rows(cm[e]));
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = raw[i].get(e);
      *(uint32_t*)(turned + (l * 8 + e) * CLD + g * 4) = numbers4(v, b);
      if (g % 4 == 0) cscale[l * 8 + e][w] = (uint8_t)b;
    }
  }
  if constexpr (SUMS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = sum_q(cs[e]);
    if (g % 4 == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) csum[w][l * 8 + e] = cs[e];
    }
  }
  __syncthreads();
  if (turn) {
    // four lanes to a column, 16 bytes each
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int at = k * 64 + (threadIdx.x >> 2), piece = threadIdx.x & 3;
      const int64_t c = cb * 128 + at, r = rb * 128 + piece * 32;
      const uint32_t* from = (const uint32_t*)(turned + at * CLD + piece * 16);
      if (c < a.cols && r < up_rows) *(uint4*)(a.qt + c * a.ldqt + r / 2) = uint4{from[0], from[1], from[2], from[3]};
    }
  }
  const int t = threadIdx.x & 127;
  const int64_t r = rb * 128 + t, c = cb * 128 + t;
  if (threadIdx.x < 128) {
    if (a.q != nullptr && r < a.rows) ((uint32_t*)a.scale)[cb * a.rows + r] = rscale[t];
  } else if (c < a.cols) {
    if (turn) ((uint32_t*)a.scale_t)[rb * a.cols + c] = *(const uint32_t*)cscale[t];
    if constexpr (SUMS) a.part[rb * a.cols + c] = ((csum[0][t] + csum[1][t]) + csum[2][t]) + csum[3][t];
  }
}

// Back: lanes of N numbers, 16 bytes of y each, to 128 columns.  LARGE: y is larger than the L2s.
template <typename YT, bool LARGE>
__global__ void __launch_bounds__(256) k_dequant4(Dequant4 a) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef YT out __attribute__((ext_vector_type(16 / sizeof(YT)), aligned(2)));
  constexpr int N = 16 / sizeof(YT), LANES = 128 / N, ROWS = 256 / LANES;
  const int l = threadIdx.x & (LANES - 1);
  const int64_t end = (a.a.cols + 31) & ~31LL;
  const uint32_t cbs = (uint32_t)ceil_div(a.a.cols, 128);
  const int64_t u0 = (blockIdx.y * (int64_t)kGridRow + blockIdx.x) * kUnits;
  auto place = [&](int k, int64_t& r, int64_t& cb) {
    const int64_t g = (u0 + k) / cbs;
    cb = u0 + k - g * cbs;
    r = g * ROWS + threadIdx.x / LANES;
  };
  uint32_t w[kUnits];
  uint8_t s[kUnits];
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    int64_t r, cb;
    place(k, r, cb);
    const int64_t c = cb * 128 + l * N;
    const uint8_t* q = a.a.q + r * a.a.ld + c / 2;
    const bool in = r < a.a.rows && c < end;
    w[k] = in ? (N == 8 ? *(const uint32_t*)q : *(const uint16_t*)q) : 0;
    s[k] = in ? a.a.scale[(cb * a.a.rows + r) * 4 + l * N / 32] : 0;
  }
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    int64_t r, cb;
    place(k, r, cb);
    const int64_t c = cb * 128 + l * N;
    if (r >= a.a.rows) break;
    const float x = power(s[k]);
    const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], x, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], x, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], x, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], x, 3)};
    out y;
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = (YT)(s[k] == 255 ? __builtin_nanf("") : v[e >> 1][e & 1]);
    YT* to = (YT*)a.y + r * a.ldy + c;
    if (c + N <= a.a.cols) {
      if (LARGE)
        __builtin_nontemporal_store(y, (out*)to);
      else
        *(out*)to = y;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (c + e < a.a.cols) to[e] = y[e];
    }
  }
}

}  // namespace dev

using namespace dev;

// Reads of more than half the last-level cache (256 MB), and writes of more than all L2s
// hold, do not pass through L2: 852,640 x 256 fp32 to both copies 264 to 234 us, 32,768 x
// 4096 bf16 93 to 77, but 5120 x 5120 bf16, which the last level holds, 20 to 23; back to
// fp32 852,640 x 256 (with 16 bytes a lane) 324 to 139, but rows that are not aligned meet
// in L2 (5120 x 4999 bf16 14 us, past it 19).
constexpr int64_t kLargeIn = 128LL << 20, kLargeOut = 32LL << 20;

template <typename XT, bool SUMS>
void launch_tiles(const Quant4& a, hipStream_t s) {
  const dim3 g = grid_of(ceil_div(a.rows, 128) * ceil_div(a.cols, 128));
  if (a.rows * a.cols * (int64_t)sizeof(XT) > kLargeIn)
    hipLaunchKernelGGL((k_quant4_tile<XT, SUMS, true>), g, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_quant4_tile<XT, SUMS, false>), g, dim3(256), 0, s, a);
}

hipError_t launch_quant4(const Quant4& a, hipStream_t s) {
  if (a.rows > 0) {
    if (!a.qt && !a.colsum) {
      const dim3 g = grid_of(ceil_div(ceil_div(a.rows, 16) * ceil_div(a.cols, 128), kUnits));
      if (a.x_type == MGN_FP32)
        hipLaunchKernelGGL((k_quant4_rows<float>), g, dim3(256), 0, s, a);
      else
        hipLaunchKernelGGL((k_quant4_rows<bf16>), g, dim3(256), 0, s, a);
    } else if (a.x_type == MGN_FP32) {
      a.colsum ? launch_tiles<float, true>(a, s) : launch_tiles<float, false>(a, s);
    } else {
      a.colsum ? launch_tiles<bf16, true>(a, s) : launch_tiles<bf16, false>(a, s);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.colsum)
    return launch_column_reduce(a.part, ceil_div(a.rows, 128), a.cols, &a.colsum, 1, a.accumulate, s);
  return hipSuccess;
}

template <typename YT>
void launch_back(const Dequant4& a, hipStream_t s) {
  const dim3 g = grid_of(ceil_div(ceil_div(a.a.rows, (int64_t)(32 / sizeof(YT))) * ceil_div(a.a.cols, 128), kUnits));
  if (a.a.rows * a.a.cols * (int64_t)sizeof(YT) > kLargeOut && (((uintptr_t)a.y | (uintptr_t)(a.ldy * sizeof(YT))) & 15) == 0)
    hipLaunchKernelGGL((k_dequant4<YT, true>), g, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_dequant4<YT, false>), g, dim3(256), 0, s, a);
}

hipError_t launch_dequant4(const Dequant4& a, hipStream_t s) {
  a.y_type == MGN_FP32 ? launch_back<float>(a, s) : launch_back<bf16>(a, s);
  return hipGetLastError();
}

}  // namespace mgn
