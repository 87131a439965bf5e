// 8-bit quantisation with one scale for each block of 1 or 128 rows and 128
// columns (see include/mgn.h): scale = max(amax / F, 2^-126), numbers = the
// 8-bit numbers nearest x / scale, ties to even.
//
// Bound by memory: an element is read once (2 or 4 bytes) and written as one
// byte a copy.  k_quant_rows (rows only, block_rows 1) gives 16 lanes to a
// block of 128; k_quant_tile takes a tile of 128 x 128, lane (g, l) the rows
// [8 g, 8 g + 8) of columns [8 l, 8 l + 8), so that a lane holds 8 consecutive
// numbers of a row and of a column: rows are written from registers, the
// transpose goes through LDS as 8-byte pieces of a column, and the column
// maxima and sums need one step across the 16 row groups.
//
// The quotient is exact where it matters: x * fl(1 / scale) is within 2 ulp
// of it, so it rounds as the quotient does unless it is that close to the
// middle of two 8-bit numbers, or subnormal in the format; those elements
// (some 2^-17 of all) are divided in double.
#include "dev_common.hpp"
#include "row_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

__device__ __forceinline__ uint32_t abs_bits(float f) { return __float_as_uint(f) & 0x7fffffffu; }
constexpr uint32_t kInfBits = 0x7f800000u;

template <int F>
struct Format;
template <>
struct Format<MGN_E4M3> {
  static constexpr float most = 448.f;
  static constexpr int low = 20;           // float32 mantissa bits below the format's
  static constexpr float normal = 0x1p-6f; // smallest normal number
  static __device__ __forceinline__ uint32_t pack(float a, float b, uint32_t old, bool hi) {
    return hi ? __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, true) : __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, false);
  }
};
template <>
struct Format<MGN_E5M2> {
  static constexpr float most = 57344.f;
  static constexpr int low = 21;
  static constexpr float normal = 0x1p-14f;
  static __device__ __forceinline__ uint32_t pack(float a, float b, uint32_t old, bool hi) {
    return hi ? __builtin_amdgcn_cvt_pk_bf8_f32(a, b, old, true) : __builtin_amdgcn_cvt_pk_bf8_f32(a, b, old, false);
  }
};

// A block's scale and its reciprocal from the largest magnitude's bits (NaN
// bits are above infinity's).  A block with a NaN or an infinity: inv 0.
template <int F>
__device__ __forceinline__ float scale_of(uint32_t amax, float& inv) {
  if (amax >= kInfBits) {
    inv = 0.f;
    return __uint_as_float(0x7fc00000u);
  }
  const float s = fmaxf(__uint_as_float(amax) / Format<F>::most, 0x1p-126f);
  inv = 1.f / s;
  return s;
}

// Whether t = x * inv may round to another number of the format than x / s.
template <int F>
__device__ __forceinline__ bool unsure(float t) {
  constexpr uint32_t mask = (1u << Format<F>::low) - 1, half = 1u << (Format<F>::low - 1);
  const uint32_t b = abs_bits(t);
  return ((b - half + 4) & mask) <= 8 || (t != 0.f && b < __float_as_uint(Format<F>::normal) + 8);
}

// x / s as a float that rounds to the format as the quotient itself does:
// rounded to odd, so that the last bit remembers what the quotient has beyond it.
__device__ __forceinline__ float quotient(float x, float s) {
  const double d = (double)x / (double)s;
  const float t = (float)d;
  uint32_t u = __float_as_uint(t);
  if ((double)t != d && (u & 1) == 0) u += fabs((double)t) < fabs(d) ? 1 : -1;
  return __uint_as_float(u);
}

template <int F>
__device__ __forceinline__ uint2 numbers8(const float (&v)[8], float s, float inv) {
  float t[8];
  bool slow = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t[e] = inv == 0.f ? 0.f : v[e] * inv;
    slow |= unsure<F>(t[e]);
  }
  if (slow) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (unsure<F>(t[e])) t[e] = quotient(v[e], s);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = fminf(fmaxf(t[e], -Format<F>::most), Format<F>::most);
  uint2 r;
  r.x = Format<F>::pack(t[2], t[3], Format<F>::pack(t[0], t[1], 0, false), true);
  r.y = Format<F>::pack(t[6], t[7], Format<F>::pack(t[4], t[5], 0, false), true);
  return r;
}

// The largest of 16 lanes that share a DPP row.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  auto step = [](uint32_t a, float f) { return max(a, __float_as_uint(f)); };
  v = step(v, dpp_f<0x128>(__uint_as_float(v)));
  v = step(v, dpp_f<0x124>(__uint_as_float(v)));
  v = step(v, dpp_f<0x122>(__uint_as_float(v)));
  v = step(v, dpp_f<0x121>(__uint_as_float(v)));
  return v;
}

constexpr int kChunk = 4;  // column blocks that a block of k_quant_rows takes from its 16 rows

template <typename XT, int F>
__global__ void __launch_bounds__(256) k_quant_rows(Quant8 a) {
  const int l = threadIdx.x & 15;
  const int64_t cb = ceil_div(a.cols, 128), chunks = ceil_div(cb, (int64_t)kChunk);
  const int64_t r = blockIdx.x / chunks * 16 + (threadIdx.x >> 4), k0 = blockIdx.x % chunks * kChunk;
  if (r >= a.rows) return;  // all 16 lanes of the row
  Raw8<XT> raw[kChunk];
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    const int64_t c = (k0 + k) * 128 + l * 8;
    raw[k] = load8((const XT*)a.x + r * a.ldx + c, (int)min(a.cols - c, (int64_t)8));
  }
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    const int64_t c = (k0 + k) * 128 + l * 8;
    float v[8], s, inv;
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = raw[k].get(e);
      m = max(m, abs_bits(v[e]));
    }
    m = max16(m);
    s = scale_of<F>(m, inv);
    if (k0 + k >= cb) break;
    // 8 bytes: whole inside the row's zero padding to 16 bytes, or beyond it
    if (c < ((a.cols + 15) & ~15LL)) *(uint2*)(a.q + r * a.ldq + c) = numbers8<F>(v, s, inv);
    if (l == 0) a.scale[(k0 + k) * a.rows + r] = s;
  }
}

constexpr int64_t kTileBlocks = 1024;  // of k_quant_tile, four a CU
constexpr int kColLd = 132;  // bytes of a column in LDS: 16 lanes' 8-byte pieces in distinct banks

template <typename XT, int F>
__global__ void __launch_bounds__(256) k_quant_tile(Quant8 a) {
  __shared__ __align__(16) uint8_t turned[128 * kColLd];
  __shared__ uint32_t cmax[16][128];
  __shared__ float csum[16][128];
  __shared__ uint32_t wmax[2][4];  // in turn: a block of waves may be a tile ahead
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int64_t cbs = ceil_div(a.cols, 128), rbs = ceil_div(a.rows, 128);
  const int64_t cb = blockIdx.x % cbs, run = blockIdx.x / cbs;
  const int64_t up_cols = (a.cols + 15) & ~15LL, up_rows = (a.rows + 15) & ~15LL;
  const bool square = a.block_rows == 128, turn = a.qt != nullptr;
  float cs[8] = {};
  for (int64_t rb = run * a.per; rb < min((run + 1) * a.per, rbs); ++rb) {
    // the lane's columns are opaque, or the addresses of all its rows are kept
    // in registers from tile to tile
    int lc = l * 8;
    asm volatile("" : "+v"(lc));
    const int64_t r0 = rb * 128 + g * 8, c0 = cb * 128 + lc;
    const int n = (int)min(max(a.cols - c0, (int64_t)0), (int64_t)8);
    Raw8<XT> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = min(r0 + i, a.rows - 1);
      raw[i] = load8((const XT*)a.x + r * a.ldx + c0, r0 + i < a.rows ? n : 0);
    }
    uint32_t rmax[8], cm[8] = {};
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      rmax[i] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = raw[i].get(e);
        const uint32_t m = abs_bits(f);
        rmax[i] = max(rmax[i], m);
        cm[e] = max(cm[e], m);
        cs[e] += f;
      }
      all = max(all, rmax[i]);
    }
    if (turn && !square) {
#pragma unroll
      for (int e = 0; e < 8; ++e) cmax[g][l * 8 + e] = cm[e];
    }
    if (square) {
      all = max16(all);
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 64; j += 16) w = max(w, (uint32_t)__builtin_amdgcn_readlane((int)all, j));
      if ((threadIdx.x & 63) == 0) wmax[rb & 1][threadIdx.x >> 6] = w;
    }
    __syncthreads();
    float s1 = 0.f, i1 = 0.f;
    if (square) {
      const uint32_t* w = wmax[rb & 1];
      s1 = scale_of<F>(max(max(w[0], w[1]), max(w[2], w[3])), i1);
      if (threadIdx.x == 0) {
        if (a.q != nullptr) a.scale[cb * rbs + rb] = s1;
        if (turn) a.scale_t[rb * cbs + cb] = s1;
      }
    }
    if (a.q != nullptr) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8], s = s1, inv = i1;
        if (!square) s = scale_of<F>(max16(rmax[i]), inv);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = raw[i].get(e);
        __builtin_amdgcn_sched_barrier(0);  // one row at a time, for the registers
        if (r0 + i < a.rows) {
          if (c0 < up_cols) *(uint2*)(a.q + (r0 + i) * a.ldq + c0) = numbers8<F>(v, s, inv);
          if (!square && l == 0) a.scale[cb * a.rows + r0 + i] = s;
        }
      }
    }
    if (turn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v[8], s = s1, inv = i1;
        if (!square) {
          uint32_t m = 0;
#pragma unroll
          for (int j = 0; j < 16; ++j) m = max(m, cmax[j][l * 8 + e]);
          s = scale_of<F>(m, inv);
          if (g == 0 && c0 + e < a.cols) a.scale_t[rb * a.cols + c0 + e] = s;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = raw[i].get(e);
        const uint2 p = numbers8<F>(v, s, inv);
        uint32_t* to = (uint32_t*)(turned + (l * 8 + e) * kColLd + g * 8);
        to[0] = p.x;
        to[1] = p.y;
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();
      const int64_t c = cb * 128 + (threadIdx.x >> 1);
      if (c < a.cols) {
        const uint32_t* from = (const uint32_t*)(turned + (threadIdx.x >> 1) * kColLd + (threadIdx.x & 1) * 64);
        const int64_t r = rb * 128 + (threadIdx.x & 1) * 64;
        uint8_t* to = a.qt + c * a.ldqt + r;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (r + 16 * k < up_rows) *(uint4*)(to + 16 * k) = uint4{from[4 * k], from[4 * k + 1], from[4 * k + 2], from[4 * k + 3]};
      }
    }
  }
  if (a.colsum != nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) csum[g][l * 8 + e] = cs[e];
    __syncthreads();
    const int64_t c = cb * 128 + threadIdx.x;
    if (threadIdx.x < 128 && c < a.cols) {
      float t = 0.f;
#pragma unroll
      for (int j = 0; j < 16; ++j) t += csum[j][threadIdx.x];
      a.part[run * a.cols + c] = t;
    }
  }
}

}  // namespace dev

using namespace dev;

hipError_t launch_quant8(const Quant8& in, hipStream_t s) {
  Quant8 a = in;
  const int64_t cbs = ceil_div(a.cols, 128), rbs = ceil_div(a.rows, 128);
  // blocks of k_quant_tile: with sums over the columns as many as run at a time,
  // each leaving one row of partial sums
  a.per = a.colsum ? std::max<int64_t>(1, rbs * cbs / kTileBlocks) : 1;
  const int64_t runs = ceil_div(rbs, a.per);
#define MGN_Q8(K, n)                                                                                 \
  do {                                                                                               \
    if (a.x_type == MGN_FP32 && a.format == MGN_E4M3)                                                \
      hipLaunchKernelGGL((K<float, MGN_E4M3>), dim3((unsigned)(n)), dim3(256), 0, s, a);             \
    else if (a.x_type == MGN_FP32)                                                                   \
      hipLaunchKernelGGL((K<float, MGN_E5M2>), dim3((unsigned)(n)), dim3(256), 0, s, a);             \
    else if (a.format == MGN_E4M3)                                                                   \
      hipLaunchKernelGGL((K<bf16, MGN_E4M3>), dim3((unsigned)(n)), dim3(256), 0, s, a);              \
    else                                                                                             \
      hipLaunchKernelGGL((K<bf16, MGN_E5M2>), dim3((unsigned)(n)), dim3(256), 0, s, a);              \
  } while (0)
  if (a.rows > 0) {
    if (!a.qt && !a.colsum && a.block_rows == 1)
      MGN_Q8(k_quant_rows, ceil_div(a.rows, 16) * ceil_div(cbs, kChunk));
    else
      MGN_Q8(k_quant_tile, runs * cbs);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.colsum) return launch_column_reduce(a.part, runs, a.cols, a.cols, a.colsum, a.accumulate, s);
  return hipSuccess;
}

}  // namespace mgn
