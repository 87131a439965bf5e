// 8-bit quantisation with one scale for each block of 1 or 128 rows and 128
// columns (see include/mgn.h): scale = max(amax / F, 2^-126), numbers = the
// 8-bit numbers nearest x / scale, ties to even.
//
// Bound by memory: an element is read once (2 or 4 bytes) and written as one
// byte a copy.  k_quant_rows (rows only, block_rows 1) gives 16 lanes to a
// block of 128; k_quant_tile takes a tile of 128 x 128, lane (g, l) the rows
// [4 g, 4 g + 4) of columns [8 l, 8 l + 8): rows are written from registers, the
// transpose goes through LDS as 4-byte pieces of a column: of the same numbers
// where rows and columns share the block's scale, else of numbers of its own.  A
// block takes one tile, and three blocks a CU (six waves a SIMD) hide its three
// phases: with 13 tiles a block, sums kept, 118 registers allowed two, and 852,640 x
// 128 took 186 us.
//
// The quotient is exact where it matters: x times a reciprocal of the scale
// is within 2 ulp of it, so it rounds as the quotient does unless it is that close to the
// middle of two 8-bit numbers; groups of 4 or 8 with such an element (under 1 in
// 10,000) are corrected by their remainders.
//
// Measured: 852,640 x 128 fp32 to both copies in e5m2 and the column sums 160 us and
// 10 (663 MB at 4.1 TB/s of 4.75 in a copy), 5120 x 4999 bf16 in 128 x 128 blocks to
// both copies 26 us (3.9 TB/s; with each copy's numbers computed for itself 48), in
// blocks of one row 39, one row of 4096 4.5 us.
#include "dev_common.hpp"
#include "row_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

// The larger magnitude; a NaN wins.
__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(__builtin_fabsf(a), __builtin_fabsf(b));
}

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

// A block's scale and a reciprocal of it (within an ulp) from its largest
// magnitude.  A block with an infinity or a NaN: inv 0.  The division by the
// constant F: with y the float nearest 1 / F, q = amax y and the exact remainder
// r = amax - q F, q + r y rounds to the quotient's nearest float (Markstein); not
// where r may be subnormal, so small values are divided as such.
template <int F>
__device__ __forceinline__ float scale_of(float amax, float& inv) {
  if (!(amax < __builtin_inff())) {
    inv = 0.f;
    return __builtin_nanf("");
  }
  constexpr float y = 1.f / Format<F>::most;
  const float q = amax * y;
  float s = __builtin_fmaf(__builtin_fmaf(-q, Format<F>::most, amax), y, q);
  if (amax < 0x1p-90f) s = fmaxf(amax / Format<F>::most, 0x1p-126f);
  inv = __builtin_amdgcn_rcpf(s);
  return s;
}

// x / s as a float that rounds to the format as the quotient itself does: a float
// beside it whose last bit is set where the quotient has more bits.  t is within
// 2 ulp, and one correction by the remainder x - t s leaves an error under an ulp,
// whose side the next remainder tells: that one is exact (s in [2^-46, 2^120]; where
// it is not, t is so small that all its neighbours round to 0).
__device__ __forceinline__ float quotient(float x, float s, float inv) {
  const float a = __builtin_fabsf(x);
  float t = a * inv;
  t = __builtin_fmaf(__builtin_fmaf(-t, s, a), inv, t);
  const float r = __builtin_fmaf(-t, s, a);
  uint32_t u = __float_as_uint(t);
  if ((u & 1) == 0) u += r > 0.f ? 1 : r < 0.f ? -1 : 0;
  return __builtin_copysignf(__uint_as_float(u), x);
}

// t: what rounds to the 8-bit numbers of v.  v * inv does for all N unless one
// is within 4 ulp of the middle of two numbers; the smallest distance to that
// (from -4 ulp on) is taken in units that wrap around at 2^32.  Below the
// smallest normal number the numbers are spaced as between it and its double,
// so it is added there.  No clamp: |v / s| is at most F (1 + 2^-23), which rounds
// to F.
template <int F, int N>
__device__ __forceinline__ void to_numbers(float (&t)[N], const float (&v)[N], float s, float inv) {
  constexpr int up = 32 - Format<F>::low;
  constexpr uint32_t tie = 4u << up;
  uint32_t near = ~0u;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    t[e] = v[e] * inv;
    const float a = __builtin_fabsf(t[e]), w = a + (a < Format<F>::normal ? Format<F>::normal : 0.f);
    near = min(near, (__float_as_uint(w) << up) + (0x80000000u + tie));
  }
  if (near <= 2 * tie || inv == 0.f) {
    // both by 2^80 where s is small: products of last bits stay normal
    const float up2 = s < 0x1p-40f ? 0x1p80f : 1.f, down2 = s < 0x1p-40f ? 0x1p-80f : 1.f;
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = inv == 0.f ? 0.f : quotient(v[e] * up2, s * up2, inv * down2);
  }
}
template <int F>
__device__ __forceinline__ uint32_t numbers(const float (&v)[4], float s, float inv) {
  float t[4];
  to_numbers<F>(t, v, s, inv);
  return Format<F>::pack(t[2], t[3], Format<F>::pack(t[0], t[1], 0, false), true);
}
template <int F>
__device__ __forceinline__ uint2 numbers(const float (&v)[8], float s, float inv) {
  float t[8];
  to_numbers<F>(t, v, s, inv);
  return uint2{Format<F>::pack(t[2], t[3], Format<F>::pack(t[0], t[1], 0, false), true),
               Format<F>::pack(t[6], t[7], Format<F>::pack(t[4], t[5], 0, false), true)};
}

// The largest of 16 lanes that share a DPP row.
__device__ __forceinline__ float max16(float v) {
  v = larger(v, dpp_f<0x128>(v));
  v = larger(v, dpp_f<0x124>(v));
  v = larger(v, dpp_f<0x122>(v));
  return larger(v, dpp_f<0x121>(v));
}

constexpr int kChunk = 4;  // column blocks that a block of k_quant_rows takes from its 16 rows

template <typename XT, int F>
__global__ void __launch_bounds__(256) k_quant_rows(Quant8 a) {
  const int l = threadIdx.x & 15;
  const int64_t cb = ceil_div(a.cols, 128);
  const uint32_t chunks = (uint32_t)ceil_div(cb, (int64_t)kChunk), block = blockIdx.y * (uint32_t)kGridRow + blockIdx.x,
                 group = block / chunks;
  const int64_t r = (int64_t)group * 16 + (threadIdx.x >> 4), k0 = (int64_t)(block - group * chunks) * kChunk;
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
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = raw[k].get(e);
      m = larger(m, v[e]);
    }
    s = scale_of<F>(max16(m), inv);
    if (k0 + k >= cb) break;
    // 8 bytes: whole inside the row's zero padding to 16 bytes, or beyond it
    if (c < ((a.cols + 15) & ~15LL)) *(uint2*)(a.q + r * a.ldq + c) = numbers<F>(v, s, inv);
    if (l == 0) a.scale[(k0 + k) * a.rows + r] = s;
  }
}

// The largest of the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float max_q(float f) {
  const uint32_t v = __float_as_uint(f);
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const uint32_t u = __float_as_uint(larger(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return larger(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

constexpr int kColLd = 132;           // bytes of a column in LDS

// Four rows of four numbers as four columns.
__device__ __forceinline__ void turn4(uint32_t (&t)[4], uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
  const uint32_t a = __builtin_amdgcn_perm(r1, r0, 0x05010400), b = __builtin_amdgcn_perm(r3, r2, 0x05010400),
                 c = __builtin_amdgcn_perm(r1, r0, 0x07030602), d = __builtin_amdgcn_perm(r3, r2, 0x07030602);
  t[0] = __builtin_amdgcn_perm(b, a, 0x05040100);
  t[1] = __builtin_amdgcn_perm(b, a, 0x07060302);
  t[2] = __builtin_amdgcn_perm(d, c, 0x05040100);
  t[3] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

template <typename XT, int F, bool SQUARE, bool SUMS>
__global__ void __launch_bounds__(512, SQUARE ? 8 : 6) k_quant_tile(Quant8 a) {
  __shared__ __align__(16) uint8_t turned[128 * kColLd];
  __shared__ __align__(16) float cmax[8][128];
  __shared__ __align__(16) float csum[8][128];
  __shared__ float wmax[8];
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, w = threadIdx.x >> 6;
  const int64_t cbs = ceil_div(a.cols, 128), rbs = ceil_div(a.rows, 128);
  const uint32_t block = blockIdx.y * (uint32_t)kGridRow + blockIdx.x;
  const int64_t rb = block / (uint32_t)cbs, cb = block - rb * cbs;
  if (rb >= rbs) return;  // behind the last block
  const int64_t up_cols = (a.cols + 15) & ~15LL, up_rows = (a.rows + 15) & ~15LL;
  const int64_t c0 = cb * 128 + l * 8;
  const int n = (int)min(max(a.cols - c0, (int64_t)0), (int64_t)8);
  const bool turn = a.qt != nullptr;
  float cs[8] = {};
  const int64_t r0 = rb * 128 + g * 4;
  Raw8<XT> raw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = min(r0 + i, a.rows - 1);
    raw[i] = load8((const XT*)a.x + r * a.ldx + c0, r0 + i < a.rows ? n : 0);
  }
  float rmax[4], cm[8] = {}, all = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    rmax[i] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = raw[i].get(e);
      rmax[i] = larger(rmax[i], f);
      if (!SQUARE) cm[e] = larger(cm[e], f);
      if (SUMS) cs[e] += f;
    }
    all = larger(all, rmax[i]);
  }
  if (turn && !SQUARE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) cm[e] = max_q(cm[e]);
    if (g % 4 == 0) {
      *(float4*)&cmax[w][l * 8] = float4{cm[0], cm[1], cm[2], cm[3]};
      *(float4*)&cmax[w][l * 8 + 4] = float4{cm[4], cm[5], cm[6], cm[7]};
    }
  }
  if (SQUARE) {
    all = max_q(max16(all));
    if ((threadIdx.x & 63) == 0) wmax[w] = all;
  }
  __syncthreads();
  if constexpr (SQUARE) {
    // one scale, so the transpose has the same numbers
    float m = 0.f, s, inv;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = larger(m, wmax[j]);
    s = scale_of<F>(m, inv);
    if (threadIdx.x == 0) {
      if (a.q != nullptr) a.scale[cb * rbs + rb] = s;
      if (turn) a.scale_t[rb * cbs + cb] = s;
    }
    uint2 k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = raw[i].get(e);
      k[i] = numbers<F>(v, s, inv);
      if (a.q != nullptr && r0 + i < a.rows && c0 < up_cols) *(uint2*)(a.q + (r0 + i) * a.ldq + c0) = k[i];
    }
    if (turn) {
      uint32_t t[4];
      turn4(t, k[0].x, k[1].x, k[2].x, k[3].x);
#pragma unroll
      for (int e = 0; e < 4; ++e) *(uint32_t*)(turned + (l * 8 + e) * kColLd + g * 4) = t[e];
      turn4(t, k[0].y, k[1].y, k[2].y, k[3].y);
#pragma unroll
      for (int e = 0; e < 4; ++e) *(uint32_t*)(turned + (l * 8 + 4 + e) * kColLd + g * 4) = t[e];
    }
  } else {
    if (a.q != nullptr) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8], inv;
        const float s = scale_of<F>(max16(rmax[i]), inv);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = raw[i].get(e);
        if (r0 + i < a.rows) {
          if (c0 < up_cols) *(uint2*)(a.q + (r0 + i) * a.ldq + c0) = numbers<F>(v, s, inv);
          if (l == 0) a.scale[cb * a.rows + r0 + i] = s;
        }
      }
    }
    if (turn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) cm[e] = 0.f;
#pragma unroll 2  // all at once: 64 registers
      for (int j = 0; j < 8; ++j) {
        const float4 x = *(const float4*)&cmax[j][l * 8], y = *(const float4*)&cmax[j][l * 8 + 4];
        const float m[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) cm[e] = larger(cm[e], m[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v[4], inv;
        const float s = scale_of<F>(cm[e], inv);
        if (g == 0 && e < n) a.scale_t[rb * a.cols + c0 + e] = s;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = raw[i].get(e);
        *(uint32_t*)(turned + (l * 8 + e) * kColLd + g * 4) = numbers<F>(v, s, inv);
      }
    }
  }
  if (turn) {
    __syncthreads();
    // 32 bytes of a column a thread
    const int64_t c = cb * 128 + (threadIdx.x >> 2), r = rb * 128 + (threadIdx.x & 3) * 32;
    if (c < a.cols) {
      const uint32_t* from = (const uint32_t*)(turned + (threadIdx.x >> 2) * kColLd + (threadIdx.x & 3) * 32);
      uint8_t* to = a.qt + c * a.ldqt + r;
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (r + 16 * k < up_rows) *(uint4*)(to + 16 * k) = uint4{from[4 * k], from[4 * k + 1], from[4 * k + 2], from[4 * k + 3]};
    }
  }
  if constexpr (SUMS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = sum_q(cs[e]);
    if (g % 4 == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) csum[w][l * 8 + e] = cs[e];
    }
    __syncthreads();
    const int64_t c = cb * 128 + threadIdx.x;
    if (threadIdx.x < 128 && c < a.cols) {
      float t = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) t += csum[j][threadIdx.x];
      a.part[rb * a.cols + c] = t;
    }
  }
}

}  // namespace dev

using namespace dev;

hipError_t launch_quant8(const Quant8& a, hipStream_t s) {
  const int64_t cbs = ceil_div(a.cols, 128), rbs = ceil_div(a.rows, 128);
#define MGN_Q8(n, threads, K, ...)                                                                            \
  do {                                                                                                        \
    if (a.x_type == MGN_FP32 && a.format == MGN_E4M3)                                                         \
      hipLaunchKernelGGL((K<float, MGN_E4M3 __VA_ARGS__>), grid_of(n), dim3(threads), 0, s, a);               \
    else if (a.x_type == MGN_FP32)                                                                            \
      hipLaunchKernelGGL((K<float, MGN_E5M2 __VA_ARGS__>), grid_of(n), dim3(threads), 0, s, a);               \
    else if (a.format == MGN_E4M3)                                                                            \
      hipLaunchKernelGGL((K<bf16, MGN_E4M3 __VA_ARGS__>), grid_of(n), dim3(threads), 0, s, a);                \
    else                                                                                                      \
      hipLaunchKernelGGL((K<bf16, MGN_E5M2 __VA_ARGS__>), grid_of(n), dim3(threads), 0, s, a);                \
  } while (0)
  if (a.rows > 0) {
    if (!a.qt && !a.colsum && a.block_rows == 1)
      MGN_Q8(ceil_div(a.rows, 16) * ceil_div(cbs, kChunk), 256, k_quant_rows, );
    else if (a.block_rows == 1 && a.colsum)
      MGN_Q8(rbs * cbs, 512, k_quant_tile, , false, true);
    else if (a.block_rows == 1)
      MGN_Q8(rbs * cbs, 512, k_quant_tile, , false, false);
    else if (a.colsum)
      MGN_Q8(rbs * cbs, 512, k_quant_tile, , true, true);
    else
      MGN_Q8(rbs * cbs, 512, k_quant_tile, , true, false);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.colsum) return launch_column_reduce(a.part, rbs, a.cols, &a.colsum, 1, a.accumulate, s);
  return hipSuccess;
}

}  // namespace mgn
