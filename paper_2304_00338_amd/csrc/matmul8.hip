// Product of block-scaled 8-bit matrices (see include/mgn.h):
//   c[m][n] = act(sum_kb sa[kb][m] sb[kb][n] sum_{k in block kb} a[m][k] b[n][k] + bias[n]).
//
// Two ways to sum a block, by the type of c:
//  * bf16 c of more than 16 rows: the 8-bit matrix instruction, 32x32x64 (f8f6f4).
//    It adds eight products at a time, cut off (towards zero) 2^-13 below the largest
//    of the eight; such eights, and what came before, are added in full.  On normal
//    values a block is off by 1.5e-5 (relative 2-norm), a hundredth of the
//    rounding of c: 0.3 to 1.2% of the results are the other neighbour in bf16, and
//    their distance from 64 bits, 1.66e-3, is the same to four digits.
//  * fp32 c, and up to 16 rows: the operands widened to bf16 (exactly) for the 16-bit
//    instruction, 32x32x16, which adds in fp32; half the rate.
// Summing a bf16 c in fp32 as well would take 1089 us for 32,768 x 4096 x 4096 (580),
// 225 for 16,384 x 1000 x 5000 (125), 33.6 for 64 x 8192 x 8192 (28), 21.4 for 23 x
// 10,007 x 5000 (18.7); for one row 7.0 instead of 7.2 (4096 x 4096), for 16 rows 7.8
// instead of 7.7.
// Either way a block's sum is scaled and added to an fp32 accumulator.
//
// Lane l of an instruction holds row l & 31, and of it the bytes
// [32 (l >> 5), + 32) of 64.  Which k a byte stands for does not matter as
// long as both operands agree.  b's rows are the first operand (i), a's the
// second (j), so a lane's 16 results belong to one row of a (its scale is one
// value a lane) and to runs of 4 consecutive columns of c: result r is row
// 8 (r / 4) + 4 (l >> 5) + r % 4 of the 32.
#include "dev_common.hpp"
#include "row_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// the matrix instruction's codes of the formats are 0 and 1
static_assert(MGN_E4M3 == 2 && MGN_E5M2 == 3, "8-bit formats in the order of the instruction's codes");
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Scales.  Their product may leave the normal numbers where the result does not
// (twice 2^70 before a sum of 2^-30, or before a sum of 0, which would become a NaN).
// So half of each one's power of two, 2^floor(e / 2), goes into the matrix instruction
// with the operand, or into its widening, and the sum is multiplied by the product of
// the rests, which is a normal number for scales up to 2^124: what comes out of the
// instruction lies between the plain sum and the result.  Both are exact, so a result
// has the bits that it has by the product of the scales, where that is normal.
// (Measured against that product: 32,768 x 4096 x 4096 1% more time, three steps of
// 434,558 x 128 x 384 to fp32 3%, scales for each row of b 5%; with the halves and
// rests formed by each wave for itself 10, 13 and 6.)
__device__ __forceinline__ uint32_t half_of(float s) {  // last byte: 127 + floor(e / 2)
  return (__float_as_uint(s) & 0x7fffffffu) + 0x3f800000u;
}
__device__ __forceinline__ float rest_of(float s) {
  return __builtin_amdgcn_ldexpf(s, 127 - (int)(half_of(s) >> 24));
}

// Eight 8-bit numbers times a scale's half as bf16: exact, normal or 0.
template <int F>
__device__ __forceinline__ bf16x8 widen(int lo, int hi, uint32_t half) {
  const float s = __uint_as_float(half >> 1);  // its exponent is what counts
  bf16x2 v[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int w = i ? hi : lo;
    if constexpr (F == MGN_E4M3) {
      v[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
      v[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true);
    } else {
      v[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, false);
      v[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, true);
    }
  }
  return bf16x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

// What a call asks for, and how it is dealt to blocks.
struct Job {
  Matmul8 p;
  int64_t mt, nt;      // tiles
  int64_t kb, per;     // blocks of 128 columns, and of a split
  int splits;          // > 1: sums of the splits go to p.part [splits][M][N]
};

__device__ const uint4 zero16 = {0, 0, 0, 0};

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
__device__ __forceinline__ void finish(const Matmul8& p, int64_t m, int64_t n, f32x4 v) {
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
__device__ __forceinline__ void put4(const Job& J, int split, int64_t m, int64_t n, f32x4 v) {
  if (J.splits == 1)
    finish(J.p, m, n, v);
  else
    store4(J.p.part + ((int64_t)split * J.p.a.rows + m) * J.p.b.rows + n, v, (int)min(J.p.b.rows - n, (int64_t)4));
}

// Sums of the splits, 4 columns a thread: G threads for each, thread g the splits
// g, g + G, ..., then the G sums in order.
template <int G>
__global__ void __launch_bounds__(256) k_matmul8_join(Job J) {
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

// ---- tiles: BM x BN of c a block of WM x WN waves, each TM x TN times 32 x 32.
//
// Steps of 128 columns, one scale block, go through two LDS buffers by loads
// that write LDS themselves (16 bytes a lane, 8 rows of 128 bytes a wave and
// load), the next step's under the products of the current one, with one
// barrier a step.  A row's 16-byte chunk c sits at place c ^ (row / 2 % 8), so
// that 16 rows of a fragment read cover all 64 banks; the lanes' source
// addresses are permuted to match.  What lies beyond the matrix comes from 16
// zero bytes.  The results go through the wave's own piece of LDS to be
// stored as whole rows.
//
// Measured: 32,768 x 4096 x 4096 to bf16 567 to 591 us on three cards (1.9 PFLOP/s; the
// library's product with one scale an operand reaches 2.5).  Without the loads 0.09 ms
// less, without the scaled additions 0.05: a step's loads take longer than its 64
// products a SIMD, and the eight waves wait at its barrier.  434,558 x 128 x 384 to fp32
// 117 us (3.4 TB/s), weight gradient 128 x 256 x 852,640 86 us (3.8 TB/s) and 8 to join.
template <bool WIDE, int FA, int FB, bool BROW, int WM, int WN, int TM, int TN>
__global__ void __launch_bounds__(WM * WN * 64, 2) k_matmul8_tile(Job J) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32, NWV = WM * WN;
  constexpr int LOADS = (BM + BN) / 8 / NWV;  // of a wave and step
  static_assert((BM / 8) % NWV == 0 && (BN / 8) % NWV == 0, "a load is of one operand for all waves");
  static_assert(NWV % 2 == 0, "a wave's groups of 8 rows have one parity");
  static_assert((BM + BN) * 128 >= NWV * 32 * TN * 32 * 4, "results fit a buffer");
  __shared__ __align__(16) uint8_t buf0[(BM + BN) * 128], buf1[(BM + BN) * 128];
  // scales of a's rows and (BROW) of b's, each as its half and its rest
  constexpr int ROWS = BM + (BROW ? BN : 0);
  __shared__ __align__(16) float rest[2][ROWS];
  __shared__ uint32_t half[2][ROWS];
  const Matmul8& p = J.p;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = l & 31, h = l >> 5;
  const int wm = w / WN, wn = w % WN;
  // XCD x (blocks go to the 8 XCDs in turn) takes an eighth of the tiles of all
  // splits, a split's tiles one after the other in groups of 8 rows of tiles, so
  // that the blocks it runs at a time share operands in its L2
  const uint32_t nt = (uint32_t)J.nt, tiles = (uint32_t)J.mt * nt, all = tiles * J.splits, chunk = (all + 7) / 8;
  const uint32_t job = (blockIdx.x & 7) * chunk + (blockIdx.x >> 3);
  if (job >= all) return;
  const uint32_t split = job / tiles, t = job - split * tiles;
  const uint32_t group = t / (8 * nt), in = t - group * 8 * nt, gm = min((uint32_t)J.mt - group * 8, 8u);
  const uint32_t tn = in / gm;
  const int64_t m0 = (int64_t)(group * 8 + in - tn * gm) * BM, n0 = (int64_t)tn * BN;
  const int64_t kb0 = split * J.per, kb1 = min(kb0 + J.per, J.kb);
  const int64_t end = (p.a.cols + 15) & ~15LL;

  // loads: of wave w the 8 rows from 8 (i NWV + w) on.  A wave's rows have a
  // scalar base and 32-bit offsets.  At the matrices' ends, with an ld of 2^28 or
  // more, and in a step that the columns end in, addresses are of 64 bits: a row
  // that is not there is the last one again (its results are not stored), and
  // what lies beyond the columns comes from the 16 zero bytes.  Those addresses
  // are formed anew each time (opaque lane): kept, they would spill.
  const int lrow = l >> 3, lchunk = ((l & 7) ^ ((4 * (w & 1) + (l >> 4)) & 7)) * 16;
  const uint32_t ata = lrow * (uint32_t)p.a.ld + lchunk, atb = lrow * (uint32_t)p.b.ld + lchunk;
  const bool inner = m0 + BM <= p.a.rows && n0 + BN <= p.b.rows && max(p.a.ld, p.b.ld) < (1LL << 28);
  const uint8_t* const wa = p.a.q + (m0 + w * 8) * p.a.ld;
  const uint8_t* const wb = p.b.q + (n0 + w * 8) * p.b.ld;
  auto to_lds = [&](const uint8_t* src, uint8_t* buf, int i) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                     (__attribute__((address_space(3))) void*)(buf + (i * NWV + w) * 1024), 16, 0, 0);
  };
  auto fetch = [&](uint8_t* buf, int64_t kb) {
    const int64_t k = kb * 128;
    if (inner && k + 128 <= end) {
      int64_t lda = p.a.ld * (NWV * 8), ldb = p.b.ld * (NWV * 8);
      uint32_t la = ata, lb = atb;
      asm volatile("" : "+v"(la), "+v"(lb));
      const uint8_t *xa = wa + k, *xb = wb + k;
#pragma unroll
      for (int i = 0; i < BM / 8 / NWV; ++i) {
        asm volatile("" : "+s"(xa));
        to_lds(xa + la, buf, i);
        xa += lda;
      }
#pragma unroll
      for (int i = 0; i < BN / 8 / NWV; ++i) {
        asm volatile("" : "+s"(xb));
        to_lds(xb + lb, buf, i + BM / 8 / NWV);
        xb += ldb;
      }
    } else {
      int lr = lrow, lc = lchunk;
      asm volatile("" : "+v"(lr), "+v"(lc));
      const uint8_t* zero = (const uint8_t*)&zero16;
#pragma unroll 1
      for (int i = 0; i < LOADS; ++i) {
        const bool isa = i < BM / 8 / NWV;
        const mgn_mat8& x = isa ? p.a : p.b;
        const int64_t r = min((isa ? m0 + (i * NWV + w) * 8 : n0 + (i * NWV + w) * 8 - BM) + lr, x.rows - 1);
        to_lds(k + lc < end ? x.q + r * x.ld + k + lc : zero, buf, i);
      }
    }
  };
  // scales: a thread fetches that of one row of a, or (BROW) of b; what all waves need
  // of it is formed once and goes through LDS.  Else one of b is all that a wave's
  // columns have, which lie in one block of 128.
  static_assert((ROWS & (ROWS - 1)) == 0 && ROWS <= NWV * 64, "threads for all rows");
  const int sha = p.a.block_rows == 128 ? 7 : 0, shb = p.b.block_rows == 128 ? 7 : 0;
  const int64_t Ra = ceil_div(p.a.rows, p.a.block_rows), Rb = ceil_div(p.b.rows, p.b.block_rows);
  const int srow = threadIdx.x & (ROWS - 1);
  const bool ofb = BROW && srow >= BM;
  const int64_t sstep = ofb ? Rb : Ra;
  const float* sfrom = (ofb ? p.b.scale + min(n0 + srow - BM, p.b.rows - 1)
                            : p.a.scale + (min(m0 + srow, p.a.rows - 1) >> sha)) + kb0 * sstep;
  const int64_t nb0 = min(n0 + wn * TN * 32, p.b.rows - 1) >> shb;
  uint32_t hb = 0;
  float rb = 0.f, ns, nb = 0.f;
  auto scales = [&](int64_t kb) {  // kb0, and the next one each time
    ns = *sfrom;
    sfrom += sstep;
    if constexpr (!BROW) nb = (p.b.scale + kb * Rb)[nb0];
  };

  f32x16 acc[TM][TN] = {};
  int off[2][2];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int c = 0; c < 2; ++c) off[s][c] = j * 128 + (((4 * s + 2 * h + c) ^ ((j >> 1) & 7)) * 16);
  auto frag = [&](const uint8_t* rows, int s) {
    const uint4 lo = *(const uint4*)(rows + off[s][0]), hi = *(const uint4*)(rows + off[s][1]);
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
  };
  // fa, fb, rests: of the scales
  auto add = [&](f32x16& to, const f32x16& part, float fa, float fb, const float* rests) {
    if constexpr (BROW) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 s4 = *(const f32x4*)(rests + 8 * g + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[4 * g + e] = __builtin_fmaf(part[4 * g + e], fa * s4[e], to[4 * g + e]);
      }
    } else {
      const float f = fa * fb;
#pragma unroll
      for (int r = 0; r < 16; ++r) to[r] = __builtin_fmaf(part[r], f, to[r]);
    }
  };
  // 8-bit products of the step's last 32 rows that are still to be added
  f32x16 open[TN] = {};
  float open_a = 0.f, open_b = 0.f;
  auto settle = [&]() {
    if constexpr (!WIDE && !BROW) {
#pragma unroll
      for (int n = 0; n < TN; ++n) add(acc[TM - 1][n], open[n], open_a, open_b, nullptr);
    }
  };
  auto products = [&](const uint8_t* buf, int at) {
    const uint8_t* rowsa = buf + wm * TM * 32 * 128;
    const uint8_t* rowsb = buf + (BM + wn * TN * 32) * 128;
    const float *const resta = rest[at] + wm * TM * 32 + j, *const restb = rest[at] + (BROW ? BM + wn * TN * 32 : 0);
    const uint32_t *const halfa = half[at] + wm * TM * 32 + j, *const halfb = half[at] + (BROW ? BM + wn * TN * 32 : 0) + j;
    uint32_t hbn[TN];
#pragma unroll
    for (int n = 0; n < TN; ++n) hbn[n] = BROW ? halfb[n * 32] : hb;
    if constexpr (WIDE) {
      // every operand is widened once: 16 columns of all TM + TN at a time
      f32x16 part[TM][TN] = {};
      uint32_t han[TM];
#pragma unroll
      for (int m = 0; m < TM; ++m) han[m] = halfa[m * 32];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        i32x8 fa[TM], fb[TN];
#pragma unroll
        for (int m = 0; m < TM; ++m) fa[m] = frag(rowsa + m * 4096, s);
#pragma unroll
        for (int n = 0; n < TN; ++n) fb[n] = frag(rowsb + n * 4096, s);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          bf16x8 va[TM], vb[TN];
#pragma unroll
          for (int m = 0; m < TM; ++m) va[m] = widen<FA>(fa[m][i], fa[m][i + 1], han[m]);
#pragma unroll
          for (int n = 0; n < TN; ++n) vb[n] = widen<FB>(fb[n][i], fb[n][i + 1], hbn[n]);
#pragma unroll
          for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int n = 0; n < TN; ++n)
              part[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[n], va[m], part[m][n], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int n = 0; n < TN; ++n) add(acc[m][n], part[m][n], resta[m * 32], rb, restb + (BROW ? n * 32 : 0));
    } else {
      // the last 32 rows' products are added under the next step's first reads
      i32x8 fb[TN][2], fa[2][2];
      uint32_t han[2];
      float ran[2];
      han[0] = halfa[0];
      ran[0] = resta[0];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        fa[0][s] = frag(rowsa, s);
#pragma unroll
        for (int n = 0; n < TN; ++n) fb[n][s] = frag(rowsb + n * 4096, s);
        __builtin_amdgcn_sched_barrier(0);
      }
      settle();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < TM; ++m) {
        f32x16 part[TN];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int n = 0; n < TN; ++n)
            part[n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[n][s], fa[m & 1][s], s ? part[n] : f32x16{},
                                                                      FB - MGN_E4M3, FA - MGN_E4M3, 3, (int)hbn[n], 3,
                                                                      (int)han[m & 1]);
        if (m + 1 < TM) {
#pragma unroll
          for (int s = 0; s < 2; ++s) fa[(m + 1) & 1][s] = frag(rowsa + (m + 1) * 4096, s);
          han[(m + 1) & 1] = halfa[(m + 1) * 32];
          ran[(m + 1) & 1] = resta[(m + 1) * 32];
        }
        if (BROW || m + 1 < TM) {
#pragma unroll
          for (int n = 0; n < TN; ++n) add(acc[m][n], part[n], ran[m & 1], rb, restb + (BROW ? n * 32 : 0));
        } else {
#pragma unroll
          for (int n = 0; n < TN; ++n) open[n] = part[n];
          open_a = ran[m & 1];
          open_b = rb;
        }
        // else the compiler has all reads and products of a step in registers at once
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // The fetched scales are the next step's.  (Where there are more threads than rows two
  // write the same value: a branch here moved products of the step behind it, and
  // the large tiles spilled.)
  auto take = [&](int to) {
    half[to][srow] = half_of(ns);
    rest[to][srow] = rest_of(ns);
    if constexpr (!BROW) {  // one for the wave
      hb = __builtin_amdgcn_readfirstlane(half_of(nb));
      rb = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(rest_of(nb))));
    }
  };

  if (kb0 < kb1) {
    scales(kb0);
    fetch(buf0, kb0);
    take(0);
    __syncthreads();
    for (int64_t kb = kb0; kb < kb1; kb += 2) {
      const int64_t left = kb1 - kb;
      if (left > 1) {
        scales(kb + 1);
        fetch(buf1, kb + 1);
      }
      products(buf0, 0);
      if (left > 1) {
        take(1);
        __syncthreads();
        if (left > 2) {
          scales(kb + 2);
          fetch(buf0, kb + 2);
        }
        products(buf1, 1);
        take(0);
        __syncthreads();
      }
    }
  }
  settle();
  __syncthreads();  // every wave has read its last operands
  // rows of TN * 8 chunks of 4 columns, chunk c at place c ^ row
  constexpr int CH = TN * 8;
  f32x4* mine = (f32x4*)buf0 + w * 32 * CH;
#pragma unroll
  for (int m = 0; m < TM; ++m) {
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        mine[j * CH + ((n * 8 + 2 * g + h) ^ (j & (CH - 1)))] =
            f32x4{acc[m][n][4 * g], acc[m][n][4 * g + 1], acc[m][n][4 * g + 2], acc[m][n][4 * g + 3]};
    wave_lds_sync();
    const int64_t n = n0 + wn * TN * 32 + (l % CH) * 4;
#pragma unroll
    for (int i = 0; i < 32; i += 64 / CH) {
      const int r = i + l / CH;
      const int64_t row = m0 + (wm * TM + m) * 32 + r;
      const f32x4 v = mine[r * CH + ((l % CH) ^ (r & (CH - 1)))];
      if (row < p.a.rows && n < p.b.rows) put4(J, split, row, n, v);
    }
    wave_lds_sync();
  }
}

// ---- few rows of a (up to TM times 16), bound by the weights' bytes.
//
// A block takes 16 rows of b, its 8 waves the steps of 128 columns in turn;
// operands come straight from memory, 32 consecutive bytes a lane (four lanes
// cover a row's 128), a step ahead, and the waves' sums meet in LDS.  The
// instruction is 16x16x128: lane l holds row l & 15, bytes [32 (l >> 4), + 32);
// result r is row 4 (l >> 4) + r of b, column l & 15 a row of a.
//
// Measured in a graph over weights of more bytes than the caches hold: 1 x 4096 x 4096
// 7.0 us, 1 x 4096 x 14336 16.3 (3.6 TB/s), 23 x 10007 x 5000 25 (2.0 TB/s: every block
// reads a through L1, 1.4 times the weights' bytes); the last one over weights of 150 MB
// in turn, which the last-level cache holds, 18.7.
template <bool WIDE, int FB, int FA>
__device__ __forceinline__ f32x4 mma16(i32x8 b, i32x8 a, uint32_t hb, uint32_t ha) {
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(b[i], b[i + 1], hb), widen<FA>(a[i], a[i + 1], ha), c, 0, 0, 0);
    return c;
  } else {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, FB - MGN_E4M3, FA - MGN_E4M3, 3, (int)hb, 3,
                                                            (int)ha);
  }
}

template <bool WIDE, int FA, int FB, int TM>
__global__ void __launch_bounds__(512) k_matmul8_few(Job J) {
  constexpr int NWV = 8;
  __shared__ f32x4 sums[NWV][TM][64];
  const Matmul8& p = J.p;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, j = l & 15, q = l >> 4;
  const int64_t n0 = (blockIdx.y * kGridRow + blockIdx.x) * 16;
  const int split = blockIdx.z;
  const int64_t kb0 = split * J.per, kb1 = min(kb0 + J.per, J.kb);
  const int64_t end = (p.a.cols + 15) & ~15LL;
  const int sha = p.a.block_rows == 128 ? 7 : 0, shb = p.b.block_rows == 128 ? 7 : 0;
  const int64_t Ra = ceil_div(p.a.rows, p.a.block_rows), Rb = ceil_div(p.b.rows, p.b.block_rows);
  const uint8_t *rb = p.b.q + min(n0 + j, p.b.rows - 1) * p.b.ld + q * 32, *ra[TM];
  const float *psa[TM], *psb[4], *psj = p.b.scale + (min(n0 + j, p.b.rows - 1) >> shb);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = min((int64_t)i * 16 + j, p.a.rows - 1);
    ra[i] = p.a.q + m * p.a.ld + q * 32;
    psa[i] = p.a.scale + (m >> sha);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) psb[r] = p.b.scale + (min(n0 + 4 * q + r, p.b.rows - 1) >> shb);
  auto get = [&](const uint8_t* row, int64_t kb) {
    const int64_t k = kb * 128, lim = end - q * 32;
    const uint8_t* z = (const uint8_t*)&zero16;
    const uint4 lo = *(const uint4*)(k < lim ? row + k : z);
    const uint4 hi = *(const uint4*)(k + 16 < lim ? row + k + 16 : z);
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
  };
  struct Step {
    i32x8 a[TM], b;
    float sa[TM], sb[4], sj;
  };
  auto fetch = [&](Step& x, int64_t kb) {
    x.b = get(rb, kb);
    x.sj = psj[kb * Rb];
#pragma unroll
    for (int r = 0; r < 4; ++r) x.sb[r] = psb[r][kb * Rb];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      x.a[i] = get(ra[i], kb);
      x.sa[i] = psa[i][kb * Ra];
    }
  };
  f32x4 acc[TM] = {};
  auto products = [&](const Step& x) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const f32x4 part = mma16<WIDE, FB, FA>(x.b, x.a[i], half_of(x.sj), half_of(x.sa[i]));
#pragma unroll
      for (int r = 0; r < 4; ++r)
        acc[i][r] = __builtin_fmaf(part[r], rest_of(x.sa[i]) * rest_of(x.sb[r]), acc[i][r]);
    }
  };
  if (kb0 + w < kb1) {
    Step x, y;
    fetch(x, kb0 + w);
    for (int64_t kb = kb0 + w; kb < kb1; kb += 2 * NWV) {
      const bool more = kb + NWV < kb1;
      if (more) fetch(y, kb + NWV);
      products(x);
      if (more) {
        if (kb + 2 * NWV < kb1) fetch(x, kb + 2 * NWV);
        products(y);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) sums[w][i][l] = acc[i];
  __syncthreads();
  if (w < TM) {
    f32x4 v = sums[0][w][l];
#pragma unroll
    for (int k = 1; k < NWV; ++k) v += sums[k][w][l];
    const int64_t m = w * 16 + j, n = n0 + 4 * q;
    if (m < p.a.rows && n < p.b.rows) put4(J, split, m, n, v);
  }
}

}  // namespace dev

using namespace dev;

namespace {

constexpr int64_t kCUs = 256;

enum { kFew, kSmallTile, kBigTile };
struct Plan {
  int kind;
  int64_t mt, nt, per;
  int splits;
};

// Which kernel, and into how many parts the sums are split; us a call in a stream of
// calls, bf16 results (fp32 where marked).
//  * Up to 32 rows of a the kernel for few rows, else tiles: 17 x 4096 x 4096 12.6
//    (tiles 16.7), 32 x 1024 x 8192 16.9 (17.3), 24 x 10007 x 5000 19.1 (24.4), 32 x
//    14336 x 4096 27.0 (24.7); 64 x 8192 x 8192 43.9 with four times 16 rows (27.9).
//  * Tiles of 256 x 256 where they occupy three quarters of the CUs, need 8 steps
//    or more and pad little; else of 128 x 128, two blocks a CU: 8192 x 4096 x 4096
//    146 (small 176), 4096 x 3584 x 4096 70.6 (82.5), 16384 x 1000 x 5000 110 (154);
//    but 4096 x 2048 x 4096 66.9 (46.0), 100,000 x 512 x 512 77.0 (72.4), 434,558 x
//    128 x 384 130 (80).  With a scale for each row of b, or for fp32 results, the large
//    tiles spill.
//  * Sums split so that two blocks a CU are busy: 128 x 256 x 852,640 to fp32 110
//    (one block 119, four 121), 64 x 8192 x 8192 27.9 (35.7, 36.6).  For few rows one
//    block of 8 waves a CU is enough: 1 x 4096 x 4096 6.9 whole, 10.2 in two parts.
constexpr int64_t kFewRows = 32;
Plan plan(int64_t m, int64_t n, int64_t k, bool big_ok) {
  Plan r;
  const int64_t kb = ceil_div(k, 128);
  int64_t want;
  if (m <= kFewRows) {
    r.kind = kFew;
    r.mt = 1;
    r.nt = ceil_div(n, 16);
    want = std::min(kCUs / std::max<int64_t>(r.nt, 1), kb / 16);
  } else {
    const int64_t m2 = ceil_div(m, 256), n2 = ceil_div(n, 256), m1 = ceil_div(m, 128), n1 = ceil_div(n, 128);
    const bool big = big_ok && m2 * n2 >= kCUs * 3 / 4 && kb >= 8 && 4 * m2 * n2 * 7 <= m1 * n1 * 8;
    r.kind = big ? kBigTile : kSmallTile;
    r.mt = big ? m2 : m1;
    r.nt = big ? n2 : n1;
    want = big ? 1 : std::min(2 * kCUs / (r.mt * r.nt), kb / 4);
  }
  r.splits = (int)std::max<int64_t>(want, 1);
  r.per = std::max<int64_t>(ceil_div(kb, r.splits), 1);
  r.splits = (int)std::max<int64_t>(ceil_div(kb, r.per), 1);
  return r;
}

template <bool WIDE, int FA, int FB>
void launch(const Job& J, const Plan& r, hipStream_t s) {
  const dim3 grid((unsigned)(8 * ceil_div(r.mt * r.nt * r.splits, 8)));
  if (r.kind == kFew) {
    dim3 g = grid_of(r.nt);
    g.z = (unsigned)r.splits;
    const int64_t m = J.p.a.rows;
    if (m <= 16)  // fp32 sums cost nothing here
      hipLaunchKernelGGL((k_matmul8_few<true, FA, FB, 1>), g, dim3(512), 0, s, J);
    else
      hipLaunchKernelGGL((k_matmul8_few<WIDE, FA, FB, 2>), g, dim3(512), 0, s, J);
    return;
  }
  const bool brow = J.p.b.block_rows == 1;
  if constexpr (!WIDE) {
    if (r.kind == kBigTile) {
      hipLaunchKernelGGL((k_matmul8_tile<WIDE, FA, FB, false, 2, 4, 4, 2>), grid, dim3(512), 0, s, J);
      return;
    }
  }
  if (brow)
    hipLaunchKernelGGL((k_matmul8_tile<WIDE, FA, FB, true, 2, 2, 2, 2>), grid, dim3(256), 0, s, J);
  else
    hipLaunchKernelGGL((k_matmul8_tile<WIDE, FA, FB, false, 2, 2, 2, 2>), grid, dim3(256), 0, s, J);
}

}  // namespace

// The type of c is not known here: as much as either plan takes.
size_t matmul8_workspace(int64_t m, int64_t n, int64_t k) {
  if (m <= 0 || n <= 0) return 0;
  const int splits = std::max(plan(m, n, k, false).splits, plan(m, n, k, true).splits);
  return splits > 1 ? (size_t)splits * (size_t)m * (size_t)n * 4 : 0;
}

hipError_t launch_matmul8(const Matmul8& p, hipStream_t s) {
  const bool wide = p.c_type == MGN_FP32;
  const Plan r = plan(p.a.rows, p.b.rows, p.a.cols, !wide && p.b.block_rows == 128);
  const Job J = {p, r.mt, r.nt, ceil_div(p.a.cols, 128), r.per, r.splits};
#define MGN_MM8_FORMATS(W)                                           \
  do {                                                               \
    if (p.a.format == MGN_E4M3 && p.b.format == MGN_E4M3)            \
      launch<W, MGN_E4M3, MGN_E4M3>(J, r, s);                        \
    else if (p.a.format == MGN_E4M3)                                 \
      launch<W, MGN_E4M3, MGN_E5M2>(J, r, s);                        \
    else if (p.b.format == MGN_E4M3)                                 \
      launch<W, MGN_E5M2, MGN_E4M3>(J, r, s);                        \
    else                                                             \
      launch<W, MGN_E5M2, MGN_E5M2>(J, r, s);                        \
  } while (0)
  if (wide)
    MGN_MM8_FORMATS(true);
  else
    MGN_MM8_FORMATS(false);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || r.splits == 1) return e;
  const int64_t quads = p.a.rows * ceil_div(p.b.rows, 4);
  if (r.splits >= 16)  // 256 splits of 128 x 256: 8 us, with one thread 23
    hipLaunchKernelGGL((k_matmul8_join<16>), dim3((unsigned)ceil_div(quads, 16)), dim3(256), 0, s, J);
  else
    hipLaunchKernelGGL((k_matmul8_join<1>), dim3((unsigned)ceil_div(quads, 256)), dim3(256), 0, s, J);
  return hipGetLastError();
}

}  // namespace mgn
