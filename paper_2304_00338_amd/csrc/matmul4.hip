// Product of 4-bit matrices with a power of two for each 32 columns of a row (see
// include/mgn.h):
//   c[m][n] = act(sum_k a[m][k] b[n][k] + bias[n]).
//
// The matrix instructions take both powers of two for each row and 32 columns, and
// their sums go on in its fp32 accumulator, so there is nothing to scale outside.  What
// they add was checked by their results: a block's 32 products (multiples of a
// quarter up to 36) are exact, sums of blocks of different scales are within a
// rounding of the largest, a scale of 2^-127 counts in full, one of 255 gives NaN.
//
// Lane l of an instruction holds row l & 31 (l & 15), and of it the 16 bytes (32
// numbers) l >> 5 (l >> 4) of 64 (128) columns, with the scale of these 32.  b's rows are
// the first operand (i), a's the second (j), so a lane's results belong to one row of a
// and to runs of 4 consecutive columns of c: result r is row 8 (r / 4) + 4 (l >> 5) +
// r % 4 of the 32.
#include <cmath>

#include "dev_common.hpp"
#include "product_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

constexpr int kE2M1 = 4;  // the matrix instruction's code of the format

// What a call asks for, and how it is dealt to blocks.
struct Job4 {
  Matmul4 p;
  int64_t mt, nt;   // tiles
  int64_t kb, per;  // blocks of 128 columns, and of a split
  int splits;       // > 1: sums of the splits go to p.part [splits][M][N]
};

__device__ __forceinline__ i32x8 operand(uint4 v) { return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0}; }

// 16 bytes of a result.  PAST: past the caches, where rows are aligned: results that stay
// in L2 push out the operands (32,768 x 4096 x 1024 to fp32 170 us, through L2 208; 852,640 x
// 128 x 256 to fp32 121, 144).  Unaligned ones meet in L2 (32,768 x 4099 x 1024 to bf16
// 144, past it 166).  Small results gain too, also where the next launch reads them (calls in a
// graph: 2048 x 2048 x 512 to fp32 8.6 us, through L2 9.7; 65,536 x 256 x 128 to bf16 11.6, 12.6;
// 1024 x 1024 x 8192 with its splits' sums 22.0, 23.0; 4096 x 4096 x 512 to bf16 with a quantiser
// behind it 24.1, 24.8); fp32 results that the last-level cache holds lose (8192 x 2048 x 512
// 21.4, 20.7; 8192 x 4096 x 512 47.5, 42.2; 128 x 256 x 852,640 with 32 MB of splits' sums 66.3,
// 63.9): the rule leaves that.
template <bool PAST>
__device__ __forceinline__ void store16(void* p, uint4 v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
  const u32x4 w = {v.x, v.y, v.z, v.w};
  if (PAST)
    __builtin_nontemporal_store(w, (u32x4*)p);
  else
    *(u32x4*)p = w;
}

// ---- tiles: BM x BN of c a block of WM x WN waves, each TM x TN times 32 x 32.
//
// Steps of 128 columns (64 bytes of a row) go through NB LDS buffers by loads that
// write LDS themselves, NB - 1 steps ahead, the rows' scales (4 bytes a row and step)
// with them.  A row's 16-byte chunk c sits at place c ^ (row / 4 % 4), so that 16
// rows of a fragment read cover all 64 banks; the lanes' source addresses are permuted
// to match.  A step has two halves of 64 columns, and a half's fragments are read under
// the products of the half before it.  The barrier of a step lies between its halves: there
// a wave has read all of the step, whose buffer may be filled again, and waited for its own
// loads of the next one.
//
// Measured: 32,768 x 4096 x 4096 to bf16 305 to 313 us (3.5 PFLOP/s; the library's
// product of such matrices takes 531, and reaches 3.6 at 16,384 each way).  Power
// bounds it: 1024 of a step's 1520 cycles are products, but at 1.5 GHz on random
// numbers (2.2 on zeros: 0.71 us a step instead of 1.0; products alone, on what the
// registers hold, 0.72 and 0.54).  A tile's filling takes 2.4 us, its results 3.6.  With
// three buffers 128 x 128 has three blocks a CU: 852,640 x 128 x 256 to fp32 106 us (of
// two blocks 121), now in a graph of such calls 89 and between a layer's quantisers, which leave
// the caches full, 111; 852,640 x 256 x 128 156 (6.0 TB/s) and 161; 128 x 256 x 852,640 in 247 parts
// with their join 66 and 82 (its operands' rows are 426,320 bytes apart, so that in three of four
// rows every second step's 64 bytes lie in two lines; at 426,368, a multiple of 128, 55).  Results that read aux or c take longer,
// by 4 columns a lane: 852,640 x 128 x 256 with a ReLU's gradient 209 us (206 at the rate of a
// copy), 32,768 x 4096 x 4096 503.  Four waves of 128 x 128 took 355 us instead of 323, loads
// between the products 321.
template <int WM, int WN, int TM, int TN, int NB, bool PAST>
__global__ void __launch_bounds__(WM * WN * 64, TM * TN > 8 ? 1 : 2) k_matmul4_tile(Job4 J) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32, NWV = WM * WN, ROWS = BM + BN;
  constexpr int LA = BM / 16 / NWV, LB = BN / 16 / NWV, LS = (ROWS / 64 + NWV - 1) / NWV;  // loads of a wave and step
  constexpr int PER = LA + LB + LS;
  static_assert(BM % (16 * NWV) == 0 && BN % (16 * NWV) == 0, "as many loads for every wave");
  static_assert(BM % 64 == 0 && BN % 64 == 0, "a load of scales is of one operand");
  static_assert(PER * (NB - 2) < 63, "the counter of loads holds them");
  // arrays of their own, so that a read waits for the loads of its buffer and no others
  constexpr int BYTES = ROWS * 68;  // 64 of numbers for each row, then 4 of scales
  static_assert(NB == 3 || NB == 4, "buffers");
  __shared__ __align__(16) uint8_t b0[BYTES], b1[BYTES], b2[BYTES], b3[NB > 3 ? BYTES : 16];
  uint8_t* const bufs[4] = {b0, b1, b2, b3};
  const Matmul4& p = J.p;
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
  const int64_t kb0 = split * J.per, kb1 = min(kb0 + J.per, J.kb), steps = kb1 - kb0;
  const int64_t end = (p.a.cols + 31) / 32 * 16;  // bytes of a row

  // Loads: wave w takes 16 rows from 16 (i NWV + w) on, a lane 16 bytes of one: a scalar
  // base, which moves on by 64 bytes a step, and a 32-bit offset.  A row that is not there
  // is the last one again (its results are not stored).  Chunks behind the columns are the
  // last one again: their numbers, which are finite, count for nothing, since the scales
  // there are 2^-127 in both operands.
  const int lrow = l >> 2, lchunk = ((l & 3) ^ ((l >> 4) & 3)) * 16;
  const uint8_t *src[LA + LB], *ssrc[LS];
  uint32_t off[LA + LB], soff[LS];
  int64_t sstep[LS];
#pragma unroll
  for (int i = 0; i < LA + LB; ++i) {
    const bool isa = i < LA;
    const int64_t last = (isa ? p.a.rows : p.b.rows) - 1, ld = isa ? p.a.ld : p.b.ld;
    const int64_t row = min(isa ? m0 + (i * NWV + w) * 16 : n0 + ((i - LA) * NWV + w) * 16, last);
    src[i] = (isa ? p.a.q : p.b.q) + row * ld + kb0 * 64;
    off[i] = (uint32_t)min((int64_t)lrow, last - row) * (uint32_t)ld + lchunk;
  }
#pragma unroll
  for (int i = 0; i < LS; ++i) {
    const int at = (i * NWV + w) % (ROWS / 64) * 64;  // some twice, where the waves are more
    const bool isa = at < BM;
    const int64_t rows = isa ? p.a.rows : p.b.rows, row = min(isa ? m0 + at : n0 + at - BM, rows - 1);
    sstep[i] = rows * 4;
    ssrc[i] = (isa ? p.a.scale : p.b.scale) + (kb0 * rows + row) * 4;
    soff[i] = (uint32_t)min((int64_t)l, rows - 1 - row) * 4;
  }
  auto to_lds = [&](const uint8_t* from, uint8_t* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
  };
  auto to_lds4 = [&](const uint8_t* from, uint8_t* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)dst, 4, 0, 0);
  };
  int64_t left = end - kb0 * 64;  // bytes of a row from the next step on
  auto fetch = [&](uint8_t* buf) {  // the next step
    const uint32_t back = max(lchunk + 16 - (int)min(left, (int64_t)64), 0);
#pragma unroll
    for (int i = 0; i < LA + LB; ++i) {
      asm volatile("" : "+s"(src[i]));  // else the addresses of several steps are kept, and spill
      to_lds(src[i] + (off[i] - back), buf + (i < LA ? i * NWV + w : BM / 16 + (i - LA) * NWV + w) * 1024);
      src[i] += 64;
    }
#pragma unroll
    for (int i = 0; i < LS; ++i) {
      asm volatile("" : "+s"(ssrc[i]));
      to_lds4(ssrc[i] + soff[i], buf + ROWS * 64 + (i * NWV + w) % (ROWS / 64) * 256);
      ssrc[i] += sstep[i];
    }
    left -= 64;
  };
  f32x16 acc[TM][TN] = {};
  int at[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) at[s] = j * 64 + (((2 * s + h) ^ ((j >> 2) & 3)) * 16);
  struct Half {
    uint4 a[TM], b[TN];
  } f0, f1;
  struct Scales {
    uint32_t a[TM], b[TN];
  } sc[2];  // of even and odd steps
  auto read = [&](Half& f, const uint8_t* buf, int s) {
#pragma unroll
    for (int n = 0; n < TN; ++n) f.b[n] = *(const uint4*)(buf + (BM + (wn * TN + n) * 32) * 64 + at[s]);
#pragma unroll
    for (int m = 0; m < TM; ++m) f.a[m] = *(const uint4*)(buf + (wm * TM + m) * 2048 + at[s]);
  };
  auto read_scales = [&](Scales& x, const uint8_t* buf) {
    const uint32_t* scl = (const uint32_t*)(buf + ROWS * 64);
#pragma unroll
    for (int n = 0; n < TN; ++n) x.b[n] = scl[BM + (wn * TN + n) * 32 + j];
#pragma unroll
    for (int m = 0; m < TM; ++m) x.a[m] = scl[(wm * TM + m) * 32 + j];
  };
  auto of_half = [&](Scales& x) {  // bytes h and 2 + h, at places 0 and 2
#pragma unroll
    for (int n = 0; n < TN; ++n) x.b[n] >>= 8 * h;
#pragma unroll
    for (int m = 0; m < TM; ++m) x.a[m] >>= 8 * h;
  };
  auto products = [&](const Half& f, const Scales& x, auto sel) {
    // in this order, and no others between: moved about, sums get copies and spill
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
      for (int n = 0; n < TN; ++n)
        acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(f.b[n]), operand(f.a[m]), acc[m][n], kE2M1, kE2M1,
                                                                    decltype(sel)::value, (int)x.b[n], decltype(sel)::value,
                                                                    (int)x.a[m]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // waits for all loads but those of n steps
  auto arrived = [&](auto n) {
    constexpr int c = decltype(n)::value * PER;
    __builtin_amdgcn_s_waitcnt(0x0f70 | (c & 15) | ((c >> 4) << 14));
  };
  auto meet = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // step i, whose buffer is `mine`; the one before it had `old`, the next one has `next`
  // (full: NB - 1 steps and more follow, which the compiler's own waits go by)
  auto step = [&](auto full, int64_t i, const uint8_t* mine, uint8_t* old, const uint8_t* next, Scales& x, Scales& y) {
    constexpr bool F = decltype(full)::value;
    read(f1, mine, 1);
    if (F || i + NB - 1 < steps) fetch(old);
    of_half(x);
    products(f0, x, std::integral_constant<int, 0>());  // they go on while the wave waits
    if (F || i + NB - 1 < steps)
      arrived(std::integral_constant<int, NB - 2>());
    else
      arrived(std::integral_constant<int, 0>());
    meet();
    if (F || i + 1 < steps) {
      read(f0, next, 0);
      read_scales(y, next);
    }
    products(f1, x, std::integral_constant<int, 2>());
  };
  if (steps > 0) {
#pragma unroll
    for (int u = 0; u < NB - 1; ++u)
      if (u < steps) fetch(bufs[u]);
    if (steps >= NB - 1)
      arrived(std::integral_constant<int, NB - 2>());
    else
      arrived(std::integral_constant<int, 0>());
    meet();
    read(f0, b0, 0);
    read_scales(sc[0], b0);
    int64_t i = 0;
    constexpr int UN = NB % 2 ? 2 * NB : NB;  // steps after which buffers and scales are the same again
    for (; i + UN + NB - 1 <= steps; i += UN) {
#pragma unroll
      for (int u = 0; u < UN; ++u)
        step(std::true_type(), i + u, bufs[u % NB], bufs[(u + NB - 1) % NB], bufs[(u + 1) % NB], sc[u & 1], sc[(u + 1) & 1]);
    }
    for (; i < steps; i += UN) {
#pragma unroll
      for (int u = 0; u < UN; ++u)
        if (i + u < steps)
          step(std::false_type(), i + u, bufs[u % NB], bufs[(u + NB - 1) % NB], bufs[(u + 1) % NB], sc[u & 1], sc[(u + 1) & 1]);
    }
  }
  __syncthreads();  // every wave has read its last operands
  // The results go through the wave's own piece of LDS to be stored as whole rows, a
  // bf16 c as bf16 and all at once.
  constexpr int PIECE = TM * TN * 2048;
  static_assert(NB * (BYTES / PIECE) >= NWV, "a piece for each wave");
  const int of = w / (BYTES / PIECE);
  uint8_t* const piece = (of == 0 ? b0 : of == 1 ? b1 : of == 2 ? b2 : b3) + w % (BYTES / PIECE) * PIECE;
  const int64_t mw = m0 + wm * TM * 32, nw = n0 + wn * TN * 32;
  const bool raw = J.splits > 1, plain = raw || (p.ep.act != MGN_ACT_RELU_GRAD && !p.ep.accumulate);
  if (plain && !raw) {
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int64_t col = nw + n * 32 + 8 * g + 4 * h;
        f32x4 bias = {0.f, 0.f, 0.f, 0.f};
        if (p.ep.bias != nullptr) bias = load4(p.ep.bias + col, (int)min(max(p.b.rows - col, (int64_t)0), (int64_t)4));
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = p.ep.bias != nullptr ? acc[m][n][4 * g + e] + bias[e] : acc[m][n][4 * g + e];
            acc[m][n][4 * g + e] = p.ep.act == MGN_ACT_RELU && v < 0.f ? 0.f : v;  // a NaN stays
          }
      }
  }
  if (plain && !raw && p.c_type == MGN_BF16) {
    // rows of TN * 4 chunks of 8 columns, chunk c at place c ^ row
    constexpr int CH = TN * 4;
    static_assert(TM * 32 * CH * 16 <= PIECE, "the wave's results fit");
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const bf16 v[4] = {(bf16)acc[m][n][4 * g], (bf16)acc[m][n][4 * g + 1], (bf16)acc[m][n][4 * g + 2],
                             (bf16)acc[m][n][4 * g + 3]};
          __builtin_memcpy(piece + (m * 32 + j) * CH * 16 + ((n * 4 + g) ^ (j & (CH - 1))) * 16 + 8 * h, v, 8);
        }
    wave_lds_sync();
    const int c = l % CH;
    const int64_t n = nw + c * 8;
    bf16* to = (bf16*)p.c + mw * p.ldc + n;
#pragma unroll
    for (int i = 0; i < TM * 32; i += 64 / CH) {
      const int r = i + l / CH;
      const uint4 v = *(const uint4*)(piece + r * CH * 16 + (c ^ (r & (CH - 1))) * 16);
      if (mw + r < p.a.rows) {
        if (n + 8 <= p.b.rows) {
          store16<PAST>(to + r * p.ldc, v);
        } else {
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (n + e < p.b.rows) to[r * p.ldc + e] = __builtin_bit_cast(bf16, (uint16_t)(u[e >> 1] >> (16 * (e & 1))));
        }
      }
    }
    return;
  }
  // rows of TN * 8 chunks of 4 columns, chunk c at place c ^ row, MR times 32 of them at a time
  constexpr int CH = TN * 8, MR = PIECE / (32 * CH * 16) < TM ? PIECE / (32 * CH * 16) : TM;
  static_assert(MR >= 1 && TM % MR == 0, "whole rounds");
  f32x4* const mine = (f32x4*)piece;
  float* const out = raw ? p.part + (int64_t)split * p.a.rows * p.b.rows : (float*)p.c;
  const int64_t ldo = raw ? p.b.rows : p.ldc;
#pragma unroll
  for (int m = 0; m < TM; m += MR) {
#pragma unroll
    for (int q = 0; q < MR; ++q)
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x16& v = acc[m + q][n];
          mine[(q * 32 + j) * CH + ((n * 8 + 2 * g + h) ^ (j & (CH - 1)))] =
              f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
        }
    wave_lds_sync();
    const int c = l % CH;
    const int64_t n = nw + c * 4;
    const int k = (int)min(p.b.rows - n, (int64_t)4);
    if (plain) {
#pragma unroll
      for (int i = 0; i < MR * 32; i += 64 / CH) {
        const int r = i + l / CH;
        const int64_t row = mw + m * 32 + r;
        const f32x4 v = mine[r * CH + (c ^ (r & (CH - 1)))];
        if (row < p.a.rows && k > 0) {
          if (k == 4)
            store16<PAST>(out + row * ldo + n, __builtin_bit_cast(uint4, v));
          else
            store4(out + row * ldo + n, v, k);
        }
      }
    } else {
#pragma unroll 2
      for (int i = 0; i < MR * 32; i += 64 / CH) {
        const int r = i + l / CH;
        const int64_t row = mw + m * 32 + r;
        const f32x4 v = mine[r * CH + (c ^ (r & (CH - 1)))];
        if (row < p.a.rows && k > 0) finish(p, row, n, v);
      }
    }
    wave_lds_sync();
  }
}

// ---- few rows of a (up to TM times 16), bound by the weights' bytes.
//
// A block takes TN times 16 rows of b, its 8 waves the steps of 256 columns in turn;
// operands come straight from memory, 16 bytes a lane (four lanes cover a row's 128
// columns, two loads its 128-byte line), a step ahead, and the waves' sums meet in LDS.
// Measured, in a graph of such calls: 1 x 4096 x 4096 4.6 us, 21 x 9001 x 6000 10.0 (188 blocks;
// 2.9 TB/s of weights that the last-level cache holds), 32 x 14,336 x 4096 10.8; through the
// binding 9.7 and under the profiler 10.5 for the second.
template <int TM, int TN>
__global__ void __launch_bounds__(512) k_matmul4_few(Job4 J) {
  constexpr int NWV = 8;
  __shared__ f32x4 sums[NWV][TM * TN][64];
  const Matmul4& p = J.p;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, j = l & 15, q = l >> 4;
  const int64_t n0 = (blockIdx.y * kGridRow + blockIdx.x) * (16 * TN);
  const int split = blockIdx.z;
  const int64_t kb0 = split * J.per, kb1 = min(kb0 + J.per, J.kb);
  const int64_t end = (p.a.cols + 31) / 32 * 16 - q * 16;
  const uint8_t *rb[TN], *sb[TN], *ra[TM], *sa[TM];
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    const int64_t n = min(n0 + i * 16 + j, p.b.rows - 1);
    rb[i] = p.b.q + n * p.b.ld + q * 16;
    sb[i] = p.b.scale + n * 4 + q;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = min((int64_t)i * 16 + j, p.a.rows - 1);
    ra[i] = p.a.q + m * p.a.ld + q * 16;
    sa[i] = p.a.scale + m * 4 + q;
  }
  struct Step {
    uint4 a[2][TM], b[2][TN];
    uint32_t sa[2][TM], sb[2][TN];
  };
  auto fetch = [&](Step& x, int64_t kb) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      // of a step that is another split's, or behind the last, b's scales are 2^-127 and the
      // numbers zero
      const int64_t at = min(kb + u, J.kb - 1), k = (kb + u) * 64;
      const bool in = kb + u < kb1 && k < end;
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        x.b[u][i] = *(const uint4*)(in ? rb[i] + k : (const uint8_t*)&zero16);
        x.sb[u][i] = sb[i][at * p.b.rows * 4];
        if (kb + u >= kb1) x.sb[u][i] = 0;
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        x.a[u][i] = *(const uint4*)(in ? ra[i] + k : (const uint8_t*)&zero16);
        x.sa[u][i] = sa[i][at * p.a.rows * 4];
        if (kb + u >= kb1) x.sa[u][i] = 0;
      }
    }
  };
  f32x4 acc[TM][TN] = {};
  auto products = [&](const Step& x) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int n = 0; n < TN; ++n)
          acc[i][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(x.b[u][n]), operand(x.a[u][i]), acc[i][n], kE2M1,
                                                                       kE2M1, 0, (int)x.sb[u][n], 0, (int)x.sa[u][i]);
  };
  if (kb0 + 2 * w < kb1) {
    Step x, y;
    fetch(x, kb0 + 2 * w);
    for (int64_t kb = kb0 + 2 * w; kb < kb1; kb += 4 * NWV) {
      const bool more = kb + 2 * NWV < kb1;
      if (more) fetch(y, kb + 2 * NWV);
      products(x);
      if (more) {
        if (kb + 4 * NWV < kb1) fetch(x, kb + 4 * NWV);
        products(y);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int n = 0; n < TN; ++n) sums[w][i * TN + n][l] = acc[i][n];
  __syncthreads();
  if (w < TM * TN) {
    f32x4 v = sums[0][w][l];
#pragma unroll
    for (int k = 1; k < NWV; ++k) v += sums[k][w][l];
    const int64_t m = w / TN * 16 + j, n = n0 + w % TN * 16 + 4 * q;
    if (m < p.a.rows && n < p.b.rows) put4(J, split, m, n, v);
  }
}

}  // namespace dev

using namespace dev;

namespace {

constexpr int64_t kCUs = 256, kFewRows = 64;

enum { kFew, kSmallTile, kBigTile };
struct Plan {
  int kind;
  int64_t mt, nt, per;
  int splits;
  int tn;  // times 16 rows of b (few rows)
};

// Which kernel, and into how many parts the sums are split: the least of what these
// take by a model of their times (us), fitted to calls in a graph.  A tile's times have no
// bytes in them: where memory bounds a call they are too short, which leaves the choice as it is
// for many rows (852,640 x 128 x 256 57 expected, 89 measured; 852,640 x 256 x 128 93, 156; 128 x
// 256 x 852,640 42, 66), and for a few rows takes tiles of wide and long weights (1 x 65,536 x 4096 25,
// 34, which is 4 TB/s).
//  * few rows: 3 and what all blocks read (their rows of b, and a each) at 6.2 TB/s
//    (1 x 4096 x 4096 4.2, 32 x 4096 x 4096 6.4, 64 x 4096 x 4096 8.8, tiles 12.5; 21 x
//    9001 x 6000 with 16, 32, 48 and 64 rows of b a block 12.9, 13.3, 9.5, 10.9; 64 x 8192
//    x 8192 with 32 17.4, tiles 16.7);
//  * tiles of 128 x 128: 1.4 a tile of a CU and 0.31 a step and tile where all CUs have
//    two or more, else 0.34 to 0.54 a step (2048 x 2048 x 2048 11.9, of 256 x 256 17.9);
//    sums split into s parts add a launch and 8 s bytes a result (512 x 512 x 20,000 whole
//    67, in 4, 8 and 32 parts 21.8, 17.5, 26.6);
//  * tiles of 256 x 256: 7 and 0.98 a step for every 256 of them (4096 x 4096 x 4096 42,
//    of 128 x 128 51; 32,768 x 4096 x 1024 144, 125).
Plan plan(int64_t m, int64_t n, int64_t k) {
  const int64_t kb = ceil_div(k, 128), m1 = ceil_div(m, 128), n1 = ceil_div(n, 128), m2 = ceil_div(m, 256),
                n2 = ceil_div(n, 256);
  Plan r = {kSmallTile, m1, n1, 0, 1, 0};
  double best = 1e30;
  for (int64_t s = 1; s <= 512 && (s == 1 || 2 * s <= kb); s *= 2) {
    const double blocks = (double)m1 * n1 * s, rounds = std::ceil(blocks / kCUs);
    const double step = blocks <= kCUs ? 0.34 * std::max(1.0, blocks / 160) : 0.31 * rounds;
    const double t = 2.5 + 1.4 * rounds + step * ceil_div(kb, s) + (s > 1 ? 3.5 + 8e-6 / 4 * s * m * n : 0.0);
    if (t < best) {
      best = t;
      r.splits = (int)s;
    }
  }
  const double big = (7 + 0.98 * kb) * std::ceil((double)m2 * n2 / kCUs);
  if (big < best) {
    best = big;
    r = {kBigTile, m2, n2, 0, 1, 0};
  }
  if (m <= kFewRows) {
    // as many rows of b a block as leave it a CU of its own, up to what registers and LDS hold.
    // For up to 16 rows of a and over 16,384 of b up to 32: 1 x 20,000 x 4096 11.4 us, with 64
    // 14.6; 16 x 32,768 x 1024 8.1, 8.6; 16 x 65,536 x 1024 10.7, 15.0; but 1 x 32,768 x 4096 21, 17.0.
    const int64_t rows = m <= 16 ? 16 : m <= 32 ? 32 : 64, most = rows == 64 || (rows == 16 && n > 4 * 16 * kCUs) ? 2 : 4;
    const int64_t tn = std::min(ceil_div(ceil_div(n, 16), kCUs), most), nt = ceil_div(n, 16 * tn);
    if (3 + (double)nt * (rows + 16 * tn) * k / 2 / 6.2e6 < best)
      r = {kFew, 1, nt, 0, (int)std::max<int64_t>(std::min(kCUs / nt, kb / 32), 1), (int)tn};
  }
  r.per = std::max<int64_t>(ceil_div(kb, r.splits), 1);
  r.splits = (int)std::max<int64_t>(ceil_div(kb, r.per), 1);
  return r;
}

template <int TM>
void launch_few(const Job4& J, int tn, dim3 g, hipStream_t s) {
  if (tn == 1)
    hipLaunchKernelGGL((k_matmul4_few<TM, 1>), g, dim3(512), 0, s, J);
  else if (tn == 2)
    hipLaunchKernelGGL((k_matmul4_few<TM, 2>), g, dim3(512), 0, s, J);
  else if constexpr (TM <= 2) {
    if (tn == 3)
      hipLaunchKernelGGL((k_matmul4_few<TM, 3>), g, dim3(512), 0, s, J);
    else
      hipLaunchKernelGGL((k_matmul4_few<TM, 4>), g, dim3(512), 0, s, J);
  }
}

}  // namespace

size_t matmul4_workspace(int64_t m, int64_t n, int64_t k) {
  if (m <= 0 || n <= 0) return 0;
  const int splits = plan(m, n, k).splits;
  return splits > 1 ? (size_t)splits * (size_t)m * (size_t)n * 4 : 0;
}

hipError_t launch_matmul4(const Matmul4& p, hipStream_t s) {
  const Plan r = plan(p.a.rows, p.b.rows, p.a.cols);
  const Job4 J = {p, r.mt, r.nt, ceil_div(p.a.cols, 128), r.per, r.splits};
  const dim3 grid((unsigned)(8 * ceil_div(r.mt * r.nt * r.splits, 8)));
  const uintptr_t rows = r.splits > 1 ? (uintptr_t)p.b.rows * 4 : (uintptr_t)p.c | (uintptr_t)(p.ldc * (p.c_type == MGN_BF16 ? 2 : 4));
  const bool past = rows % 16 == 0;
  if (r.kind == kFew) {
    dim3 g = grid_of(r.nt);
    g.z = (unsigned)r.splits;
    if (p.a.rows <= 16)
      launch_few<1>(J, r.tn, g, s);
    else if (p.a.rows <= 32)
      launch_few<2>(J, r.tn, g, s);
    else
      launch_few<4>(J, r.tn, g, s);
  } else if (r.kind == kBigTile) {
    if (past)
      hipLaunchKernelGGL((k_matmul4_tile<2, 4, 4, 2, 4, true>), grid, dim3(512), 0, s, J);
    else
      hipLaunchKernelGGL((k_matmul4_tile<2, 4, 4, 2, 4, false>), grid, dim3(512), 0, s, J);
  } else if (past) {
    hipLaunchKernelGGL((k_matmul4_tile<2, 2, 2, 2, 3, true>), grid, dim3(256), 0, s, J);
  } else {
    hipLaunchKernelGGL((k_matmul4_tile<2, 2, 2, 2, 3, false>), grid, dim3(256), 0, s, J);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || r.splits == 1) return e;
  const int64_t quads = p.a.rows * ceil_div(p.b.rows, 4);
  if (r.splits >= 16)
    hipLaunchKernelGGL((k_product_join<16, Job4>), dim3((unsigned)ceil_div(quads, 16)), dim3(256), 0, s, J);
  else
    hipLaunchKernelGGL((k_product_join<1, Job4>), dim3((unsigned)ceil_div(quads, 256)), dim3(256), 0, s, J);
  return hipGetLastError();
}

}  // namespace mgn
