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

// ---- tiles: BM x BN of c a block of WM x WN waves, each TM x TN times 32 x 32.
//
// Steps of 128 columns (64 bytes of a row) go through four LDS buffers by loads that
// write LDS themselves, three steps ahead, the rows' scales (4 bytes a row and step)
// with them.  A row's 16-byte chunk c sits at place c ^ (row / 4 % 4), so that 16
// rows of a fragment read cover all 64 banks; the lanes' source addresses are permuted
// to match.  A step has two halves of 64 columns, and a half's fragments are read under
// the products of the half before it.  The barrier of a step lies between its halves: there
// a wave has read all of the step, whose buffer may be filled again, and waited for its own
// loads of the next one.
template <int WM, int WN, int TM, int TN, int OCC>
__global__ void __launch_bounds__(WM * WN * 64, OCC) k_matmul4_tile(Job4 J) {
  constexpr int NB = 4;
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32, NWV = WM * WN, ROWS = BM + BN;
  constexpr int LA = BM / 16 / NWV, LB = BN / 16 / NWV, LS = ROWS / 64 / NWV;  // loads of a wave and step
  constexpr int PER = LA + LB + LS;
  static_assert(BM % (16 * NWV) == 0 && BN % (16 * NWV) == 0 && ROWS % (64 * NWV) == 0, "as many loads for every wave");
  static_assert(BM % 64 == 0, "a load of scales is of one operand");
  static_assert(PER * (NB - 2) < 63, "the counter of loads holds them");
  constexpr int CH = TN * 8;  // chunks of 4 columns of a wave's results
  static_assert(ROWS * 64 >= NWV * 32 * CH * 16 / 2, "results fit two buffers");
  // arrays of their own, so that a read waits for the loads of its buffer and no others
  constexpr int BYTES = ROWS * 68;  // 64 of numbers for each row, then 4 of scales
  __shared__ __align__(16) uint8_t b0[BYTES], b1[BYTES], b2[BYTES], b3[BYTES];
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

  // Loads: wave w takes 16 rows from 16 (i NWV + w) on, a lane 16 bytes of one, at an
  // address that moves on by 64 bytes a step.  A row that is not there is the last one
  // again (its results are not stored).  Chunks behind the columns are the last one
  // again: their numbers, which are finite, count for nothing, since the scales there
  // are 2^-127 in both operands.
  const int lrow = l >> 2, lchunk = ((l & 3) ^ ((l >> 4) & 3)) * 16;
  const uint8_t *src[LA + LB], *ssrc[LS];
#pragma unroll
  for (int i = 0; i < LA + LB; ++i) {
    const int row = (i < LA ? i * NWV + w : (i - LA) * NWV + w) * 16 + lrow;
    src[i] = (i < LA ? p.a.q + min(m0 + row, p.a.rows - 1) * p.a.ld : p.b.q + min(n0 + row, p.b.rows - 1) * p.b.ld) +
             kb0 * 64 + lchunk;
  }
  int64_t sstep[LS];
#pragma unroll
  for (int i = 0; i < LS; ++i) {
    const int row = (i * NWV + w) * 64;
    const bool isa = row < BM;
    const int64_t rows = isa ? p.a.rows : p.b.rows, r = min((isa ? m0 + row : n0 + row - BM) + l, rows - 1);
    sstep[i] = rows * 4;
    ssrc[i] = (isa ? p.a.scale : p.b.scale) + (kb0 * rows + r) * 4;
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
    const int back = max(lchunk + 16 - (int)min(left, (int64_t)64), 0);
#pragma unroll
    for (int i = 0; i < LA + LB; ++i) {
      to_lds(src[i] - back, buf + (i < LA ? i * NWV + w : BM / 16 + (i - LA) * NWV + w) * 1024);
      src[i] += 64;
    }
#pragma unroll
    for (int i = 0; i < LS; ++i) {
      to_lds4(ssrc[i], buf + ROWS * 64 + (i * NWV + w) * 256);
      ssrc[i] += sstep[i];
    }
    left -= 64;
  };
  f32x16 acc[TM][TN] = {};
  int off[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) off[s] = j * 64 + (((2 * s + h) ^ ((j >> 2) & 3)) * 16);
  struct Half {
    uint4 a[TM], b[TN];
  } f0, f1;
  struct Scales {
    uint32_t a[TM], b[TN];
  } s0, s1;  // of even and odd steps
  auto read = [&](Half& f, const uint8_t* buf, int s) {
#pragma unroll
    for (int n = 0; n < TN; ++n) f.b[n] = *(const uint4*)(buf + (BM + (wn * TN + n) * 32) * 64 + off[s]);
#pragma unroll
    for (int m = 0; m < TM; ++m) f.a[m] = *(const uint4*)(buf + (wm * TM + m) * 2048 + off[s]);
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
    fetch(b0);
    if (steps > 1) fetch(b1);
    if (steps > 2) fetch(b2);
    if (steps > 2)
      arrived(std::integral_constant<int, NB - 2>());
    else
      arrived(std::integral_constant<int, 0>());
    meet();
    read(f0, b0, 0);
    read_scales(s0, b0);
    int64_t i = 0;
    for (; i + 2 * NB - 1 <= steps; i += NB) {
      step(std::true_type(), i, b0, b3, b1, s0, s1);
      step(std::true_type(), i + 1, b1, b0, b2, s1, s0);
      step(std::true_type(), i + 2, b2, b1, b3, s0, s1);
      step(std::true_type(), i + 3, b3, b2, b0, s1, s0);
    }
    for (; i < steps; i += NB) {
      step(std::false_type(), i, b0, b3, b1, s0, s1);
      if (i + 1 < steps) step(std::false_type(), i + 1, b1, b0, b2, s1, s0);
      if (i + 2 < steps) step(std::false_type(), i + 2, b2, b1, b3, s0, s1);
      if (i + 3 < steps) step(std::false_type(), i + 3, b3, b2, b0, s1, s0);
    }
  }
  __syncthreads();  // every wave has read its last operands
  // rows of CH chunks of 4 columns, chunk c at place c ^ row
  f32x4* mine = (f32x4*)(w < NWV / 2 ? b0 : b1) + w % (NWV / 2) * 32 * CH;
#pragma unroll
  for (int m = 0; m < TM; ++m) {
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        mine[j * CH + ((n * 8 + 2 * g + h) ^ (j & (CH - 1)))] =
            f32x4{acc[m][n][4 * g], acc[m][n][4 * g + 1], acc[m][n][4 * g + 2], acc[m][n][4 * g + 3]};
    wave_lds_sync();
    constexpr int LPR = CH / 2;  // lanes of a row
    const int c = l % LPR * 2;
    const int64_t n = n0 + wn * TN * 32 + c * 4;
#pragma unroll 2
    for (int i = 0; i < 32; i += 64 / LPR) {
      const int r = i + l / LPR;
      const int64_t row = m0 + (wm * TM + m) * 32 + r;
      const f32x4 v = mine[r * CH + (c ^ (r & (CH - 1)))], u = mine[r * CH + ((c + 1) ^ (r & (CH - 1)))];
      if (row < p.a.rows && n < p.b.rows) put8(J, split, row, n, v, u);
    }
    wave_lds_sync();
  }
}

// ---- few rows of a (up to TM times 16), bound by the weights' bytes.
//
// A block takes 16 rows of b, its 8 waves the steps of 256 columns in turn; operands
// come straight from memory, 16 bytes a lane (four lanes cover a row's 128 columns,
// two loads its 128-byte line), a step ahead, and the waves' sums meet in LDS.
template <int TM>
__global__ void __launch_bounds__(512) k_matmul4_few(Job4 J) {
  constexpr int NWV = 8;
  __shared__ f32x4 sums[NWV][TM][64];
  const Matmul4& p = J.p;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, j = l & 15, q = l >> 4;
  const int64_t n0 = (blockIdx.y * kGridRow + blockIdx.x) * 16;
  const int split = blockIdx.z;
  const int64_t kb0 = split * J.per, kb1 = min(kb0 + J.per, J.kb);
  const int64_t end = (p.a.cols + 31) / 32 * 16 - q * 16;
  const int64_t nj = min(n0 + j, p.b.rows - 1);
  const uint8_t *rb = p.b.q + nj * p.b.ld + q * 16, *sb = p.b.scale + nj * 4 + q;
  const uint8_t *ra[TM], *sa[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = min((int64_t)i * 16 + j, p.a.rows - 1);
    ra[i] = p.a.q + m * p.a.ld + q * 16;
    sa[i] = p.a.scale + m * 4 + q;
  }
  struct Step {
    uint4 a[2][TM], b[2];
    uint32_t sa[2][TM], sb[2];
  };
  auto fetch = [&](Step& x, int64_t kb) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t at = min(kb + u, J.kb - 1), k = (kb + u) * 64;
      const bool in = kb + u < kb1 && k < end;
      x.b[u] = *(const uint4*)(in ? rb + k : (const uint8_t*)&zero16);
      x.sb[u] = sb[at * p.b.rows * 4];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        x.a[u][i] = *(const uint4*)(in ? ra[i] + k : (const uint8_t*)&zero16);
        x.sa[u][i] = sa[i][at * p.a.rows * 4];
      }
      // of a step that is another split's the scales count for nothing
      if (kb + u >= kb1) x.sb[u] = 0;
    }
  };
  f32x4 acc[TM] = {};
  auto products = [&](const Step& x) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < TM; ++i)
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(x.b[u]), operand(x.a[u][i]), acc[i], kE2M1, kE2M1, 0,
                                                                  (int)x.sb[u], 0, (int)x.sa[u][i]);
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

constexpr int64_t kFewRows = 32;
Plan plan(int64_t m, int64_t n, int64_t k) {
  Plan r;
  const int64_t kb = ceil_div(k, 128);
  int64_t want;
  if (m <= kFewRows) {
    r.kind = kFew;
    r.mt = 1;
    r.nt = ceil_div(n, 16);
    want = std::min(kCUs / std::max<int64_t>(r.nt, 1), kb / 32);
  } else {
    const int64_t m2 = ceil_div(m, 256), n2 = ceil_div(n, 256), m1 = ceil_div(m, 128), n1 = ceil_div(n, 128);
    const bool big = m2 * n2 >= kCUs * 3 / 4 && kb >= 8 && 4 * m2 * n2 * 7 <= m1 * n1 * 8;
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
  if (r.kind == kFew) {
    dim3 g = grid_of(r.nt);
    g.z = (unsigned)r.splits;
    if (p.a.rows <= 16)
      hipLaunchKernelGGL((k_matmul4_few<1>), g, dim3(512), 0, s, J);
    else
      hipLaunchKernelGGL((k_matmul4_few<2>), g, dim3(512), 0, s, J);
  } else if (r.kind == kBigTile) {
    hipLaunchKernelGGL((k_matmul4_tile<2, 4, 4, 2, 2>), grid, dim3(512), 0, s, J);
  } else {
    hipLaunchKernelGGL((k_matmul4_tile<2, 2, 2, 2, 2>), grid, dim3(256), 0, s, J);
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
