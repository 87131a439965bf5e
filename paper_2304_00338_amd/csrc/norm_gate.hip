// The step between two blocks of a residual stream: norm after the block,
// gate, residual, norm before the next block, in one pass over the rows, and
// its reverse with the gradients of the vectors (see include/mgn.h).
//
// A row is held by a walker: 16, 32 or 64 lanes of a wave, or a whole block
// of 2 to 16 waves, each lane with one or two runs of 8 consecutive columns.
// So a row is read once and its statistics (two passes: mean, then squared
// deviations) come from registers, all in fp32.  A walker takes consecutive
// rows, keeps gamma, beta and the gate in registers and, in the reverse, the
// column sums of the vectors' gradients; a block's sums are added over its
// walkers, and the blocks' in a second launch, always in the same order.
#include "dev_common.hpp"
#include "row_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

// Sums over the lanes of a walker.  LPR 0: the walker is the block.
template <int LPR>
struct Reduce {
  float* buf;  // LPR 0: [2][16][2] in LDS
  int flip = 0;
  __device__ __forceinline__ void sum2(float& a, float& b) {
    a = sum16(a);
    b = sum16(b);
    if constexpr (LPR == 32) {
      a = pair16(a);
      b = pair16(b);
    } else if constexpr (LPR == 64 || LPR == 0) {
      a = sum_q(a);
      b = sum_q(b);
    }
    if constexpr (LPR == 0) {
      // one barrier a sum: the next one goes through the other half, and a
      // half is written again only after a barrier that follows its reads
      float* p = buf + flip * 32;
      flip ^= 1;
      const int w = threadIdx.x >> 6, n = blockDim.x >> 6;
      if ((threadIdx.x & 63) == 0) {
        p[2 * w] = a;
        p[2 * w + 1] = b;
      }
      __syncthreads();
      a = p[0];
      b = p[1];
      for (int i = 1; i < n; ++i) {
        a += p[2 * i];
        b += p[2 * i + 1];
      }
    }
  }
  __device__ __forceinline__ float sum(float a) {
    float b = 0.f;
    sum2(a, b);
    return a;
  }
  static __device__ __forceinline__ float pair16(float s) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
};

// The walker's place: its lane, rows and columns.
template <int LPR, int NV>
struct Place {
  int lane, lanes;
  int64_t walker, r0, r1;
  int n[NV];  // columns of each run that are inside the row
  __device__ __forceinline__ Place(int64_t rows, int cols, int64_t per) {
    lanes = LPR ? LPR : blockDim.x;
    lane = LPR ? threadIdx.x & (LPR - 1) : threadIdx.x;
    walker = LPR ? (int64_t)blockIdx.x * (blockDim.x / LPR) + threadIdx.x / LPR : blockIdx.x;
    r0 = min(walker * per, rows);
    r1 = min(r0 + per, rows);
#pragma unroll
    for (int k = 0; k < NV; ++k) n[k] = cols - col(k);
  }
  __device__ __forceinline__ int col(int k) const { return (k * lanes + lane) * 8; }
};

template <int NV>
__device__ __forceinline__ void load_vec(float (&v)[NV][8], const float* p, const int (&col)[NV], const int (&n)[NV],
                                         float other) {
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[k][e] = p != nullptr ? (e < n[k] ? p[col[k] + e] : 0.f) : other;
}

// The gate group of a row: the largest g with ptr[g] <= r (0 if there is none).
__device__ __forceinline__ int64_t find_group(const int32_t* ptr, int64_t n, int64_t r) {
  int64_t lo = 0, hi = n - 1;
  while (lo < hi) {
    const int64_t m = (lo + hi + 1) >> 1;
    if (ptr[m] <= r)
      lo = m;
    else
      hi = m - 1;
  }
  return lo;
}

// What a norm makes of a row: mean and 1 / sqrt(variance + eps).
template <int LPR, int NV>
__device__ __forceinline__ void statistics(const float (&v)[NV][8], const int (&n)[NV], int kind, float inv, float eps,
                                           Reduce<LPR>& red, float& mean, float& rstd) {
  mean = 0.f;
  if (kind == MGN_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[k][e];  // 0 beyond the row
    mean = red.sum(s) * inv;
  }
  float q = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = e < n[k] ? v[k][e] - mean : 0.f;
      q = __builtin_fmaf(d, d, q);
    }
  rstd = 1.f / __builtin_sqrtf(__builtin_fmaf(red.sum(q), inv, eps));
}

template <typename XT, typename BT, int LPR, int NV>
__global__ void __launch_bounds__(LPR ? 256 : 1024) k_norm_gate_fwd(NormGate a) {
  __shared__ float buf[64];
  const mgn_norm_gate& op = a.op;
  const Place<LPR, NV> at(op.rows, op.cols, a.per);
  Reduce<LPR> red{buf};
  const float inv = 1.f / (float)op.cols;
  int col[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) col[k] = at.col(k);
  float pg[NV][8], pb[NV][8], qg[NV][8], qb[NV][8], gate[NV][8];
  load_vec(pg, op.post_gamma, col, at.n, 1.f);
  load_vec(pb, op.post_beta, col, at.n, 0.f);
  load_vec(qg, op.pre_gamma, col, at.n, 1.f);
  load_vec(qb, op.pre_beta, col, at.n, 0.f);
  load_vec(gate, a.gmode == kGateOne ? op.gate : nullptr, col, at.n, 1.f);
  const int64_t last = op.rows - 1;
  int64_t g = a.gmode == kGateGroup ? find_group(op.gate_ptr, op.n_gates, at.r0) : 0, held = -1;
  Raw8<XT> nx[NV];
  Raw8<BT> nb[NV];
  auto fetch = [&](int64_t r) {
    const int64_t rr = min(r, last);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      nx[k] = load8((const XT*)a.x.data + rr * a.x.ld + col[k], at.n[k]);
      nb[k] = load8((const BT*)a.b.data + rr * a.b.ld + col[k], at.n[k]);
    }
  };
  fetch(at.r0);
  // every walker of a wave or block takes as many turns: the sums cross lanes
  for (int64_t i = 0; i < a.per; ++i) {
    const int64_t r = at.r0 + i;
    bool mine = r < at.r1;
    float x[NV][8], b[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[k][e] = nx[k].get(e);
        b[k][e] = nb[k].get(e);
      }
    if (i + 1 < a.per) fetch(r + 1);
    if (a.gmode == kGateGroup && mine) {
      while (g + 1 < op.n_gates && r >= op.gate_ptr[g + 1]) ++g;
      mine = r >= op.gate_ptr[g] && r < op.gate_ptr[g + 1];
      if (mine && g != held) {
        load_vec(gate, op.gate + g * op.cols, col, at.n, 1.f);
        held = g;
      }
    }
    if (a.gmode == kGateRow && mine) load_vec(gate, op.gate + r * op.cols, col, at.n, 1.f);
    float pm = 0.f, pr = 1.f, qm = 0.f, qr = 1.f;
    if (op.post != MGN_NORM_NONE) {
      statistics(b, at.n, op.post, inv, op.eps, red, pm, pr);
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) b[k][e] = __builtin_fmaf((b[k][e] - pm) * pr, pg[k][e], pb[k][e]);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[k][e] = e < at.n[k] ? __builtin_fmaf(op.scale, gate[k][e] * b[k][e], op.skip * x[k][e]) : 0.f;
      if (mine) store8((XT*)a.y.data + r * a.y.ld + col[k], at.n[k], x[k]);
    }
    if (op.pre != MGN_NORM_NONE) {
      statistics(x, at.n, op.pre, inv, op.eps, red, qm, qr);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] = __builtin_fmaf((x[k][e] - qm) * qr, qg[k][e], qb[k][e]);
        if (mine) store8((BT*)a.z.data + r * a.z.ld + col[k], at.n[k], x[k]);
      }
    }
    if (a.stats != nullptr && mine && at.lane == 0) ((float4*)a.stats)[r] = float4{pm, pr, qm, qr};
  }
}

// Reverse.  With t = dy + pre'(dz), dp = scale gate t:
//   dx = skip t, db = post'(dp), dgate = sum of scale p t, and the gammas' and
//   betas' sums; norm'(d) = rstd (u - mean(u) - vhat mean(u vhat)), u = gamma d
//   (RMS: without mean(u)).  y is formed again from x and b, unrounded, and
// with the forward's statistics no sum precedes those of the gradients.
template <typename XT, typename BT, int LPR, int NV>
__global__ void __launch_bounds__(LPR ? 256 : 1024) k_norm_gate_bwd(NormGate a) {
  __shared__ float buf[64];
  extern __shared__ float sums[];  // LPR: [walkers of the block][cols]
  const mgn_norm_gate& op = a.op;
  const Place<LPR, NV> at(op.rows, op.cols, a.per);
  Reduce<LPR> red{buf};
  const float inv = 1.f / (float)op.cols;
  int col[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) col[k] = at.col(k);
  float pg[NV][8], pb[NV][8], qg[NV][8], gate[NV][8];
  load_vec(pg, op.post_gamma, col, at.n, 1.f);
  load_vec(pb, op.post_beta, col, at.n, 0.f);
  load_vec(qg, op.pre_gamma, col, at.n, 1.f);
  load_vec(gate, a.gmode == kGateOne ? op.gate : nullptr, col, at.n, 1.f);
  float dpg[NV][8] = {}, dpb[NV][8] = {}, dqg[NV][8] = {}, dqb[NV][8] = {}, dg[NV][8] = {};
  const int64_t last = op.rows - 1;
  int64_t g = a.gmode == kGateGroup ? find_group(op.gate_ptr, op.n_gates, at.r0) : 0, held = -1;
  // the gate's sums of a group that ends here: into dgate if all its rows are
  // this walker's, else into one of its two slots (first: the group began
  // before its rows)
  auto flush = [&]() {
    if (held < 0) return;
    if (a.grads.gate != nullptr) {
      const int64_t p0 = op.gate_ptr[held], p1 = op.gate_ptr[held + 1];
      const bool head = p0 < at.r0, tail = p1 > at.r1;
      float* to = head || tail ? a.slots + (at.walker * 2 + (head ? 0 : 1)) * op.cols : a.grads.gate + held * op.cols;
      const bool add = !(head || tail) && a.grads.accumulate;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < at.n[k]) to[col[k] + e] = add ? to[col[k] + e] + dg[k][e] : dg[k][e];
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) dg[k][e] = 0.f;
  };
  for (int64_t i = 0; i < a.per; ++i) {
    const int64_t r = at.r0 + i, rr = min(r, last);
    bool mine = r < at.r1;
    float x[NV][8], b[NV][8], t[NV][8], z[NV][8];
    const float4 st = ((const float4*)a.stats)[rr];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Raw8<XT> rx = load8((const XT*)a.x.data + rr * a.x.ld + col[k], at.n[k]);
      const Raw8<BT> rb = load8((const BT*)a.b.data + rr * a.b.ld + col[k], at.n[k]);
      const Raw8<XT> ry = load8((const XT*)a.dy.data + rr * a.dy.ld + col[k], a.dy.data ? at.n[k] : 0);
      const Raw8<BT> rz = load8((const BT*)a.dz.data + rr * a.dz.ld + col[k], a.dz.data ? at.n[k] : 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[k][e] = rx.get(e);
        b[k][e] = rb.get(e);
        t[k][e] = ry.get(e);
        z[k][e] = rz.get(e);
      }
    }
    if (a.gmode == kGateGroup && mine) {
      while (g + 1 < op.n_gates && r >= op.gate_ptr[g + 1]) ++g;
      mine = r >= op.gate_ptr[g] && r < op.gate_ptr[g + 1];
      if (mine && g != held) {
        flush();
        load_vec(gate, op.gate + g * op.cols, col, at.n, 1.f);
        held = g;
      }
    }
    if (a.gmode == kGateRow && mine) load_vec(gate, op.gate + r * op.cols, col, at.n, 1.f);
    float p[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[k][e] = b[k][e];
        if (op.post != MGN_NORM_NONE) {
          b[k][e] = (b[k][e] - st.x) * st.y;  // bhat
          p[k][e] = __builtin_fmaf(b[k][e], pg[k][e], pb[k][e]);
        }
      }
    if (op.pre != MGN_NORM_NONE && a.dz.data != nullptr) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = __builtin_fmaf(op.scale, gate[k][e] * p[k][e], op.skip * x[k][e]);
          const float yhat = (y - st.z) * st.w, u = z[k][e] * qg[k][e];
          if (mine && e < at.n[k]) {
            dqb[k][e] += z[k][e];
            dqg[k][e] = __builtin_fmaf(z[k][e], yhat, dqg[k][e]);
            s1 += u;
            s2 = __builtin_fmaf(u, yhat, s2);
          }
          x[k][e] = yhat;
        }
      red.sum2(s1, s2);
      s1 = op.pre == MGN_NORM_LAYER ? s1 * inv : 0.f;
      s2 *= inv;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          t[k][e] = __builtin_fmaf(st.w, z[k][e] * qg[k][e] - s1 - x[k][e] * s2, t[k][e]);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float dx[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dx[e] = op.skip * t[k][e];
        const float dgv = op.scale * (p[k][e] * t[k][e]);
        const float dp = op.scale * (gate[k][e] * t[k][e]), u = dp * pg[k][e];
        if (mine && e < at.n[k]) {
          dg[k][e] = a.gmode == kGateRow ? dgv : dg[k][e] + dgv;
          dpb[k][e] += dp;
          dpg[k][e] = __builtin_fmaf(dp, b[k][e], dpg[k][e]);
          s1 += u;
          s2 = __builtin_fmaf(u, b[k][e], s2);
        }
        t[k][e] = op.post != MGN_NORM_NONE ? u : dp;
      }
      if (mine) store8((XT*)a.dx.data + r * a.dx.ld + col[k], at.n[k], dx);
    }
    if (op.post != MGN_NORM_NONE) {
      red.sum2(s1, s2);
      s1 = op.post == MGN_NORM_LAYER ? s1 * inv : 0.f;
      s2 *= inv;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[k][e] = st.y * (t[k][e] - s1 - b[k][e] * s2);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (mine) store8((BT*)a.db.data + r * a.db.ld + col[k], at.n[k], t[k]);
    if (a.gmode == kGateRow && mine && a.grads.gate != nullptr) {
      float* to = a.grads.gate + r * op.cols;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < at.n[k]) to[col[k] + e] = a.grads.accumulate ? to[col[k] + e] + dg[k][e] : dg[k][e];
    }
  }
  if (a.gmode == kGateGroup) flush();
  // the block's sums, one vector after the other
  float* part = a.part + (int64_t)blockIdx.x * 5 * op.cols;
  auto put = [&](int which, const float (&v)[NV][8]) {
    if constexpr (LPR != 0) {
      const int w = threadIdx.x / LPR, nw = blockDim.x / LPR;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < at.n[k]) sums[w * op.cols + col[k] + e] = v[k][e];
      __syncthreads();
      for (int c = threadIdx.x; c < op.cols; c += blockDim.x) {
        float s = 0.f;
        for (int j = 0; j < nw; ++j) s += sums[j * op.cols + c];
        part[which * op.cols + c] = s;
      }
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < at.n[k]) part[which * op.cols + col[k] + e] = v[k][e];
    }
  };
  if (a.grads.post_gamma != nullptr) put(0, dpg);
  if (a.grads.post_beta != nullptr) put(1, dpb);
  if (a.grads.pre_gamma != nullptr) put(2, dqg);
  if (a.grads.pre_beta != nullptr) put(3, dqb);
  if (a.grads.gate != nullptr && a.gmode == kGateOne) put(4, dg);
}

// Sums over blocks of up to five vectors: 64 columns x 16 groups of rows a
// block, each group's rows and then the groups in order.
struct ColumnSums {
  const float* part;
  int64_t nb, stride, cols;
  float* out[5];
  int32_t accumulate;
};
__global__ void __launch_bounds__(1024) k_column_sums(ColumnSums a) {
  __shared__ float s[16][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + c;
  float* out = a.out[blockIdx.y];
  if (out == nullptr) return;  // the whole block
  const float* p = a.part + blockIdx.y * a.cols + col;
  float v = 0.f;
  if (col < a.cols)
    for (int64_t b = g; b < a.nb; b += 16) v += p[b * a.stride];
  s[g][c] = v;
  __syncthreads();
  if (g == 0 && col < a.cols) {
    float t = a.accumulate ? out[col] : 0.f;
    float u = 0.f;
    for (int j = 0; j < 16; ++j) u += s[j][c];
    out[col] = t + u;
  }
}

// dgate rows of the groups that several walkers share, summed in the walkers'
// order, and zeros for groups without rows.
__global__ void __launch_bounds__(1024) k_gate_slots(NormGate a) {
  __shared__ float s[16][64];
  const mgn_norm_gate& op = a.op;
  const int c = threadIdx.x & 63, q = threadIdx.x >> 6;
  const int col = blockIdx.y * 64 + c;
  const int64_t g = blockIdx.x;
  const int64_t p0 = max((int64_t)op.gate_ptr[g], (int64_t)0), p1 = min((int64_t)op.gate_ptr[g + 1], op.rows);
  const bool none = p1 <= p0;
  const int64_t w0 = none ? 0 : p0 / a.per, w1 = none ? 0 : (p1 - 1) / a.per;
  // one walker's rows only: it has written the sums itself (its last row may
  // be the group's)
  if (!none && w0 == w1 && op.gate_ptr[g] >= w0 * a.per && op.gate_ptr[g + 1] <= min((w0 + 1) * a.per, op.rows)) return;
  float v = 0.f;
  if (!none && col < op.cols)
    for (int64_t w = w0 + q; w <= w1; w += 16) {
      const bool head = op.gate_ptr[g] < w * a.per;
      v += a.slots[(w * 2 + (head ? 0 : 1)) * op.cols + col];
    }
  s[q][c] = v;
  __syncthreads();
  if (q == 0 && col < op.cols) {
    float u = 0.f;
    for (int j = 0; j < 16; ++j) u += s[j][c];
    float* to = a.grads.gate + g * op.cols + col;
    *to = a.grads.accumulate ? *to + u : u;
  }
}

}  // namespace dev

using namespace dev;

NormPlan norm_plan(int64_t rows, int cols, bool backward) {
  NormPlan p;
  p.vpt = cols <= 8192 ? 8 : 16;
  const int lanes = (cols + p.vpt - 1) / p.vpt;
  p.lpr = lanes <= 16 ? 16 : lanes <= 32 ? 32 : lanes <= 64 ? 64 : 0;
  p.threads = p.lpr ? 256 : (lanes + 63) / 64 * 64;
  const int per_block = p.lpr ? 256 / p.lpr : 1;
  // threads in flight: 256 CUs
  const int64_t most = std::max<int64_t>(1, 256 * (backward ? 1024 : 2048) / p.threads) * per_block;
  p.per = std::max<int64_t>(1, ceil_div(rows, most));
  p.blocks = ceil_div(ceil_div(rows, p.per), per_block);
  p.walkers = p.blocks * per_block;
  return p;
}

#define MGN_NG_LAUNCH(K, XT, BT)                                                                       \
  do {                                                                                                 \
    if (p.lpr == 16)                                                                                   \
      hipLaunchKernelGGL((K<XT, BT, 16, 1>), dim3((unsigned)p.blocks), dim3(p.threads), lds, s, a);    \
    else if (p.lpr == 32)                                                                              \
      hipLaunchKernelGGL((K<XT, BT, 32, 1>), dim3((unsigned)p.blocks), dim3(p.threads), lds, s, a);    \
    else if (p.lpr == 64)                                                                              \
      hipLaunchKernelGGL((K<XT, BT, 64, 1>), dim3((unsigned)p.blocks), dim3(p.threads), lds, s, a);    \
    else if (p.vpt == 8)                                                                               \
      hipLaunchKernelGGL((K<XT, BT, 0, 1>), dim3((unsigned)p.blocks), dim3(p.threads), lds, s, a);     \
    else                                                                                               \
      hipLaunchKernelGGL((K<XT, BT, 0, 2>), dim3((unsigned)p.blocks), dim3(p.threads), lds, s, a);     \
  } while (0)
#define MGN_NG_TYPES(K)                                           \
  do {                                                            \
    if (a.op.x_type == MGN_FP32 && a.op.b_type == MGN_FP32)       \
      MGN_NG_LAUNCH(K, float, float);                             \
    else if (a.op.x_type == MGN_FP32)                             \
      MGN_NG_LAUNCH(K, float, bf16);                              \
    else if (a.op.b_type == MGN_FP32)                             \
      MGN_NG_LAUNCH(K, bf16, float);                              \
    else                                                          \
      MGN_NG_LAUNCH(K, bf16, bf16);                               \
  } while (0)

hipError_t launch_norm_gate_forward(const NormGate& in, hipStream_t s) {
  NormGate a = in;
  const NormPlan p = norm_plan(a.op.rows, a.op.cols, false);
  a.per = p.per;
  const size_t lds = 0;
  MGN_NG_TYPES(k_norm_gate_fwd);
  return hipGetLastError();
}

hipError_t launch_norm_gate_backward(const NormGate& in, hipStream_t s) {
  NormGate a = in;
  const NormPlan p = norm_plan(a.op.rows, a.op.cols, true);
  a.per = p.per;
  if (p.blocks > 0) {
    const size_t lds = p.lpr ? (size_t)(p.threads / p.lpr) * a.op.cols * 4 : 0;
    MGN_NG_TYPES(k_norm_gate_bwd);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const bool one = a.gmode == kGateOne;
  if (a.grads.post_gamma || a.grads.post_beta || a.grads.pre_gamma || a.grads.pre_beta || (one && a.grads.gate)) {
    const ColumnSums c = {a.part, p.blocks, 5LL * a.op.cols, a.op.cols,
                          {a.grads.post_gamma, a.grads.post_beta, a.grads.pre_gamma, a.grads.pre_beta,
                           one ? a.grads.gate : nullptr},
                          a.grads.accumulate};
    hipLaunchKernelGGL(k_column_sums, dim3((a.op.cols + 63) / 64, 5), dim3(1024), 0, s, c);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.gmode == kGateGroup && a.grads.gate) {
    hipLaunchKernelGGL(k_gate_slots, dim3((unsigned)a.op.n_gates, (a.op.cols + 63) / 64), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  return hipSuccess;
}

hipError_t launch_column_reduce(const float* part, int64_t nb, int64_t stride, int64_t cols, float* out,
                                int32_t accumulate, hipStream_t s) {
  const ColumnSums c = {part, nb, stride, cols, {out, nullptr, nullptr, nullptr, nullptr}, accumulate};
  hipLaunchKernelGGL(k_column_sums, dim3((unsigned)((cols + 63) / 64), 1), dim3(1024), 0, s, c);
  return hipGetLastError();
}

}  // namespace mgn
