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
//
// Measured, forward and reverse: 307,981 x 128 fp32 / bf16, 32 gates 130 and 189 us
// (3.6 and 3.8 TB/s), 16,384 x 5001 bf16 192 and 234 us (3.4 and 4.2), with 32 gates 276
// and 284, 307,981 x 128 with a gate for each row 288 and 575, one row of 4096 8.8
// us.  Bound by memory at narrow rows; a row of a whole block adds the barriers of its
// two to four sums, another gate than the row's before the loads of its vectors.
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

// The walker's place: its lane, rows and columns.  Runs of 8 columns start at
// multiples of 8, but the last at cols - 8, so that every load is one of 16 or
// 32 bytes inside the row; of that run a lane has the columns [lo, 8), of a run
// behind the row none (lo 8), and what it has not counts as 0.  (With loads of
// single elements for the last columns, each wait in their branch waited for the
// next row's loads too: 16,384 x 5000 bf16 took 282 us in the reverse, 5120
// columns 172.)  Rows of under 8 columns are one run [0, hi).
template <int LPR, int NV>
struct Place {
  int lane, lanes;
  int64_t walker, r0, r1;
  int col[NV], lo[NV], hi;
  bool tiny;
  __device__ __forceinline__ Place(int64_t rows, int cols, int64_t per) {
    lanes = LPR ? LPR : blockDim.x;
    lane = LPR ? threadIdx.x & (LPR - 1) : threadIdx.x;
    walker = LPR ? (int64_t)blockIdx.x * (blockDim.x / LPR) + threadIdx.x / LPR : blockIdx.x;
    r0 = min(walker * per, rows);
    r1 = min(r0 + per, rows);
    tiny = cols < 8;
    hi = min(cols, 8);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * lanes + lane) * 8;
      col[k] = max(min(c, cols - 8), 0);
      lo[k] = min(c - col[k], 8);
    }
  }
  __device__ __forceinline__ bool has(int k, int e) const { return e >= lo[k] && e < hi; }
  template <typename T>
  __device__ __forceinline__ Raw8<T> load(const mgn_rows& t, int64_t r, int k) const {
    const T* p = (const T*)t.data + r * t.ld + col[k];
    return load8(p, tiny ? hi : 8);
  }
  template <typename T>
  __device__ __forceinline__ void store(const mgn_rows& t, int64_t r, int k, const float (&f)[8]) const {
    store8((T*)t.data + r * t.ld + col[k], lo[k], hi, f);
  }
};

template <int LPR, int NV>
__device__ __forceinline__ void load_vec(float (&v)[NV][8], const float* p, const Place<LPR, NV>& at, float other) {
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[k][e] = p != nullptr ? (at.has(k, e) ? p[at.col[k] + e] : 0.f) : other;
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
__device__ __forceinline__ void statistics(const float (&v)[NV][8], const Place<LPR, NV>& at, int kind, float inv, float eps,
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
      const float d = at.has(k, e) ? v[k][e] - mean : 0.f;
      q = __builtin_fmaf(d, d, q);
    }
  rstd = 1.f / __builtin_sqrtf(__builtin_fmaf(red.sum(q), inv, eps));
}

// Which gate a row has.  Groups are looked up once and followed from row to row: a
// step to the next group, and behind that, where groups are empty, a search again
// (any number of them can lie between two rows).
struct Gates {
  int64_t g = 0, held = -1;
  __device__ __forceinline__ Gates(const NormGate& a, int64_t r0) {
    if (a.gmode == kGateGroup) g = find_group(a.op.gate_ptr, a.op.n_gates, r0);
  }
  // Whether row r has one; fresh: it is another than the row's before.
  __device__ __forceinline__ bool at(const NormGate& a, int64_t r, bool& fresh) {
    fresh = false;
    if (a.gmode == kGateRow) {
      fresh = true;
      held = r;
    } else if (a.gmode == kGateGroup) {
      if (g + 1 < a.op.n_gates && r >= a.op.gate_ptr[g + 1]) {
        ++g;
        if (g + 1 < a.op.n_gates && r >= a.op.gate_ptr[g + 1]) g += find_group(a.op.gate_ptr + g, a.op.n_gates - g, r);
      }
      if (r < a.op.gate_ptr[g] || r >= a.op.gate_ptr[g + 1]) return false;
      fresh = g != held;
      held = g;
    }
    return true;
  }
};

// y = skip x + ga bhat + gb: ga = scale gate gamma, gb = scale gate beta.
template <int LPR, int NV>
__device__ __forceinline__ void gate_vectors(float (&ga)[NV][8], float (&gb)[NV][8], const NormGate& a, int64_t gate,
                                             const Place<LPR, NV>& at) {
  const mgn_norm_gate& op = a.op;
  const float* g = a.gmode == kGateNone ? nullptr : op.gate + gate * op.cols;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    // opaque, or the addresses of all vectors are kept in registers from row to row
    int c0 = at.col[k];
    asm volatile("" : "+v"(c0));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = at.has(k, e);
      const int c = in ? c0 + e : 0;
      const float v = in ? op.scale * (g != nullptr ? g[c] : 1.f) : 0.f;
      ga[k][e] = v * (op.post_gamma != nullptr ? op.post_gamma[c] : 1.f);
      gb[k][e] = op.post_beta != nullptr ? v * op.post_beta[c] : 0.f;
    }
  }
}

template <typename XT, typename BT, int LPR, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT, LPR ? 4 : 1) k_norm_gate_fwd(NormGate a) {
  __shared__ float buf[64];
  const mgn_norm_gate& op = a.op;
  const Place<LPR, NV> at(op.rows, op.cols, a.per);
  Reduce<LPR> red{buf};
  const float inv = 1.f / (float)op.cols;
  float ga[NV][8], gb[NV][8], qg[NV][8], qb[NV][8];
  gate_vectors(ga, gb, a, 0, at);
  load_vec(qg, op.pre_gamma, at, 1.f);
  load_vec(qb, op.pre_beta, at, 0.f);
  const int64_t last = op.rows - 1;
  // the last run's first columns are loaded by two lanes: where y replaces x both
  // have to be done before either stores, which the sums of post see to
  const bool plain = op.post == MGN_NORM_NONE;
  Gates gates(a, at.r0);
  Raw8<XT> nx[NV];
  Raw8<BT> nb[NV];
  auto fetch = [&](int64_t r) {
    const int64_t rr = min(r, last);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      nx[k] = at.template load<XT>(a.x, rr, k);
      nb[k] = at.template load<BT>(a.b, rr, k);
    }
  };
  fetch(at.r0);
  // every walker of a wave or block takes as many turns: the sums cross lanes
  for (int64_t i = 0; i < a.per; ++i) {
    const int64_t r = at.r0 + i;
    float x[NV][8], b[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      // (a branch around this, for rows that need none, took 226 us instead of
      // 172 at 16,384 x 5120)
      keep(nx[k], at.lo[k], at.hi);
      keep(nb[k], at.lo[k], at.hi);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[k][e] = nx[k].get(e);
        b[k][e] = nb[k].get(e);
      }
    }
    if (LPR == 0 && plain) __syncthreads();
    if (i + 1 < a.per) fetch(r + 1);
    bool fresh = false;
    const bool mine = r < at.r1 && gates.at(a, r, fresh);
    if (fresh) gate_vectors(ga, gb, a, gates.held, at);
    float pm = 0.f, pr = 1.f, qm = 0.f, qr = 1.f;
    if (op.post != MGN_NORM_NONE) statistics(b, at, op.post, inv, op.eps, red, pm, pr);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      // beyond the row x, ga and gb are 0
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[k][e] = __builtin_fmaf(op.skip, x[k][e], __builtin_fmaf((b[k][e] - pm) * pr, ga[k][e], gb[k][e]));
      if (mine) at.template store<XT>(a.y, r, k, x[k]);
    }
    if (op.pre != MGN_NORM_NONE) {
      statistics(x, at, op.pre, inv, op.eps, red, qm, qr);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] = __builtin_fmaf((x[k][e] - qm) * qr, qg[k][e], qb[k][e]);
        if (mine) at.template store<BT>(a.z, r, k, x[k]);
      }
    }
    if (a.stats != nullptr && mine && at.lane == 0) ((float4*)a.stats)[r] = float4{pm, pr, qm, qr};
  }
}

// Reverse.  With t = dy + pre'(dz), dp = scale gate t:
//   dx = skip t, db = post'(dp), dgate = sum of scale p t, dgamma_post = sum of
//   dp bhat, dbeta_post = sum of dp, dgamma_pre = sum of dz yhat, dbeta_pre =
//   sum of dz; norm'(d) = rstd (u - mean(u) - vhat mean(u vhat)), u = gamma d
//   (RMS: without mean(u)).
// y is formed again from x and b, unrounded, and with the forward's statistics
// no sum precedes those of the gradients.  While the gate stays the same, two
// column sums, st = sum of t and sb = sum of t bhat, stand for three:
//   dgate = scale (gamma sb + beta st), dgamma_post += scale gate sb,
//   dbeta_post += scale gate st.
// MANY: there are gates of rows or groups; without, these are formed once.
template <typename XT, typename BT, int LPR, int NV, int MAXT, bool MANY>
__global__ void __launch_bounds__(MAXT) k_norm_gate_bwd(NormGate a) {
  __shared__ float buf[64];
  extern __shared__ float sums[];  // LPR: [walkers of the block][cols]
  const mgn_norm_gate& op = a.op;
  // the next row's loads under this one, where the registers hold them
  constexpr bool PRE = LPR == 0 && NV == 1;
  const Place<LPR, NV> at(op.rows, op.cols, a.per);
  Reduce<LPR> red{buf};
  const float inv = 1.f / (float)op.cols;
  float ga[NV][8], gb[NV][8], qg[NV][8];
  gate_vectors(ga, gb, a, 0, at);
  load_vec(qg, op.pre_gamma, at, 1.f);
  float st[NV][8] = {}, sb[NV][8] = {}, dqg[NV][8] = {}, dqb[NV][8] = {};
  float dpg[MANY ? NV : 1][8] = {}, dpb[MANY ? NV : 1][8] = {};
  const int64_t last = op.rows - 1;
  // as in the forward: dx may replace what two lanes load; the sums of pre come
  // before it is stored
  const bool plain = op.pre == MGN_NORM_NONE || a.dz.data == nullptr;
  Gates gates(a, at.r0);
  auto vec = [&](const float* p, int c, float other) { return p != nullptr ? p[c] : other; };
  // The sums st and sb of a gate become those of the vectors.  dgate goes to
  // its place if all the group's rows are this walker's, else into one of its
  // two slots (first: the group began before its rows).
  auto settle = [&](int64_t held) {
    const float* gate = op.gate + held * op.cols;
    float* to = nullptr;
    bool add = a.grads.accumulate;
    if (a.grads.gate != nullptr) {
      to = a.grads.gate + held * op.cols;
      if (a.gmode == kGateGroup) {
        const bool head = op.gate_ptr[held] < at.r0, tail = op.gate_ptr[held + 1] > at.r1;
        if (head || tail) {
          to = a.slots + (at.walker * 2 + (head ? 0 : 1)) * op.cols;
          add = false;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < (MANY ? NV : 1); ++k) {
      int c0 = at.col[k];
      asm volatile("" : "+v"(c0));  // as in gate_vectors
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at.has(k, e)) {
          const int c = c0 + e;
          const float v = op.scale * gate[c];
          const float d = op.scale * (vec(op.post_gamma, c, 1.f) * sb[k][e] + vec(op.post_beta, c, 0.f) * st[k][e]);
          dpg[k][e] = __builtin_fmaf(v, sb[k][e], dpg[k][e]);
          dpb[k][e] = __builtin_fmaf(v, st[k][e], dpb[k][e]);
          if (to != nullptr) to[c] = add ? to[c] + d : d;
          st[k][e] = 0.f;
          sb[k][e] = 0.f;
        }
    }
  };
  Raw8<XT> nx[NV], ny[NV] = {};
  Raw8<BT> nb[NV], nz[NV] = {};
  float4 ns;
  auto fetch = [&](int64_t r) {
    const int64_t rr = min(r, last);
    ns = ((const float4*)a.stats)[rr];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      nx[k] = at.template load<XT>(a.x, rr, k);
      nb[k] = at.template load<BT>(a.b, rr, k);
      if (a.dy.data != nullptr) ny[k] = at.template load<XT>(a.dy, rr, k);
      if (a.dz.data != nullptr) nz[k] = at.template load<BT>(a.dz, rr, k);
    }
  };
  if (PRE) fetch(at.r0);
  int64_t open = -1;  // the gate that st and sb belong to
  for (int64_t i = 0; i < a.per; ++i) {
    const int64_t r = at.r0 + i;
    bool fresh = false;
    const bool mine = r < at.r1 && (!MANY || gates.at(a, r, fresh));
    if (MANY && fresh) {
      if (open >= 0) settle(open);
      open = gates.held;
      gate_vectors(ga, gb, a, open, at);
    }
    // A row that counts for nothing may hold anything, and the gate at hand may
    // be of no row: the walker's lanes, which agree on it, form nothing of it (0
    // times an infinity would be a NaN in all sums).
    if (LPR != 0 && !mine) continue;
    if (!PRE) fetch(r);
    float x[NV][8], b[NV][8], t[NV][8], z[NV][8];
    const float4 s = ns;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      // bhat is not 0 beyond the lane's columns, but ga and the gradients are
      keep(nx[k], at.lo[k], at.hi);
      keep(ny[k], at.lo[k], at.hi);
      keep(nz[k], at.lo[k], at.hi);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[k][e] = nx[k].get(e);
        b[k][e] = (nb[k].get(e) - s.x) * s.y;  // bhat (b itself without a norm: statistics 0 and 1)
        t[k][e] = ny[k].get(e);
        z[k][e] = nz[k].get(e);
      }
    }
    if (LPR == 0 && plain) __syncthreads();
    if (PRE && i + 1 < a.per) fetch(r + 1);
    if (LPR == 0 && !mine) continue;  // the whole block
    if (op.pre != MGN_NORM_NONE && a.dz.data != nullptr) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = __builtin_fmaf(op.skip, x[k][e], __builtin_fmaf(b[k][e], ga[k][e], gb[k][e]));
          x[k][e] = (y - s.z) * s.w;  // yhat
          dqb[k][e] += z[k][e];
          dqg[k][e] = __builtin_fmaf(z[k][e], x[k][e], dqg[k][e]);
          z[k][e] *= qg[k][e];
          s1 += z[k][e];
          s2 = __builtin_fmaf(z[k][e], x[k][e], s2);
        }
      red.sum2(s1, s2);
      s1 = op.pre == MGN_NORM_LAYER ? s1 * inv : 0.f;
      s2 *= inv;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          t[k][e] = __builtin_fmaf(s.w, z[k][e] - s1 - x[k][e] * s2, t[k][e]);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float dx[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dx[e] = op.skip * t[k][e];
        st[k][e] += t[k][e];
        sb[k][e] = __builtin_fmaf(t[k][e], b[k][e], sb[k][e]);
        t[k][e] *= ga[k][e];  // gamma dp; 0 beyond the row
        s1 += t[k][e];
        s2 = __builtin_fmaf(t[k][e], b[k][e], s2);
      }
      at.template store<XT>(a.dx, r, k, dx);
    }
    if (op.post != MGN_NORM_NONE) {
      red.sum2(s1, s2);
      s1 = op.post == MGN_NORM_LAYER ? s1 * inv : 0.f;
      s2 *= inv;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[k][e] = s.y * (t[k][e] - s1 - b[k][e] * s2);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) at.template store<BT>(a.db, r, k, t[k]);
  }
  if (MANY && open >= 0) settle(open);
  // the block's sums, one vector after the other
  float* part = a.part + (int64_t)blockIdx.x * 5 * op.cols;
  auto put = [&](int which, auto value) {
    if constexpr (LPR != 0) {
      const int w = threadIdx.x / LPR, nw = blockDim.x / LPR;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at.has(k, e)) sums[w * op.cols + at.col[k] + e] = value(k, e, at.col[k] + e);
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
          if (at.has(k, e)) part[which * op.cols + at.col[k] + e] = value(k, e, at.col[k] + e);
    }
  };
  const float* one = a.gmode == kGateOne ? op.gate : nullptr;
  if (a.grads.post_gamma != nullptr)
    put(0, [&](int k, int e, int c) { return MANY ? dpg[MANY ? k : 0][e] : op.scale * vec(one, c, 1.f) * sb[k][e]; });
  if (a.grads.post_beta != nullptr)
    put(1, [&](int k, int e, int c) { return MANY ? dpb[MANY ? k : 0][e] : op.scale * vec(one, c, 1.f) * st[k][e]; });
  if (a.grads.pre_gamma != nullptr) put(2, [&](int k, int e, int) { return dqg[k][e]; });
  if (a.grads.pre_beta != nullptr) put(3, [&](int k, int e, int) { return dqb[k][e]; });
  if (a.grads.gate != nullptr && one != nullptr)
    put(4, [&](int k, int e, int c) {
      return op.scale * (vec(op.post_gamma, c, 1.f) * sb[k][e] + vec(op.post_beta, c, 0.f) * st[k][e]);
    });
}

// Sums over rows of partial sums, 16 columns x 64 groups of rows a block: a
// group's rows in order, then the groups in order.
constexpr int kSumCols = 16, kSumGroups = 64;
template <typename F>
__device__ __forceinline__ float column_sum(int64_t n, bool in, F value) {
  __shared__ float s[kSumGroups][kSumCols + 1];
  const int c = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols;
  float v = 0.f;
  if (in) {
#pragma unroll 4
    for (int64_t b = g; b < n; b += kSumGroups) v += value(b);
  }
  s[g][c] = v;
  __syncthreads();
  float u = 0.f;
  if (g < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) u += s[8 * g + j][c];
  }
  __syncthreads();
  if (g < 8) s[g][c] = u;
  __syncthreads();
  u = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) u += s[j][c];
  return u;  // of column c, for every group
}

struct ColumnSums {
  const float* part;
  int64_t nb, stride, cols;
  float* out[5];
  int32_t accumulate;
};
__global__ void __launch_bounds__(1024) k_column_sums(ColumnSums a) {
  const int64_t col = (blockIdx.y * kGridRow + blockIdx.x) * kSumCols + threadIdx.x % kSumCols;
  float* out = a.out[blockIdx.z];
  if (out == nullptr) return;  // the whole block
  const float* p = a.part + blockIdx.z * a.cols + col;
  const float v = column_sum(a.nb, col < a.cols, [&](int64_t b) { return p[b * a.stride]; });
  if (threadIdx.x < kSumCols && col < a.cols) out[col] = a.accumulate ? out[col] + v : v;
}

// The first half of a long sum: `per` rows into the first of them.
__global__ void __launch_bounds__(1024) k_column_fold(float* part, int64_t nb, int64_t cols, int64_t per) {
  const int64_t col = (blockIdx.y * kGridRow + blockIdx.x) * kSumCols + threadIdx.x % kSumCols, b0 = blockIdx.z * per;
  float* p = part + b0 * cols + col;
  const float v = column_sum(min(per, nb - b0), col < cols, [&](int64_t b) { return p[b * cols]; });
  if (threadIdx.x < kSumCols && col < cols) *p = v;
}

// dgate rows of the groups that several walkers share, and zeros for groups
// without rows.
__global__ void __launch_bounds__(1024) k_gate_slots(NormGate a) {
  const mgn_norm_gate& op = a.op;
  const int col = blockIdx.z * kSumCols + threadIdx.x % kSumCols;
  const int64_t g = blockIdx.y * kGridRow + blockIdx.x;
  if (g >= op.n_gates) return;
  const int64_t b0 = op.gate_ptr[g], b1 = op.gate_ptr[g + 1];
  const int64_t p0 = max(b0, (int64_t)0), p1 = min(b1, op.rows);
  const bool none = p1 <= p0;
  const int64_t w0 = none ? 0 : p0 / a.per, w1 = none ? -1 : (p1 - 1) / a.per;
  // one walker's rows only: it has written the sums itself (its last row may
  // be the group's)
  if (!none && w0 == w1 && b0 >= w0 * a.per && b1 <= min((w0 + 1) * a.per, op.rows)) return;
  const float v = column_sum(w1 - w0 + 1, col < op.cols, [&](int64_t i) {
    const int64_t w = w0 + i;
    return a.slots[(w * 2 + (b0 < w * a.per ? 0 : 1)) * op.cols + col];
  });
  if (threadIdx.x < kSumCols && col < op.cols) {
    float* to = a.grads.gate + g * op.cols + col;
    *to = a.grads.accumulate ? *to + v : v;
  }
}

}  // namespace dev

using namespace dev;

NormPlan norm_plan(int64_t rows, int cols, bool backward) {
  NormPlan p;
  // In the reverse two runs a lane from 5121 columns on.  With one run blocks have up
  // to 1024 threads, whose 128 registers do not hold it: forward and reverse of 16,384
  // rows of 8192 bf16 924 us (two runs 607), of 7168 856 (544).  Blocks of 704 and 768
  // threads would still have 168: compiled for 768, one run takes 455 us at 6144
  // columns (two 497) and 421 at 5632 (484).
  // What spills: with gates of rows or groups one run from 4097 columns on 6 to 11
  // registers, two runs 37 to 86, each for three of the four pairs of types (reverse of
  // 16,384 x 8192 bf16 with 32 gates 583 us, without 354); above 8192 columns, in blocks of
  // 1024, the reverse 173 to 412 and the forward 84 to 102 (8192 x 16,384 1.69 ms and
  // 390 us).
  p.vpt = cols <= (backward ? 5120 : 8192) ? 8 : 16;
  const int lanes = (cols + p.vpt - 1) / p.vpt;
  p.lpr = lanes <= 16 ? 16 : lanes <= 32 ? 32 : lanes <= 64 ? 64 : 0;
  p.threads = p.lpr ? 256 : (lanes + 63) / 64 * 64;
  const int per_block = p.lpr ? 256 / p.lpr : 1;
  // as many blocks as run at a time on 256 CUs: by registers 16 waves of the
  // forward fit a CU (20 in blocks of 640), 12 of the reverse (16 in blocks of 1024)
  const int waves = p.threads / 64;
  const int64_t most = 256 * std::max(1, (backward ? 12 : p.lpr ? 16 : 20) / waves) * per_block;
  p.per = std::max<int64_t>(1, ceil_div(rows, most));
  p.blocks = ceil_div(ceil_div(rows, p.per), per_block);
  p.walkers = p.blocks * per_block;
  return p;
}

// The instantiation for a plan: K(lanes, runs of a lane, most threads).  The forward's
// with one run has 89 to 95 registers for any number of threads.
template <typename XT, typename BT>
void launch_fwd(const NormGate& a, const NormPlan& p, hipStream_t s) {
  const dim3 g((unsigned)p.blocks), t(p.threads);
#define MGN_NG_FWD(L, NV, MAXT) hipLaunchKernelGGL((k_norm_gate_fwd<XT, BT, L, NV, MAXT>), g, t, 0, s, a)
  if (p.lpr == 16)
    MGN_NG_FWD(16, 1, 256);
  else if (p.lpr == 32)
    MGN_NG_FWD(32, 1, 256);
  else if (p.lpr == 64)
    MGN_NG_FWD(64, 1, 256);
  else if (p.vpt == 8)
    MGN_NG_FWD(0, 1, 1024);
  else
    MGN_NG_FWD(0, 2, 1024);
}
template <typename XT, typename BT, bool MANY>
void launch_bwd(const NormGate& a, const NormPlan& p, hipStream_t s) {
  const dim3 g((unsigned)p.blocks), t(p.threads);
  const size_t lds = p.lpr ? (size_t)(p.threads / p.lpr) * a.op.cols * 4 : 0;
#define MGN_NG_BWD(L, NV, MAXT) hipLaunchKernelGGL((k_norm_gate_bwd<XT, BT, L, NV, MAXT, MANY>), g, t, lds, s, a)
  if (p.lpr == 16)
    MGN_NG_BWD(16, 1, 256);
  else if (p.lpr == 32)
    MGN_NG_BWD(32, 1, 256);
  else if (p.lpr == 64)
    MGN_NG_BWD(64, 1, 256);
  else if (p.vpt == 8 && p.threads <= 512)
    MGN_NG_BWD(0, 1, 512);
  else if (p.vpt == 8)
    MGN_NG_BWD(0, 1, 640);
  else if (p.threads <= 512)
    MGN_NG_BWD(0, 2, 512);
  else
    MGN_NG_BWD(0, 2, 1024);
}
template <typename XT, typename BT>
void launch_bwd(const NormGate& a, const NormPlan& p, hipStream_t s) {
  if (a.gmode == kGateRow || a.gmode == kGateGroup)
    launch_bwd<XT, BT, true>(a, p, s);
  else
    launch_bwd<XT, BT, false>(a, p, s);
}
#define MGN_NG_TYPES(LAUNCH)                                \
  do {                                                      \
    if (a.op.x_type == MGN_FP32 && a.op.b_type == MGN_FP32) \
      LAUNCH<float, float>(a, p, s);                        \
    else if (a.op.x_type == MGN_FP32)                       \
      LAUNCH<float, bf16>(a, p, s);                         \
    else if (a.op.b_type == MGN_FP32)                       \
      LAUNCH<bf16, float>(a, p, s);                         \
    else                                                    \
      LAUNCH<bf16, bf16>(a, p, s);                          \
  } while (0)

hipError_t launch_norm_gate_forward(const NormGate& in, hipStream_t s) {
  NormGate a = in;
  const NormPlan p = norm_plan(a.op.rows, a.op.cols, false);
  a.per = p.per;
  MGN_NG_TYPES(launch_fwd);
  return hipGetLastError();
}

hipError_t launch_norm_gate_backward(const NormGate& in, hipStream_t s) {
  NormGate a = in;
  const NormPlan p = norm_plan(a.op.rows, a.op.cols, true);
  a.per = p.per;
  if (p.blocks > 0) {
    MGN_NG_TYPES(launch_bwd);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const bool one = a.gmode == kGateOne;
  if (a.grads.post_gamma || a.grads.post_beta || a.grads.pre_gamma || a.grads.pre_beta || (one && a.grads.gate)) {
    const ColumnSums c = {a.part, p.blocks, 5LL * a.op.cols, a.op.cols,
                          {a.grads.post_gamma, a.grads.post_beta, a.grads.pre_gamma, a.grads.pre_beta,
                           one ? a.grads.gate : nullptr},
                          a.grads.accumulate};
    dim3 g = grid_of(ceil_div(a.op.cols, kSumCols));
    g.z = 5;
    hipLaunchKernelGGL(k_column_sums, g, dim3(1024), 0, s, c);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.gmode == kGateGroup && a.grads.gate) {
    dim3 g = grid_of(a.op.n_gates);
    g.z = (unsigned)ceil_div(a.op.cols, kSumCols);
    hipLaunchKernelGGL(k_gate_slots, g, dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  return hipSuccess;
}

hipError_t launch_column_reduce(float* part, int64_t nb, int64_t cols, float* const* out, int n, int32_t accumulate,
                                hipStream_t s) {
  const int64_t all = cols * n;
  int64_t stride = all;
  if (nb > 1024) {  // 6662 x 128: 10.2 us in two steps, 16.4 in one, whose 8 blocks wait for memory
    dim3 g = grid_of(ceil_div(all, kSumCols));
    const int64_t per = std::max<int64_t>(256, ceil_div(nb, 32768));
    g.z = (unsigned)ceil_div(nb, per);
    hipLaunchKernelGGL(k_column_fold, g, dim3(1024), 0, s, part, nb, all, per);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    nb = g.z;
    stride = per * all;
  }
  ColumnSums c = {part, nb, stride, cols, {}, accumulate};
  for (int i = 0; i < n; ++i) c.out[i] = out[i];
  dim3 g = grid_of(ceil_div(cols, kSumCols));
  g.z = (unsigned)n;
  hipLaunchKernelGGL(k_column_sums, g, dim3(1024), 0, s, c);
  return hipGetLastError();
}

}  // namespace mgn
