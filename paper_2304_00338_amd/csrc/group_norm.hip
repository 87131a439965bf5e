// Group norm with an activation, rows of channels, samples being runs of rows, and its
// reverse (see include/mgn.h).
//
// Rows are cut into tiles of as many rows, whatever samples they belong to, so that
// ragged samples load the device evenly.  A block takes a tile's rows in columns of whole
// groups (up to 2048 columns, wider groups in strips), a thread 8 neighbouring columns of
// every RL-th row.  A launch forms the sums of every piece that a tile and a sample
// share; tile t's and sample s's lies in slot t + s, which no other pair has, since
// of two such pairs one has the larger tile or sample and neither the smaller.  A second
// joins a sample's slots in order, a third reads the rows again and writes the results.
// Sums of x and x^2 are of 64 bits, exact enough for any mean: var = E x^2 - (E x)^2
// loses (mean / std)^2 2^-53.  Small calls take one block for a sample and group columns
// instead, in one launch.
#include "dev_common.hpp"
#include "row_io.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

constexpr int kStrip = 2048;  // columns that 256 threads hold, 8 each

struct GnPlan {
  bool whole;    // a block has all rows of a sample
  int threads;
  int width;     // columns of a block: whole groups
  int cblocks;
  int64_t tile;  // rows
  int64_t tiles;
};

struct GnJob {
  GroupNorm a;
  GnPlan p;
  float2* stats;   // [n_samples][groups]: mean, 1 / standard deviation
  float2* means;   // [n_samples][groups]: of u and u xhat (reverse)
  double2* slots;  // forward: [tiles + n_samples][groups] sums of x and x^2
  float2* bslots;  // reverse: of u and u xhat
  float* part;     // reverse: [tiles or n_samples][2][cols] sums of d xhat and d
};

template <typename V>
struct Pair {
  V x, y;
};

// A thread's place in a strip of columns [c0, c1): runs of 8 columns, the last one moved
// to end at c1, so that every load is a whole one; of it the thread has the columns
// [lo, hi).  Strips of under 8 columns are one run of hi columns.
struct Cols {
  int c0, c1, cl, rl, RL;
  int col, lo, hi;
  bool on;
  __device__ __forceinline__ Cols(int c0, int c1) : c0(c0), c1(c1) {
    const int CL = (c1 - c0 + 7) >> 3;
    RL = (int)blockDim.x / CL;
    rl = (int)threadIdx.x / CL;
    cl = (int)threadIdx.x - rl * CL;
    on = rl < RL;
    col = max(min(c0 + cl * 8, c1 - 8), c0);
    lo = c0 + cl * 8 - col;
    hi = min(c1 - c0, 8);
  }
  __device__ __forceinline__ bool has(int e) const { return e >= lo && e < hi; }
  template <typename T>
  __device__ __forceinline__ Raw8<T> load(const mgn_rows& t, int64_t r) const {
    return load8((const T*)t.data + r * t.ld + col, hi);
  }
};

template <int ACT>
__device__ __forceinline__ float activated(float z) {
  if constexpr (ACT == MGN_ACT_RELU) return z < 0.f ? 0.f : z;  // a NaN stays
  if constexpr (ACT == MGN_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
  return z;
}
// dy act'(z)
template <int ACT>
__device__ __forceinline__ float activated_grad(float z, float dy) {
  if constexpr (ACT == MGN_ACT_RELU) return z > 0.f ? dy : 0.f;
  if constexpr (ACT == MGN_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.f + __expf(-z));
    return dy * s * __builtin_fmaf(z, 1.f - s, 1.f);
  }
  return dy;
}

// The sample that row r is of: the largest s with ptr[s] <= r.  (-1: none has it.)
__device__ __forceinline__ int64_t sample_of(const mgn_group_norm& op, int64_t r) {
  if (op.sample_ptr == nullptr) return r / (op.rows / op.n_samples);
  int64_t lo = 0, hi = op.n_samples - 1;
  while (lo < hi) {
    const int64_t m = (lo + hi + 1) >> 1;
    if (op.sample_ptr[m] <= r)
      lo = m;
    else
      hi = m - 1;
  }
  return lo;
}
// The rows of sample s, inside the tensor whatever sample_ptr holds.
__device__ __forceinline__ void rows_of(const mgn_group_norm& op, int64_t s, int64_t& b, int64_t& e) {
  if (op.sample_ptr == nullptr) {
    const int64_t n = op.rows / op.n_samples;
    b = s * n;
    e = b + n;
  } else {
    b = max((int64_t)op.sample_ptr[s], (int64_t)0);
    e = min((int64_t)op.sample_ptr[s + 1], op.rows);
  }
}
// f(s, r, e) for every sample s with rows [r, e) in [r0, r1).
template <typename F>
__device__ __forceinline__ void for_samples(const mgn_group_norm& op, int64_t r0, int64_t r1, F f) {
  int64_t r = op.sample_ptr != nullptr ? max(r0, (int64_t)op.sample_ptr[0]) : r0;
  while (r < r1) {
    const int64_t s = sample_of(op, r);
    int64_t b, e;
    rows_of(op, s, b, e);
    e = min(e, r1);
    if (e <= r) return;  // behind the last one
    f(s, r, e);
    r = e;
  }
}

// Sums over a strip's rows and the columns of each of its groups (d columns) from every
// thread's eight: put(g, sums) by one thread for each group.  buf: a pair for each of
// the block's threads' columns.  Ends with the block together.
template <typename V, typename F>
__device__ __forceinline__ void group_sums(const Cols& at, int d, const V (&s1)[8], const V (&s2)[8], Pair<V>* buf, F put) {
  const int w = at.c1 - at.c0, gs = max(w / d, 1), dw = min(d, w);
  if (at.on) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at.has(e)) buf[at.rl * w + at.col - at.c0 + e] = Pair<V>{s1[e], s2[e]};
  }
  __syncthreads();
  int P = 64;
  while (P > 1 && P * gs > (int)blockDim.x) P >>= 1;
  const int p = threadIdx.x & (P - 1), n = at.RL * dw;
  const float inv = 1.f / (float)dw;
  for (int g = (int)threadIdx.x / P; g < gs; g += (int)blockDim.x / P) {
    Pair<V> t = {0, 0};
    for (int i = p; i < n; i += P) {
      const int rl = (int)(((float)i + 0.5f) * inv);
      const Pair<V> v = buf[rl * w + g * dw + (i - rl * dw)];
      t.x += v.x;
      t.y += v.y;
    }
    for (int k = P >> 1; k > 0; k >>= 1) {
      t.x += __shfl_xor(t.x, k);
      t.y += __shfl_xor(t.y, k);
    }
    if (p == 0) put(g, t);
  }
  __syncthreads();
}

// Sums of x and x^2 of rows [r, e).
template <typename T>
__device__ __forceinline__ void moments(const mgn_rows& x, const Cols& at, int64_t r, int64_t e, double (&s1)[8], double (&s2)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) s1[k] = s2[k] = 0.0;
  if (!at.on) return;
  for (int64_t i = r + at.rl; i < e; i += 4 * at.RL) {
    Raw8<T> v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = at.template load<T>(x, min(i + u * at.RL, e - 1));
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * at.RL < e) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const double f = (double)v[u].get(k);
          s1[k] += f;
          s2[k] = __builtin_fma(f, f, s2[k]);
        }
      }
  }
}

__device__ __forceinline__ float2 moments_to_stats(Pair<double> t, double n, float eps) {
  if (!(n > 0.0)) return float2{0.f, (float)(1.0 / __builtin_sqrt((double)eps))};
  const double mean = t.x / n, var = t.y / n - mean * mean;
  return float2{(float)mean, (float)(1.0 / __builtin_sqrt((var > 0.0 || var != var ? var : 0.0) + (double)eps))};
}

// What a thread keeps of its columns.
struct Vec8 {
  float v[8];
  __device__ __forceinline__ Vec8(const float* p, const Cols& at, float other) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p != nullptr && at.has(e) ? p[at.col + e] : other;
  }
};

// y of rows [r, e) by the statistics of their sample's groups.
template <typename T, int ACT, typename S>
__device__ __forceinline__ void apply(const GnJob& J, const Cols& at, int d, int64_t r, int64_t e, S stats_of) {
  if (!at.on) return;
  const Vec8 gamma(J.a.op.gamma, at, 1.f), beta(J.a.op.beta, at, 0.f);
  float mean[8], f[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float2 s = at.has(k) ? stats_of((at.col + k) / d) : float2{0.f, 0.f};
    mean[k] = s.x;
    f[k] = s.y * gamma.v[k];
  }
  for (int64_t i = r + at.rl; i < e; i += 4 * at.RL) {
    Raw8<T> v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = at.template load<T>(J.a.x, min(i + u * at.RL, e - 1));
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * at.RL < e) {
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = activated<ACT>(__builtin_fmaf(v[u].get(k) - mean[k], f[k], beta.v[k]));
        store8((T*)J.a.y.data + (i + u * at.RL) * J.a.y.ld + at.col, at.lo, at.hi, y);
      }
  }
}

// f(u, k, xhat, d) for rows [r, e): d = dy act'(z).
template <typename T, int ACT, typename S, typename F, typename G>
__device__ __forceinline__ void reversed(const GnJob& J, const Cols& at, int d, int64_t r, int64_t e, S stats_of, F each, G row) {
  const Vec8 gamma(J.a.op.gamma, at, 1.f), beta(J.a.op.beta, at, 0.f);
  float mean[8], rstd[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float2 s = at.has(k) ? stats_of((at.col + k) / d) : float2{0.f, 0.f};
    mean[k] = s.x;
    rstd[k] = s.y;
  }
  for (int64_t i = r + at.rl; i < e; i += 2 * at.RL) {
    Raw8<T> v[2], w[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      v[u] = at.template load<T>(J.a.x, min(i + u * at.RL, e - 1));
      w[u] = at.template load<T>(J.a.dy, min(i + u * at.RL, e - 1));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (i + u * at.RL < e) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float xhat = (v[u].get(k) - mean[k]) * rstd[k];
          each(k, xhat, activated_grad<ACT>(__builtin_fmaf(xhat, gamma.v[k], beta.v[k]), w[u].get(k)), gamma.v[k], rstd[k]);
        }
        row(i + u * at.RL);
      }
  }
}
// Sums of d xhat and d over rows [r, e).
template <typename T, int ACT, typename S>
__device__ __forceinline__ void gradient_sums(const GnJob& J, const Cols& at, int d, int64_t r, int64_t e, S stats_of,
                                              float (&b)[8], float (&a)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) a[k] = b[k] = 0.f;
  if (!at.on) return;
  reversed<T, ACT>(
      J, at, d, r, e, stats_of,
      [&](int k, float xhat, float g, float, float) {
        a[k] += g;
        b[k] = __builtin_fmaf(g, xhat, b[k]);
      },
      [](int64_t) {});
}
template <typename T, int ACT, typename S, typename M>
__device__ __forceinline__ void input_gradient(const GnJob& J, const Cols& at, int d, int64_t r, int64_t e, S stats_of, M means_of) {
  if (!at.on) return;
  float m1[8], m2[8], dx[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float2 s = at.has(k) ? means_of((at.col + k) / d) : float2{0.f, 0.f};
    m1[k] = s.x;
    m2[k] = s.y;
  }
  reversed<T, ACT>(
      J, at, d, r, e, stats_of,
      [&](int k, float xhat, float g, float gamma, float rstd) {
        dx[k] = rstd * (__builtin_fmaf(gamma, g, -m1[k]) - xhat * m2[k]);
      },
      [&](int64_t i) { store8((T*)J.a.dx.data + i * J.a.dx.ld + at.col, at.lo, at.hi, dx); });
}
// A strip's columns' sums over the threads that share them: put(column, sums).
template <typename F>
__device__ __forceinline__ void column_pairs(const Cols& at, const float (&s1)[8], const float (&s2)[8], Pair<float>* buf, F put) {
  const int w = at.c1 - at.c0;
  if (at.on) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at.has(e)) buf[at.rl * w + at.col - at.c0 + e] = Pair<float>{s1[e], s2[e]};
  }
  __syncthreads();
  for (int c = threadIdx.x; c < w; c += blockDim.x) {
    Pair<float> t = {0.f, 0.f};
    for (int i = 0; i < at.RL; ++i) {
      t.x += buf[i * w + c].x;
      t.y += buf[i * w + c].y;
    }
    put(at.c0 + c, t);
  }
  __syncthreads();
}
__device__ __forceinline__ void times_gamma(const GnJob& J, const Cols& at, float (&u)[8], float (&v)[8], const float (&a)[8],
                                            const float (&b)[8]) {
  const Vec8 gamma(J.a.op.gamma, at, 1.f);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    u[k] = a[k] * gamma.v[k];
    v[k] = b[k] * gamma.v[k];
  }
}

extern __shared__ __align__(16) uint8_t gn_lds[];

// ---- tiles
struct TilePlace {
  int64_t tile, r0, r1;
  int c0, c1, d;
  __device__ __forceinline__ TilePlace(const GnJob& J) {
    tile = blockIdx.x;
    r0 = tile * J.p.tile;
    r1 = min(r0 + J.p.tile, J.a.op.rows);
    d = J.a.op.cols / J.a.op.groups;
    c0 = blockIdx.y * J.p.width;
    c1 = min(c0 + J.p.width, J.a.op.cols);
  }
};

template <typename T>
__global__ void __launch_bounds__(256) k_group_moments(GnJob J) {
  const TilePlace t(J);
  const mgn_group_norm& op = J.a.op;
  Pair<double>* buf = (Pair<double>*)gn_lds;
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    for_samples(op, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      double s1[8], s2[8];
      moments<T>(J.a.x, at, r, e, s1, s2);
      group_sums(at, t.d, s1, s2, buf, [&](int g, Pair<double> v) {
        double2* to = J.slots + (t.tile + s) * op.groups + c / t.d + g;
        *to = c > t.c0 ? double2{to->x + v.x, to->y + v.y} : double2{v.x, v.y};
      });
    });
  }
}

// Statistics (MEANS false) or the means of u and u xhat (true): 32 groups of a sample a block.
template <bool MEANS>
__global__ void __launch_bounds__(1024) k_group_join(GnJob J) {
  __shared__ Pair<double> buf[32][33];
  const mgn_group_norm& op = J.a.op;
  const int g = blockIdx.y * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
  const int64_t s = blockIdx.x;
  int64_t b, e;
  rows_of(op, s, b, e);
  const bool any = e > b;
  const int64_t t0 = any ? b / J.p.tile : 0, t1 = any ? (e - 1) / J.p.tile : -1;
  Pair<double> t = {0.0, 0.0};
  if (g < op.groups) {
#pragma unroll 4
    for (int64_t i = t0 + part; i <= t1; i += 32) {
      const int64_t at = (i + s) * op.groups + g;
      if constexpr (MEANS) {
        const float2 v = J.bslots[at];
        t.x += v.x;
        t.y += v.y;
      } else {
        const double2 v = J.slots[at];
        t.x += v.x;
        t.y += v.y;
      }
    }
  }
  buf[part][threadIdx.x & 31] = t;
  __syncthreads();
  if (part > 0 || g >= op.groups) return;
  for (int i = 1; i < 32; ++i) {
    t.x += buf[i][threadIdx.x].x;
    t.y += buf[i][threadIdx.x].y;
  }
  const double n = any ? (double)(e - b) * (double)(op.cols / op.groups) : 0.0;
  if constexpr (MEANS)
    J.means[s * op.groups + g] = any ? float2{(float)(t.x / n), (float)(t.y / n)} : float2{0.f, 0.f};
  else
    J.stats[s * op.groups + g] = moments_to_stats(t, n, op.eps);
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_group_apply(GnJob J) {
  const TilePlace t(J);
  const mgn_group_norm& op = J.a.op;
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    for_samples(op, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      apply<T, ACT>(J, at, t.d, r, e, [&](int g) { return J.stats[s * op.groups + g]; });
    });
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_group_bwd_sums(GnJob J) {
  const TilePlace t(J);
  const mgn_group_norm& op = J.a.op;
  Pair<float>* buf = (Pair<float>*)gn_lds;
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    float ta[8] = {}, tb[8] = {};
    for_samples(op, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      float a[8], b[8], u[8], v[8];
      gradient_sums<T, ACT>(J, at, t.d, r, e, [&](int g) { return J.stats[s * op.groups + g]; }, b, a);
      times_gamma(J, at, u, v, a, b);
      group_sums(at, t.d, u, v, buf, [&](int g, Pair<float> w) {
        float2* to = J.bslots + (t.tile + s) * op.groups + c / t.d + g;
        *to = c > t.c0 ? float2{to->x + w.x, to->y + w.y} : float2{w.x, w.y};
      });
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        ta[k] += a[k];
        tb[k] += b[k];
      }
    });
    if (J.part != nullptr)
      column_pairs(at, tb, ta, buf, [&](int col, Pair<float> w) {
        float* to = J.part + t.tile * 2 * op.cols + col;
        to[0] = w.x;
        to[op.cols] = w.y;
      });
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_group_bwd_apply(GnJob J) {
  const TilePlace t(J);
  const mgn_group_norm& op = J.a.op;
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    for_samples(op, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      input_gradient<T, ACT>(J, at, t.d, r, e, [&](int g) { return J.stats[s * op.groups + g]; },
                             [&](int g) { return J.means[s * op.groups + g]; });
    });
  }
}

// ---- a sample's rows in one block
struct WholePlace {
  int64_t s, r0, r1;
  int c0, c1, d, gs;
  double n;
  __device__ __forceinline__ WholePlace(const GnJob& J) {
    s = blockIdx.x;
    rows_of(J.a.op, s, r0, r1);
    d = J.a.op.cols / J.a.op.groups;
    c0 = blockIdx.y * J.p.width;
    c1 = min(c0 + J.p.width, J.a.op.cols);
    gs = (c1 - c0) / d;
    n = (double)max(r1 - r0, (int64_t)0) * (double)d;
  }
};

template <typename T, int ACT>
__global__ void __launch_bounds__(512) k_group_whole(GnJob J) {
  const WholePlace t(J);
  const mgn_group_norm& op = J.a.op;
  Pair<double>* buf = (Pair<double>*)gn_lds;
  Pair<double>* sums = buf + blockDim.x * 8;  // of the block's groups
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    double s1[8], s2[8];
    moments<T>(J.a.x, at, t.r0, t.r1, s1, s2);
    group_sums(at, t.d, s1, s2, buf, [&](int g, Pair<double> v) {
      sums[g] = c > t.c0 ? Pair<double>{sums[g].x + v.x, sums[g].y + v.y} : v;
    });
  }
  const int g0 = t.c0 / t.d;
  float2* st = (float2*)buf;
  for (int g = threadIdx.x; g < t.gs; g += blockDim.x) {
    st[g] = moments_to_stats(sums[g], t.n, op.eps);
    if (J.stats != nullptr) J.stats[t.s * op.groups + g0 + g] = st[g];
  }
  __syncthreads();
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    apply<T, ACT>(J, at, t.d, t.r0, t.r1, [&](int g) { return st[g - g0]; });
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(512) k_group_bwd_whole(GnJob J) {
  const WholePlace t(J);
  const mgn_group_norm& op = J.a.op;
  Pair<float>* buf = (Pair<float>*)gn_lds;
  Pair<float>* sums = buf + blockDim.x * 8;
  auto stats_of = [&](int g) { return J.stats[t.s * op.groups + g]; };
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    float a[8], b[8], u[8], v[8];
    gradient_sums<T, ACT>(J, at, t.d, t.r0, t.r1, stats_of, b, a);
    times_gamma(J, at, u, v, a, b);
    group_sums(at, t.d, u, v, buf, [&](int g, Pair<float> w) {
      sums[g] = c > t.c0 ? Pair<float>{sums[g].x + w.x, sums[g].y + w.y} : w;
    });
    if (J.part != nullptr)
      column_pairs(at, b, a, buf, [&](int col, Pair<float> w) {
        float* to = J.part + t.s * 2 * op.cols + col;
        to[0] = w.x;
        to[op.cols] = w.y;
      });
  }
  const int g0 = t.c0 / t.d;
  const float inv = t.n > 0.0 ? (float)(1.0 / t.n) : 0.f;
  for (int c = t.c0; c < t.c1; c += kStrip) {
    const Cols at(c, min(c + kStrip, t.c1));
    input_gradient<T, ACT>(J, at, t.d, t.r0, t.r1, stats_of,
                           [&](int g) { return float2{sums[g - g0].x * inv, sums[g - g0].y * inv}; });
  }
}

}  // namespace dev

using namespace dev;

namespace {

GnPlan plan(const mgn_group_norm& op) {
  GnPlan p;
  const int d = op.cols / op.groups;
  const int64_t size = op.type == MGN_BF16 ? 2 : 4;
  p.width = d >= kStrip ? d : kStrip / d * d;
  if (p.width > op.cols) p.width = op.cols;
  p.cblocks = (int)ceil_div(op.cols, p.width);
  const int64_t bytes = op.rows * p.width * size;
  p.whole = bytes <= (1 << 20) ||
            (op.sample_ptr == nullptr && bytes / op.n_samples <= (1 << 17) && op.n_samples * p.cblocks >= 256);
  p.threads = 256;
  // about 2048 blocks, of 4 rows a thread or more
  const int64_t lanes = ceil_div(std::min(p.width, kStrip), 8), rl = std::max<int64_t>(256 / lanes, 1);
  p.tile = std::max(rl * 4, ceil_div(op.rows * p.cblocks, 2048));
  p.tiles = p.whole ? 0 : ceil_div(op.rows, p.tile);
  return p;
}

struct Layout {
  size_t stats, means, slots, part, total;
};
Layout layout(const mgn_group_norm& op, const GnPlan& p, bool backward) {
  Layout l = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
  };
  const size_t per = (size_t)op.n_samples * op.groups;
  if (!p.whole) {
    l.stats = take(backward ? 0 : per * 8);
    l.means = take(backward ? per * 8 : 0);
    l.slots = take((size_t)(p.tiles + op.n_samples) * op.groups * (backward ? 8 : 16));
  }
  if (backward) l.part = take((size_t)(p.whole ? op.n_samples : p.tiles) * 2 * op.cols * 4);
  l.total = at;
  return l;
}

GnJob job(const GroupNorm& a, const GnPlan& p, bool backward) {
  GnJob J = {a, p, (float2*)a.stats, nullptr, nullptr, nullptr, nullptr};
  const Layout l = layout(a.op, p, backward);
  char* ws = (char*)a.ws;
  if (!p.whole) {
    if (backward) {
      J.means = (float2*)(ws + l.means);
      J.bslots = (float2*)(ws + l.slots);
    } else {
      if (!J.stats) J.stats = (float2*)(ws + l.stats);
      J.slots = (double2*)(ws + l.slots);
    }
  }
  if (backward && (a.dgamma || a.dbeta)) J.part = (float*)(ws + l.part);
  return J;
}

#define MGN_GN(K, grid, threads, lds)                                                                          \
  do {                                                                                                         \
    const bool f32 = a.op.type == MGN_FP32;                                                                    \
    if (a.op.act == MGN_ACT_NONE) {                                                                            \
      if (f32) hipLaunchKernelGGL((K<float, MGN_ACT_NONE>), grid, dim3(threads), lds, s, J);                   \
      else hipLaunchKernelGGL((K<bf16, MGN_ACT_NONE>), grid, dim3(threads), lds, s, J);                        \
    } else if (a.op.act == MGN_ACT_RELU) {                                                                     \
      if (f32) hipLaunchKernelGGL((K<float, MGN_ACT_RELU>), grid, dim3(threads), lds, s, J);                   \
      else hipLaunchKernelGGL((K<bf16, MGN_ACT_RELU>), grid, dim3(threads), lds, s, J);                        \
    } else {                                                                                                   \
      if (f32) hipLaunchKernelGGL((K<float, MGN_ACT_SILU>), grid, dim3(threads), lds, s, J);                   \
      else hipLaunchKernelGGL((K<bf16, MGN_ACT_SILU>), grid, dim3(threads), lds, s, J);                        \
    }                                                                                                          \
    const hipError_t err = hipGetLastError();                                                                  \
    if (err != hipSuccess) return err;                                                                         \
  } while (0)

}  // namespace

size_t group_norm_workspace(const mgn_group_norm& op, bool backward) {
  if (op.n_samples == 0) return 0;
  return layout(op, plan(op), backward).total;
}

hipError_t launch_group_norm_forward(const GroupNorm& a, hipStream_t s) {
  if (a.op.n_samples == 0) return hipSuccess;
  const GnPlan p = plan(a.op);
  const GnJob J = job(a, p, false);
  if (p.whole) {
    const dim3 g((unsigned)a.op.n_samples, p.cblocks);
    MGN_GN(k_group_whole, g, p.threads, p.threads * 128 + (size_t)(p.width / (a.op.cols / a.op.groups)) * 16);
    return hipSuccess;
  }
  const dim3 g((unsigned)p.tiles, p.cblocks);
  if (a.op.type == MGN_FP32)
    hipLaunchKernelGGL((k_group_moments<float>), g, dim3(256), 256 * 128, s, J);
  else
    hipLaunchKernelGGL((k_group_moments<bf16>), g, dim3(256), 256 * 128, s, J);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_group_join<false>), dim3((unsigned)a.op.n_samples, (unsigned)ceil_div(a.op.groups, 32)), dim3(1024), 0,
                     s, J);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  MGN_GN(k_group_apply, g, 256, 0);
  return hipSuccess;
}

hipError_t launch_group_norm_backward(const GroupNorm& a, hipStream_t s) {
  float* const out[2] = {a.dgamma, a.dbeta};
  if (a.op.n_samples == 0)
    return a.dgamma || a.dbeta ? launch_column_reduce(nullptr, 0, a.op.cols, out, 2, a.accumulate, s) : hipSuccess;
  const GnPlan p = plan(a.op);
  const GnJob J = job(a, p, true);
  if (p.whole) {
    const dim3 g((unsigned)a.op.n_samples, p.cblocks);
    MGN_GN(k_group_bwd_whole, g, p.threads, p.threads * 64 + (size_t)(p.width / (a.op.cols / a.op.groups)) * 8);
  } else {
    const dim3 g((unsigned)p.tiles, p.cblocks);
    MGN_GN(k_group_bwd_sums, g, 256, 256 * 64);
    hipLaunchKernelGGL((k_group_join<true>), dim3((unsigned)a.op.n_samples, (unsigned)ceil_div(a.op.groups, 32)), dim3(1024), 0,
                       s, J);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    MGN_GN(k_group_bwd_apply, g, 256, 0);
  }
  if (!J.part) return hipSuccess;
  return launch_column_reduce(J.part, p.whole ? a.op.n_samples : p.tiles, a.op.cols, out, 2, a.accumulate, s);
}

}  // namespace mgn
