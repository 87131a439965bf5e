// Group norm with an activation, rows of channels, samples being runs of rows, and its
// reverse (see include/mgn.h).
//
// Rows are cut into tiles of as many rows, whatever samples they belong to, so that
// ragged samples load the device evenly.  A block takes a tile's rows in columns of whole
// groups (up to 2048 columns in bf16, 1024 in fp32, wider groups in strips), a thread 16
// neighbouring bytes of every RL-th row.  A launch forms the sums of every piece that a
// tile and a sample share; tile t's and sample s's lies in slot t + s, which no other pair
// has, since of two such pairs one has the larger tile or sample and neither the smaller.
// A second joins a sample's slots in order, a third reads the rows again and writes the
// results.
// Sums of x and x^2 are of 64 bits: var = E x^2 - (E x)^2 loses (mean / std)^2 2^-53 an
// addition.  The mean is then rounded to float32, as stats keep it, which shifts xhat of a whole
// group by up to 2^-24 |mean| / std: as much as half a step of x itself at its mean does, and
// the reverse, which has z and xhat to the bit, takes them so.  Small calls take one block for a
// sample and group columns instead, in one launch.
//
// Bound by memory in fp32: 307,981 x 128 with SiLU, forward 34 us for the sums (4.7 TB/s) and 50
// for the results (6.3), reverse 53 (5.9) and 75 (6.3), joins 5 and 6.  In bf16 the vector
// units share it: 65,536 x 640 21, 29, 41 and 44 us, of which 22 instructions and two
// transcendental ones for an element take 27 in each launch of the reverse.
#include "dev_common.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace dev {

// A thread has 16 bytes of a row: so many columns, and so many 256 threads.
template <typename T>
struct Run {
  static constexpr int V = 16 / sizeof(T), strip = 256 * V;
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(2)));
};

struct GnPlan {
  bool whole;    // a block has all rows of a sample
  int width;     // columns of a block: whole groups
  int cblocks;
  int64_t tile;  // rows of a tile of the sums
  int64_t tiles;
  int64_t atile, atiles;  // of the results
  uint32_t even;  // rows of a sample, without sample_ptr
};

struct GnJob {
  GroupNorm a;
  GnPlan p;
  float2* stats;   // [n_samples][groups]: mean, 1 / standard deviation
  float2* means;   // [n_samples][groups]: of u and u xhat (reverse)
  double2* slots;  // forward: [tiles + n_samples][groups] sums of x and x^2
  float2* bslots;  // reverse: of u and u xhat
  float* part;     // reverse: [tiles or whole_blocks][2][cols] sums of d xhat and d
};

template <typename V>
struct Pair {
  V x, y;
};

// A thread's place in a strip of columns [c0, c1): runs of V columns, the last one moved
// to end at c1, so that every load is a whole one; of it the thread has the columns
// [lo, hi).  Strips of under V columns are one run of hi columns.
template <typename T>
struct Cols {
  static constexpr int V = Run<T>::V;
  typedef typename Run<T>::vec vec;
  int c0, c1, cl, rl, RL;
  int col, lo, hi;
  bool on;
  __device__ __forceinline__ Cols(int c0, int c1) : c0(c0), c1(c1) {
    const int CL = (c1 - c0 + V - 1) / V;
    RL = (int)blockDim.x / CL;
    rl = (int)threadIdx.x / CL;
    cl = (int)threadIdx.x - rl * CL;
    on = rl < RL;
    col = max(min(c0 + cl * V, c1 - V), c0);
    lo = c0 + cl * V - col;
    hi = min(c1 - c0, V);
  }
  __device__ __forceinline__ bool has(int e) const { return e >= lo && e < hi; }
  __device__ __forceinline__ vec load(const mgn_rows& t, int64_t r) const {
    const T* p = (const T*)t.data + r * t.ld + col;
    vec v = {};
    if (hi == V) {
      v = *(const vec*)p;
    } else {
#pragma unroll
      for (int e = 0; e < V - 1; ++e)
        if (e < hi) v[e] = p[e];
    }
    return v;
  }
  // PAST: past L2.
  template <bool PAST>
  __device__ __forceinline__ void store(const mgn_rows& t, int64_t r, const float (&f)[V]) const {
    T* p = (T*)t.data + r * t.ld + col;
    vec v;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (T)f[e];
    if (hi - lo == V) {
      if (PAST)
        __builtin_nontemporal_store(v, (vec*)p);
      else
        *(vec*)p = v;
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (has(e)) p[e] = v[e];
    }
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

// The sample that row r is of: the largest s with ptr[s] <= r.
__device__ __forceinline__ int64_t sample_of(const GnJob& J, int64_t r) {
  const mgn_group_norm& op = J.a.op;
  if (op.sample_ptr == nullptr) return (uint32_t)r / J.p.even;
  // every lane looks at one of 64 places: a trip to memory for each 64 times as many samples
  const uint32_t lane = threadIdx.x & 63;
  uint32_t lo = 0, n = (uint32_t)op.n_samples;
  while (n > 1) {
    const uint32_t step = (n + 63) / 64, at = lane * step;
    const uint64_t m = __ballot(at < n && op.sample_ptr[lo + at] <= r);
    const uint32_t j = m != 0 ? 63 - (uint32_t)__builtin_clzll(m) : 0;
    lo += j * step;
    n = min(step, n - j * step);
  }
  return lo;
}
// The rows of sample s, inside the tensor whatever sample_ptr holds.
__device__ __forceinline__ void rows_of(const GnJob& J, int64_t s, int64_t& b, int64_t& e) {
  const mgn_group_norm& op = J.a.op;
  if (op.sample_ptr == nullptr) {
    b = s * J.p.even;
    e = b + J.p.even;
  } else {
    b = max((int64_t)op.sample_ptr[s], (int64_t)0);
    e = min((int64_t)op.sample_ptr[s + 1], op.rows);
  }
}
// f(s, r, e) for every sample s with rows [r, e) in [r0, r1).
template <typename F>
__device__ __forceinline__ void for_samples(const GnJob& J, int64_t r0, int64_t r1, F f) {
  int64_t r = J.a.op.sample_ptr != nullptr ? max(r0, (int64_t)J.a.op.sample_ptr[0]) : r0;
  while (r < r1) {
    const int64_t s = sample_of(J, r);
    int64_t b, e;
    rows_of(J, s, b, e);
    e = min(e, r1);
    if (e <= r) return;  // behind the last one
    f(s, r, e);
    r = e;
  }
}

// Sums over a strip's rows and the columns of each of its groups (d columns) from every
// thread's: put(g, sums) by one thread for each group.  As many neighbouring columns as
// divide d and the runs are added first.  buf: a pair for each of the block's threads'
// columns.  Ends with the block together.
template <typename T, typename V, typename F>
__device__ __forceinline__ void group_sums(const Cols<T>& at, int d, const V (&s1)[Run<T>::V], const V (&s2)[Run<T>::V],
                                           Pair<V>* buf, F put) {
  constexpr int N = Run<T>::V;
  Pair<V> v[N];
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = {s1[e], s2[e]};
  int q = 1;
#pragma unroll
  for (int k = N; k > 1; k >>= 1) {
    if ((d & (2 * q - 1)) == 0) {
#pragma unroll
      for (int e = 0; e < k / 2; ++e) v[e] = {v[2 * e].x + v[2 * e + 1].x, v[2 * e].y + v[2 * e + 1].y};
      q *= 2;
    }
  }
  const int w = (at.c1 - at.c0) / q, gs = max((at.c1 - at.c0) / d, 1), dw = min(d, at.c1 - at.c0) / q;
  if (at.on) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e * q >= at.lo && e * q < at.hi) buf[at.rl * w + (at.col - at.c0) / q + e] = v[e];
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
      const Pair<V> u = buf[rl * w + g * dw + (i - rl * dw)];
      t.x += u.x;
      t.y += u.y;
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
__device__ __forceinline__ void moments(const mgn_rows& x, const Cols<T>& at, int64_t r, int64_t e, double (&s1)[Run<T>::V],
                                        double (&s2)[Run<T>::V]) {
  constexpr int U = 8, V = Run<T>::V;
#pragma unroll
  for (int k = 0; k < V; ++k) s1[k] = s2[k] = 0.0;
  if (!at.on) return;
  for (int64_t i = r + at.rl; i < e; i += U * at.RL) {
    typename Run<T>::vec v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = at.load(x, min(i + u * at.RL, e - 1));
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * at.RL < e) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const double f = (double)(float)v[u][k];
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
template <typename T>
struct Vec {
  static constexpr int V = Run<T>::V;
  typedef float vec __attribute__((ext_vector_type(V), aligned(4)));
  float v[V];
  __device__ __forceinline__ Vec(const float* p, const Cols<T>& at, float other) {
    vec w;
    if (p != nullptr && at.hi == V) {
      w = *(const vec*)(p + at.col);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = p != nullptr && e < at.hi ? p[at.col + e] : other;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = w[e];
  }
};
// Of each column's group of d: f(group) = (x, y).
template <typename T, typename F>
__device__ __forceinline__ void of_groups(const Cols<T>& at, int d, F f, float (&x)[Run<T>::V], float (&y)[Run<T>::V]) {
  int g = at.col / d, in = at.col - g * d;
  const int last = (at.c1 - 1) / d;
#pragma unroll
  for (int k = 0; k < Run<T>::V; ++k) {
    const float2 s = f(min(g, last));
    x[k] = s.x;
    y[k] = s.y;
    if (++in == d) {
      in = 0;
      ++g;
    }
  }
}

// y of rows [r, e) by the statistics of their sample's groups.
template <typename T, int ACT, bool PAST, typename S>
__device__ __forceinline__ void apply(const GnJob& J, const Cols<T>& at, int d, int64_t r, int64_t e, S stats_of) {
  constexpr int U = 4, V = Run<T>::V;
  if (!at.on) return;
  const Vec<T> gamma(J.a.op.gamma, at, 1.f), beta(J.a.op.beta, at, 0.f);
  float mean[V], f[V];
  of_groups(at, d, stats_of, mean, f);
#pragma unroll
  for (int k = 0; k < V; ++k) f[k] *= gamma.v[k];
  for (int64_t i = r + at.rl; i < e; i += U * at.RL) {
    typename Run<T>::vec v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = at.load(J.a.x, min(i + u * at.RL, e - 1));
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * at.RL < e) {
        float y[V];
#pragma unroll
        for (int k = 0; k < V; ++k)
          y[k] = activated<ACT>(__builtin_fmaf((float)v[u][k] - mean[k], f[k], beta.v[k]));
        at.template store<PAST>(J.a.y, i + u * at.RL, y);
      }
  }
}

// each(k, c, d) for every column of rows [r, e), c = x - mean, d = dy act'(z), then row(i).
// z is formed as in the forward.
template <typename T, int ACT, typename F, typename G>
__device__ __forceinline__ void reversed(const GnJob& J, const Cols<T>& at, int64_t r, int64_t e, const float (&mean)[Run<T>::V],
                                         const float (&f)[Run<T>::V], F each, G row) {
  constexpr int U = 4, V = Run<T>::V;
  const Vec<T> beta(J.a.op.beta, at, 0.f);
  for (int64_t i = r + at.rl; i < e; i += U * at.RL) {
    typename Run<T>::vec v[U], w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[u] = at.load(J.a.x, min(i + u * at.RL, e - 1));
      w[u] = at.load(J.a.dy, min(i + u * at.RL, e - 1));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * at.RL < e) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float c = (float)v[u][k] - mean[k];
          each(k, c, activated_grad<ACT>(__builtin_fmaf(c, f[k], beta.v[k]), (float)w[u][k]));
        }
        row(i + u * at.RL);
      }
  }
}
// Sums of d xhat and d over rows [r, e).
template <typename T, int ACT, typename S>
__device__ __forceinline__ void gradient_sums(const GnJob& J, const Cols<T>& at, int d, int64_t r, int64_t e, S stats_of,
                                              float (&b)[Run<T>::V], float (&a)[Run<T>::V]) {
  constexpr int V = Run<T>::V;
#pragma unroll
  for (int k = 0; k < V; ++k) a[k] = b[k] = 0.f;
  if (!at.on) return;
  const Vec<T> gamma(J.a.op.gamma, at, 1.f);
  float mean[V], rstd[V], f[V];
  of_groups(at, d, stats_of, mean, rstd);
#pragma unroll
  for (int k = 0; k < V; ++k) f[k] = rstd[k] * gamma.v[k];
  reversed<T, ACT>(
      J, at, r, e, mean, f,
      [&](int k, float c, float g) {
        a[k] += g;
        b[k] = __builtin_fmaf(g, c * rstd[k], b[k]);
      },
      [](int64_t) {});
}
// dx = rstd (gamma d - the mean of u - xhat times that of u xhat).
template <typename T, int ACT, bool PAST, typename S, typename M>
__device__ __forceinline__ void input_gradient(const GnJob& J, const Cols<T>& at, int d, int64_t r, int64_t e, S stats_of, M means_of) {
  constexpr int V = Run<T>::V;
  if (!at.on) return;
  const Vec<T> gamma(J.a.op.gamma, at, 1.f);
  float mean[V], rstd[V], f[V], m1[V], m2[V], dx[V];
  of_groups(at, d, stats_of, mean, rstd);
  of_groups(at, d, means_of, m1, m2);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    f[k] = rstd[k] * gamma.v[k];
    m1[k] *= rstd[k];
    m2[k] *= rstd[k];
  }
  reversed<T, ACT>(
      J, at, r, e, mean, f,
      [&](int k, float c, float g) { dx[k] = __builtin_fmaf(f[k], g, -m1[k]) - c * rstd[k] * m2[k]; },
      [&](int64_t i) { at.template store<PAST>(J.a.dx, i, dx); });
}
// A strip's columns' sums over the threads that share them: put(column, sums).
template <typename T, typename F>
__device__ __forceinline__ void column_pairs(const Cols<T>& at, const float (&s1)[Run<T>::V], const float (&s2)[Run<T>::V],
                                             Pair<float>* buf, F put) {
  const int w = at.c1 - at.c0;
  if (at.on) {
#pragma unroll
    for (int e = 0; e < Run<T>::V; ++e)
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
template <typename T>
__device__ __forceinline__ void times_gamma(const GnJob& J, const Cols<T>& at, float (&u)[Run<T>::V], float (&v)[Run<T>::V],
                                            const float (&a)[Run<T>::V], const float (&b)[Run<T>::V]) {
  const Vec<T> gamma(J.a.op.gamma, at, 1.f);
#pragma unroll
  for (int k = 0; k < Run<T>::V; ++k) {
    u[k] = a[k] * gamma.v[k];
    v[k] = b[k] * gamma.v[k];
  }
}

extern __shared__ __align__(16) uint8_t gn_lds[];

// ---- tiles
struct TilePlace {
  int64_t tile, r0, r1;
  int c0, c1, d;
  __device__ __forceinline__ TilePlace(const GnJob& J, int64_t rows) {
    tile = blockIdx.x;
    r0 = tile * rows;
    r1 = min(r0 + rows, J.a.op.rows);
    d = J.a.op.cols / J.a.op.groups;
    c0 = blockIdx.y * J.p.width;
    c1 = min(c0 + J.p.width, J.a.op.cols);
  }
};

template <typename T>
__global__ void __launch_bounds__(256) k_group_moments(GnJob J) {
  const TilePlace t(J, J.p.tile);
  const mgn_group_norm& op = J.a.op;
  Pair<double>* buf = (Pair<double>*)gn_lds;
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    for_samples(J, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      double s1[Run<T>::V], s2[Run<T>::V];
      moments<T>(J.a.x, at, r, e, s1, s2);
      group_sums(at, t.d, s1, s2, buf, [&](int g, Pair<double> v) {
        double2* to = J.slots + (t.tile + s) * op.groups + c / t.d + g;
        *to = c > t.c0 ? double2{to->x + v.x, to->y + v.y} : double2{v.x, v.y};
      });
    });
  }
}

// Statistics (MEANS false) or the means of u and u xhat (true): 32 groups of a sample a
// block.  In the reverse the blocks behind those sum 32 columns of the tiles' parts.
template <bool MEANS>
__global__ void __launch_bounds__(512) k_group_join(GnJob J) {
  constexpr int P = 16;
  __shared__ Pair<double> buf[P][33];
  const mgn_group_norm& op = J.a.op;
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int64_t gblocks = ceil_div(op.groups, 32);
  Pair<double> t = {0.0, 0.0};
  auto joined = [&]() {  // over the parts, in part 0
    buf[part][lane] = t;
    __syncthreads();
    if (part > 0) return false;
    for (int i = 1; i < P; ++i) {
      t.x += buf[i][lane].x;
      t.y += buf[i][lane].y;
    }
    return true;
  };
  if (MEANS && blockIdx.x >= op.n_samples * gblocks) {
    const int64_t c = (blockIdx.x - op.n_samples * gblocks) * 32 + lane;
    if (c < op.cols) {
#pragma unroll 8
      for (int64_t i = part; i < J.p.tiles; i += P) {
        const float* v = J.part + i * 2 * op.cols + c;
        t.x += v[0];
        t.y += v[op.cols];
      }
    }
    if (!joined() || c >= op.cols) return;
    float *const dg = J.a.dgamma, *const db = J.a.dbeta;
    if (dg != nullptr) dg[c] = J.a.accumulate ? dg[c] + (float)t.x : (float)t.x;
    if (db != nullptr) db[c] = J.a.accumulate ? db[c] + (float)t.y : (float)t.y;
    return;
  }
  const int64_t s = blockIdx.x / gblocks;
  const int g = (int)(blockIdx.x - s * gblocks) * 32 + lane;
  int64_t b, e;
  rows_of(J, s, b, e);
  const bool any = e > b;
  const int64_t t0 = any ? b / J.p.tile : 0, t1 = any ? (e - 1) / J.p.tile : -1;
  if (g < op.groups) {
#pragma unroll 8
    for (int64_t i = t0 + part; i <= t1; i += P) {
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
  if (!joined() || g >= op.groups) return;
  const double n = any ? (double)(e - b) * (double)(op.cols / op.groups) : 0.0;
  if constexpr (MEANS)
    J.means[s * op.groups + g] = any ? float2{(float)(t.x / n), (float)(t.y / n)} : float2{0.f, 0.f};
  else
    J.stats[s * op.groups + g] = moments_to_stats(t, n, op.eps);
}

template <typename T, int ACT, bool PAST>
__global__ void __launch_bounds__(256) k_group_apply(GnJob J) {
  const TilePlace t(J, J.p.atile);
  const mgn_group_norm& op = J.a.op;
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    for_samples(J, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      apply<T, ACT, PAST>(J, at, t.d, r, e, [&](int g) { return J.stats[s * op.groups + g]; });
    });
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_group_bwd_sums(GnJob J) {
  const TilePlace t(J, J.p.tile);
  const mgn_group_norm& op = J.a.op;
  Pair<float>* buf = (Pair<float>*)gn_lds;
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    float ta[Run<T>::V] = {}, tb[Run<T>::V] = {};
    for_samples(J, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      float a[Run<T>::V], b[Run<T>::V], u[Run<T>::V], v[Run<T>::V];
      gradient_sums<T, ACT>(J, at, t.d, r, e, [&](int g) { return J.stats[s * op.groups + g]; }, b, a);
      times_gamma(J, at, u, v, a, b);
      group_sums(at, t.d, u, v, buf, [&](int g, Pair<float> w) {
        float2* to = J.bslots + (t.tile + s) * op.groups + c / t.d + g;
        *to = c > t.c0 ? float2{to->x + w.x, to->y + w.y} : float2{w.x, w.y};
      });
#pragma unroll
      for (int k = 0; k < Run<T>::V; ++k) {
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

template <typename T, int ACT, bool PAST>
__global__ void __launch_bounds__(256) k_group_bwd_apply(GnJob J) {
  const TilePlace t(J, J.p.atile);
  const mgn_group_norm& op = J.a.op;
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    for_samples(J, t.r0, t.r1, [&](int64_t s, int64_t r, int64_t e) {
      input_gradient<T, ACT, PAST>(J, at, t.d, r, e, [&](int g) { return J.stats[s * op.groups + g]; },
                             [&](int g) { return J.means[s * op.groups + g]; });
    });
  }
}

// ---- a sample's rows in one block
struct WholePlace {
  int64_t s, r0, r1;
  int c0, c1, d, gs;
  double n;
  __device__ __forceinline__ WholePlace(const GnJob& J, int64_t sample) {
    s = sample;
    rows_of(J, s, r0, r1);
    d = J.a.op.cols / J.a.op.groups;
    c0 = blockIdx.y * J.p.width;
    c1 = min(c0 + J.p.width, J.a.op.cols);
    gs = (c1 - c0) / d;
    n = (double)max(r1 - r0, (int64_t)0) * (double)d;
  }
};

template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_group_whole(GnJob J) {
  const WholePlace t(J, blockIdx.x);
  const mgn_group_norm& op = J.a.op;
  Pair<double>* buf = (Pair<double>*)gn_lds;
  Pair<double>* sums = buf + blockDim.x * Run<T>::V;  // of the block's groups
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    double s1[Run<T>::V], s2[Run<T>::V];
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
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    apply<T, ACT, false>(J, at, t.d, t.r0, t.r1, [&](int g) { return st[g - g0]; });
  }
}

// A block takes every gridDim.x-th sample, whose columns' sums it adds up in its part.
template <typename T, int ACT>
__device__ __forceinline__ void bwd_whole(const GnJob& J, int64_t sample) {
  const WholePlace t(J, sample);
  const mgn_group_norm& op = J.a.op;
  Pair<float>* buf = (Pair<float>*)gn_lds;
  Pair<float>* sums = buf + blockDim.x * Run<T>::V;
  auto stats_of = [&](int g) { return J.stats[t.s * op.groups + g]; };
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    float a[Run<T>::V], b[Run<T>::V], u[Run<T>::V], v[Run<T>::V];
    gradient_sums<T, ACT>(J, at, t.d, t.r0, t.r1, stats_of, b, a);
    times_gamma(J, at, u, v, a, b);
    group_sums(at, t.d, u, v, buf, [&](int g, Pair<float> w) {
      sums[g] = c > t.c0 ? Pair<float>{sums[g].x + w.x, sums[g].y + w.y} : w;
    });
    if (J.part != nullptr)
      column_pairs(at, b, a, buf, [&](int col, Pair<float> w) {
        float* to = J.part + (int64_t)blockIdx.x * 2 * op.cols + col;
        const bool first = t.s == blockIdx.x;
        to[0] = first ? w.x : to[0] + w.x;
        to[op.cols] = first ? w.y : to[op.cols] + w.y;
      });
  }
  const int g0 = t.c0 / t.d;
  const float inv = t.n > 0.0 ? (float)(1.0 / t.n) : 0.f;
  for (int c = t.c0; c < t.c1; c += Run<T>::strip) {
    const Cols<T> at(c, min(c + Run<T>::strip, t.c1));
    input_gradient<T, ACT, false>(J, at, t.d, t.r0, t.r1, stats_of,
                           [&](int g) { return float2{sums[g - g0].x * inv, sums[g - g0].y * inv}; });
  }
}
template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_group_bwd_whole(GnJob J) {
  for (int64_t s = blockIdx.x; s < J.a.op.n_samples; s += gridDim.x) {
    bwd_whole<T, ACT>(J, s);
    __syncthreads();  // the sums have been read
  }
}

}  // namespace dev

using namespace dev;

namespace {

// Blocks that tiles are cut for: as many sums as run at a time (three a CU; 307,981 x 128
// fp32, forward and reverse 96 and 142 us, with 2048 blocks 96 and 154), and as many
// results, in fp32 four a CU (with three the reverse 151, of 307,981 x 128 bf16 83, with four
// 87), or tiles of 16 rows a thread where these are more than four rounds (852,640 x 128 fp32
// 231 and 397 us, one round 245 and 415).
constexpr int kSumBlocks = 768, kResultBlocks = 1024;
// A block takes a sample's rows where a thread has up to kWholeRows of them, a third on
// average where samples are ragged (and 128 if one has all rows), and the call is of up to
// kWholeBytes, 16 times that where they are not; or where samples of equal length fill the
// device.  Both directions through the binding, by tiles in brackets: 1200 x 128 bf16 41 us
// (46), 2000 rows 56 (46); 4000 x 128 fp32 of 8 ragged samples 37 (47); 2000 x 4096 bf16 of 20
// samples 38 (57), ragged 54 (61); 51,200 x 256 fp32 of 100 77 (93); 3000 x 640 bf16 of 5 ragged
// ones 58 (47); 6000 x 640 fp32 of 10 by 80 bytes of a row 55 (47).  By 64 bytes of a row instead
// of all of it: 424 x 640 bf16 of 8 37 us, 81.
constexpr int64_t kWholeRows = 24, kWholeBytes = 4 << 20;

GnPlan plan(const mgn_group_norm& op) {
  GnPlan p;
  const int d = op.cols / op.groups;
  const int64_t size = op.type == MGN_BF16 ? 2 : 4;
  const int run = (int)(16 / size), strip = 256 * run;
  // as many groups as fit a strip, and as many for every block
  p.cblocks = (int)ceil_div(op.groups, std::max(strip / d, 1));
  p.width = (int)ceil_div(op.groups, p.cblocks) * d;
  const int64_t bytes = op.rows * p.width * size;
  auto rows_at_once = [&](int64_t width) { return std::max<int64_t>(256 / ceil_div(std::min<int64_t>(width, strip), run), 1); };
  const int64_t rl = rows_at_once(p.width);
  // a block for a sample takes some 64 or 128 bytes of a row, more where there are many
  const bool even = op.sample_ptr == nullptr;
  const int64_t total = op.rows * op.cols * size, least = total <= kWholeBytes ? 64 : 128;
  const int64_t per = std::max((least + d * size / 2) / (d * size), ceil_div(op.groups * op.n_samples, (int64_t)kResultBlocks));
  const int64_t blocks = ceil_div(op.groups, std::clamp<int64_t>(per, 1, std::max(strip / d, 1)));
  const int64_t width = ceil_div(op.groups, blocks) * d, wrl = rows_at_once(width);
  p.whole = even ? (total <= 16 * kWholeBytes && op.rows <= kWholeRows * wrl * op.n_samples) ||
                       (bytes / op.n_samples <= (1 << 17) && op.n_samples * p.cblocks >= 256)
                 : total <= kWholeBytes && op.rows <= kWholeRows / 3 * wrl * op.n_samples && op.rows <= 128 * wrl;
  if (p.whole) {
    p.width = (int)width;
    p.cblocks = (int)ceil_div(op.groups, width / d);
  }
  auto rows_of = [&](int64_t blocks) { return std::max(ceil_div(op.rows * p.cblocks, blocks), rl * 4); };
  p.tile = rows_of(kSumBlocks);
  p.tiles = p.whole ? 0 : ceil_div(op.rows, p.tile);
  const int64_t results = rows_of(size == 2 ? kSumBlocks : kResultBlocks);
  p.atile = results > rl * 64 ? rl * 16 : results;
  p.atiles = p.whole ? 0 : ceil_div(op.rows, p.atile);
  p.even = (uint32_t)(op.rows / op.n_samples);
  return p;
}

// Blocks of the reverse with a sample a block.
int64_t whole_blocks(const mgn_group_norm& op) { return std::min<int64_t>(op.n_samples, 2048); }

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
  if (backward) l.part = take((size_t)(p.whole ? whole_blocks(op) : p.tiles) * 2 * op.cols * 4);
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

// K<type, act ...>
#define MGN_GN(K, grid, lds, ...)                                                                              \
  do {                                                                                                         \
    const bool f32 = a.op.type == MGN_FP32;                                                                    \
    if (a.op.act == MGN_ACT_NONE) {                                                                            \
      if (f32) hipLaunchKernelGGL((K<float, MGN_ACT_NONE __VA_ARGS__>), grid, dim3(256), lds, s, J);           \
      else hipLaunchKernelGGL((K<bf16, MGN_ACT_NONE __VA_ARGS__>), grid, dim3(256), lds, s, J);                \
    } else if (a.op.act == MGN_ACT_RELU) {                                                                     \
      if (f32) hipLaunchKernelGGL((K<float, MGN_ACT_RELU __VA_ARGS__>), grid, dim3(256), lds, s, J);           \
      else hipLaunchKernelGGL((K<bf16, MGN_ACT_RELU __VA_ARGS__>), grid, dim3(256), lds, s, J);                \
    } else {                                                                                                   \
      if (f32) hipLaunchKernelGGL((K<float, MGN_ACT_SILU __VA_ARGS__>), grid, dim3(256), lds, s, J);           \
      else hipLaunchKernelGGL((K<bf16, MGN_ACT_SILU __VA_ARGS__>), grid, dim3(256), lds, s, J);                \
    }                                                                                                          \
    const hipError_t err = hipGetLastError();                                                                  \
    if (err != hipSuccess) return err;                                                                         \
  } while (0)

// Whether results go past L2: they are more than all L2s hold (307,981 x 128 fp32, forward and
// reverse 95 and 158 us, else 112 and 185), and of aligned rows.
bool past_l2(const mgn_group_norm& op, const mgn_rows& out) {
  const int64_t size = op.type == MGN_BF16 ? 2 : 4;
  return op.rows * op.cols * size > (32LL << 20) && (((uintptr_t)out.data | (uintptr_t)(out.ld * size)) & 15) == 0;
}
// Bytes of LDS for `pair` bytes for each of the block's columns.
size_t lds_of(const mgn_group_norm& op, size_t pair) { return 256 * (op.type == MGN_BF16 ? 8 : 4) * pair; }

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
    MGN_GN(k_group_whole, g, lds_of(a.op, 16) + (size_t)(p.width / (a.op.cols / a.op.groups)) * 16, );
    return hipSuccess;
  }
  const dim3 g((unsigned)p.tiles, p.cblocks);
  if (a.op.type == MGN_FP32)
    hipLaunchKernelGGL((k_group_moments<float>), g, dim3(256), lds_of(a.op, 16), s, J);
  else
    hipLaunchKernelGGL((k_group_moments<bf16>), g, dim3(256), lds_of(a.op, 16), s, J);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_group_join<false>), dim3((unsigned)(a.op.n_samples * ceil_div(a.op.groups, 32))), dim3(512), 0, s, J);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 ga((unsigned)p.atiles, p.cblocks);
  if (past_l2(a.op, a.y))
    MGN_GN(k_group_apply, ga, 0, , true);
  else
    MGN_GN(k_group_apply, ga, 0, , false);
  return hipSuccess;
}

hipError_t launch_group_norm_backward(const GroupNorm& a, hipStream_t s) {
  float* const out[2] = {a.dgamma, a.dbeta};
  if (a.op.n_samples == 0)
    return a.dgamma || a.dbeta ? launch_column_reduce(nullptr, 0, a.op.cols, out, 2, a.accumulate, s) : hipSuccess;
  const GnPlan p = plan(a.op);
  const GnJob J = job(a, p, true);
  if (p.whole) {
    const dim3 g((unsigned)whole_blocks(a.op), p.cblocks);
    MGN_GN(k_group_bwd_whole, g, lds_of(a.op, 8) + (size_t)(p.width / (a.op.cols / a.op.groups)) * 8, );
  } else {
    const dim3 g((unsigned)p.tiles, p.cblocks);
    MGN_GN(k_group_bwd_sums, g, lds_of(a.op, 8), );
    hipLaunchKernelGGL((k_group_join<true>),
                       dim3((unsigned)(a.op.n_samples * ceil_div(a.op.groups, 32) + (J.part ? ceil_div(a.op.cols, 32) : 0))),
                       dim3(512), 0, s, J);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 ga((unsigned)p.atiles, p.cblocks);
    if (past_l2(a.op, a.dx))
      MGN_GN(k_group_bwd_apply, ga, 0, , true);
    else
      MGN_GN(k_group_bwd_apply, ga, 0, , false);
  }
  if (!J.part || !p.whole) return hipSuccess;
  return launch_column_reduce(J.part, whole_blocks(a.op), a.op.cols, out, 2, a.accumulate, s);
}

}  // namespace mgn
