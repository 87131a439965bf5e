// Internal interface of the row operators (mgn_quant8, mgn_matmul8,
// mgn_norm_gate_*, mgn_quant4, mgn_matmul4, mgn_group_norm_*, mgn_grad_*): what
// row_ops.cpp checks and plans, and what the kernels of quant8.hip,
// matmul8.hip, norm_gate.hip, quant4.hip, matmul4.hip, group_norm.hip and
// grad_clip.hip take.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mgn.h"

namespace mgn {

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// n blocks of a launch as the rows of a grid (a dimension has under 2^32 threads):
// block x + y * (blocks of a row), some of the last row being behind the last one.
constexpr int64_t kGridRow = 1 << 20;
inline dim3 grid_of(int64_t n) {
  return dim3((unsigned)(n < kGridRow ? n : kGridRow), (unsigned)ceil_div(n, kGridRow));
}

// ---- quant8
struct Quant8 {
  const void* x;
  int32_t x_type, format, block_rows;
  int64_t rows, cols, ldx;
  uint8_t *q, *qt;
  int64_t ldq, ldqt;
  float *scale, *scale_t;
  float* colsum;  // nullable
  float* part;    // [ceil(rows / 128)][cols] partial column sums
  int32_t accumulate;
};
hipError_t launch_quant8(const Quant8& a, hipStream_t s);

// ---- matmul8
struct Matmul8 {
  mgn_mat8 a, b;
  mgn_epilogue ep;
  int32_t c_type;
  void* c;
  int64_t ldc;
  float* part;  // workspace
};
hipError_t launch_matmul8(const Matmul8& a, hipStream_t s);
// Workspace that launch_matmul8 splits sums in.
size_t matmul8_workspace(int64_t m, int64_t n, int64_t k);

// ---- norm_gate
enum { kGateNone, kGateOne, kGateRow, kGateGroup };
struct NormGate {
  mgn_norm_gate op;
  int32_t gmode;
  mgn_rows x, b, y, z;
  float* stats;
  mgn_rows dy, dz, dx, db;
  mgn_norm_gate_grads grads;
  int64_t per;   // rows of a walker
  float* part;   // [blocks][5][cols]: a block's sums for the vectors' gradients
  float* slots;  // [walkers][2][cols]: sums of gate groups that a walker shares with others
};
// A walker is the lanes that hold one row; it takes `per` consecutive rows.
struct NormPlan {
  int lpr;          // lanes of a walker
  int vpt;          // columns of a lane
  int threads;      // of a block
  int64_t walkers, blocks, per;
};
NormPlan norm_plan(int64_t rows, int cols, bool backward);
hipError_t launch_norm_gate_forward(const NormGate& a, hipStream_t s);
hipError_t launch_norm_gate_backward(const NormGate& a, hipStream_t s);

// ---- quant4
struct Quant4 {
  const void* x;
  int32_t x_type;
  int64_t rows, cols, ldx;
  uint8_t *q, *qt;
  int64_t ldq, ldqt;
  uint8_t *scale, *scale_t;
  float* colsum;  // nullable
  float* part;    // [ceil(rows / 128)][cols] partial column sums
  int32_t accumulate;
};
hipError_t launch_quant4(const Quant4& a, hipStream_t s);
struct Dequant4 {
  mgn_mat4 a;
  int32_t y_type;
  void* y;
  int64_t ldy;
};
hipError_t launch_dequant4(const Dequant4& a, hipStream_t s);

// ---- matmul4
struct Matmul4 {
  mgn_mat4 a, b;
  mgn_epilogue ep;
  int32_t c_type;
  void* c;
  int64_t ldc;
  float* part;  // workspace
};
hipError_t launch_matmul4(const Matmul4& a, hipStream_t s);
size_t matmul4_workspace(int64_t m, int64_t n, int64_t k);

// ---- group_norm
struct GroupNorm {
  mgn_group_norm op;
  mgn_rows x, y, dy, dx;
  float* stats;  // the caller's, nullable in the forward
  float *dgamma, *dbeta;
  int32_t accumulate;
  void* ws;
};
size_t group_norm_workspace(const mgn_group_norm& op, bool backward);
hipError_t launch_group_norm_forward(const GroupNorm& a, hipStream_t s);
hipError_t launch_group_norm_backward(const GroupNorm& a, hipStream_t s);

// ---- grad_clip
constexpr int kPiece = 16384;
struct GradClip {
  const mgn_piece* pieces;
  int64_t n;
  double max_norm;
  float* norm;
  bool given, clip;
  double* part;
};
size_t grad_norm_workspace(int64_t n_pieces);
hipError_t launch_grad_clip(const GradClip& a, hipStream_t s);

// out[i][c] (+)= sum over b < nb of part[(b n + i) cols + c], i < n <= 5 (out[i] NULL: not
// wanted), in a fixed order; part is overwritten.
hipError_t launch_column_reduce(float* part, int64_t nb, int64_t cols, float* const* out, int n, int32_t accumulate,
                                hipStream_t s);

}  // namespace mgn
