// C-ABI entry points of the row operators: argument checks, workspace sizes,
// launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "internal.hpp"
#include "row_ops.hpp"

namespace mgn {
namespace {

constexpr int64_t kMost = (int64_t)1 << 31;

bool is_row_type(int32_t t) { return t == MGN_FP32 || t == MGN_BF16; }
bool is_format(int32_t f) { return f == MGN_E4M3 || f == MGN_E5M2; }
int64_t elem(int32_t t) { return t == MGN_BF16 ? 2 : 4; }
// bytes of a row of 4-bit numbers
int64_t half_bytes(int64_t cols) { return (cols + 31) / 32 * 16; }
int64_t up16(int64_t v) { return (v + 15) & ~(int64_t)15; }
bool aligned(const void* p, int64_t a) { return ((uintptr_t)p & (uintptr_t)(a - 1)) == 0; }
// every element's byte offset has to fit 63 bits
bool fits(int64_t rows, int64_t ld) { return ld <= ((int64_t)1 << 60) / (rows > 0 ? rows : 1); }

int launched(hipError_t e, const char* who) {
  if (e != hipSuccess) return fail(MGN_ERR_DEVICE, "%s: %s", who, hipGetErrorString(e));
  return MGN_OK;
}

int check_mat8(const mgn_mat8* a, const char* who, const char* name) {
  if (!a) return fail(MGN_ERR_ARG, "%s: null %s", who, name);
  if (!is_format(a->format)) return fail(MGN_ERR_ARG, "%s: %s: unknown 8-bit format %d", who, name, a->format);
  if (a->block_rows != 1 && a->block_rows != 128)
    return fail(MGN_ERR_ARG, "%s: %s: blocks of %d rows (1 or 128)", who, name, a->block_rows);
  if (a->rows < 0 || a->cols < 0) return fail(MGN_ERR_ARG, "%s: %s: negative size", who, name);
  if (a->rows >= kMost || a->cols >= kMost) return fail(MGN_ERR_SHAPE, "%s: %s: 2^31 rows or columns", who, name);
  if (a->rows > 0 && a->cols > 0) {
    if (!a->q || !a->scale) return fail(MGN_ERR_ARG, "%s: %s: null numbers or scales", who, name);
    if (!aligned(a->q, 16) || !aligned(a->scale, 4) || (a->ld & 15) != 0 || a->ld < up16(a->cols) ||
        !fits(a->rows, a->ld))
      return fail(MGN_ERR_ARG, "%s: %s: rows have to start at multiples of 16 bytes (ld %lld, cols %lld)", who, name,
                  (long long)a->ld, (long long)a->cols);
  }
  return MGN_OK;
}

int check_rows(const mgn_rows& t, int64_t rows, int64_t cols, int32_t type, const char* who, const char* name) {
  if (!t.data) return fail(MGN_ERR_ARG, "%s: null %s", who, name);
  if (t.ld < cols || !fits(rows, t.ld) || !aligned(t.data, elem(type)))
    return fail(MGN_ERR_ARG, "%s: %s: leading dimension %lld for %lld columns, or a misaligned pointer", who, name,
                (long long)t.ld, (long long)cols);
  return MGN_OK;
}

// An output may stand in an input's place row for row, not in another output's.
int check_in_place(const mgn_rows& out, const mgn_rows& in, int64_t rows, const char* who, const char* name) {
  if (rows > 1 && out.data == in.data && out.ld != in.ld)
    return fail(MGN_ERR_ARG, "%s: %s in place with another leading dimension (%lld, %lld)", who, name,
                (long long)out.ld, (long long)in.ld);
  return MGN_OK;
}

int check_mat4(const mgn_mat4* a, const char* who, const char* name) {
  if (!a) return fail(MGN_ERR_ARG, "%s: null %s", who, name);
  if (a->rows < 0 || a->cols < 0) return fail(MGN_ERR_ARG, "%s: %s: negative size", who, name);
  if (a->rows >= kMost || a->cols >= kMost) return fail(MGN_ERR_SHAPE, "%s: %s: 2^31 rows or columns", who, name);
  if (a->rows > 0 && a->cols > 0) {
    if (!a->q || !a->scale) return fail(MGN_ERR_ARG, "%s: %s: null numbers or scales", who, name);
    if (!aligned(a->q, 16) || !aligned(a->scale, 4) || (a->ld & 15) != 0 || a->ld < half_bytes(a->cols) ||
        a->ld >= (1 << 28))
      return fail(MGN_ERR_ARG, "%s: %s: rows have to start at multiples of 16 bytes, scales at 4, rows under 2^28 bytes apart (ld %lld, cols %lld)", who,
                  name, (long long)a->ld, (long long)a->cols);
  }
  return MGN_OK;
}

// c and the epilogue of a product of m x n.
// tiles: whether c may be cut into 128 x 128, 256 threads each.
int check_epilogue(const mgn_epilogue& ep, int32_t c_type, const void* c, int64_t ldc, int64_t m, int64_t n, bool tiles,
                   const char* who) {
  if (!c || ldc < n || !fits(m, ldc) || !aligned(c, elem(c_type)))
    return fail(MGN_ERR_ARG, "%s: null or misaligned c, or its leading dimension %lld", who, (long long)ldc);
  if (!aligned(ep.bias, 4)) return fail(MGN_ERR_ARG, "%s: misaligned bias", who);
  if (ep.act == MGN_ACT_RELU_GRAD && (!is_row_type(ep.aux_type) || !ep.aux || ep.ldaux < n || !fits(m, ep.ldaux) ||
                                      !aligned(ep.aux, elem(ep.aux_type))))
    return fail(MGN_ERR_ARG, "%s: null or misaligned aux, its type or leading dimension", who);
  if (tiles && ceil_div(m, 128) * ceil_div(n, 128) > (1 << 24) - 8)
    return fail(MGN_ERR_SHAPE, "%s: c of %lld x %lld is too large for one call", who, (long long)m, (long long)n);
  return MGN_OK;
}

int check_group_norm(const mgn_group_norm* op, const char* who) {
  if (!op) return fail(MGN_ERR_ARG, "%s: null op", who);
  if (op->rows < 0 || op->n_samples < 0) return fail(MGN_ERR_ARG, "%s: negative size", who);
  if (op->rows >= kMost) return fail(MGN_ERR_SHAPE, "%s: 2^31 rows", who);
  if (op->n_samples > (1 << 21)) return fail(MGN_ERR_SHAPE, "%s: over 2^21 samples", who);
  if (op->groups > 0 && op->n_samples * ceil_div(op->groups, 32) > (1 << 22))  // blocks of 512 threads
    return fail(MGN_ERR_SHAPE, "%s: %lld samples of %d groups", who, (long long)op->n_samples, op->groups);
  if (op->cols < 1 || op->cols > MGN_NORM_MAX_COLS)
    return fail(MGN_ERR_SHAPE, "%s: %d columns (1 to %d)", who, op->cols, MGN_NORM_MAX_COLS);
  if (op->groups < 1 || op->cols % op->groups != 0)
    return fail(MGN_ERR_ARG, "%s: %d groups do not divide %d columns", who, op->groups, op->cols);
  if (!is_row_type(op->type)) return fail(MGN_ERR_ARG, "%s: unknown type", who);
  if (op->act != MGN_ACT_NONE && op->act != MGN_ACT_RELU && op->act != MGN_ACT_SILU)
    return fail(MGN_ERR_ARG, "%s: unknown act %d", who, op->act);
  if (!(op->eps >= 1.1754944e-38f) || !std::isfinite(op->eps))
    return fail(MGN_ERR_ARG, "%s: eps has to be a positive normal number", who);
  if (!aligned(op->gamma, 4) || !aligned(op->beta, 4) || !aligned(op->sample_ptr, 4))
    return fail(MGN_ERR_ARG, "%s: misaligned gamma, beta or sample_ptr", who);
  if (!op->sample_ptr && (op->n_samples == 0 ? op->rows != 0 : op->rows % op->n_samples != 0))
    return fail(MGN_ERR_ARG, "%s: %lld rows in %lld samples need sample_ptr", who, (long long)op->rows,
                (long long)op->n_samples);
  return MGN_OK;
}

int check_norm_gate(const mgn_norm_gate* op, NormGate& a, const char* who) {
  if (!op) return fail(MGN_ERR_ARG, "%s: null op", who);
  if (op->rows < 0 || op->n_gates < 0) return fail(MGN_ERR_ARG, "%s: negative size", who);
  if (op->rows >= kMost || op->n_gates >= kMost) return fail(MGN_ERR_SHAPE, "%s: 2^31 rows or gates", who);
  if (op->cols < 1 || op->cols > MGN_NORM_MAX_COLS)
    return fail(MGN_ERR_SHAPE, "%s: %d columns (1 to %d)", who, op->cols, MGN_NORM_MAX_COLS);
  if (!is_row_type(op->x_type) || !is_row_type(op->b_type)) return fail(MGN_ERR_ARG, "%s: unknown type", who);
  if (op->post < MGN_NORM_NONE || op->post > MGN_NORM_RMS || op->pre < MGN_NORM_NONE || op->pre > MGN_NORM_RMS)
    return fail(MGN_ERR_ARG, "%s: unknown norm", who);
  if (!(op->eps >= 1.1754944e-38f) || !std::isfinite(op->eps))
    return fail(MGN_ERR_ARG, "%s: eps has to be a positive normal number", who);
  if (op->n_gates > 0 && !op->gate) return fail(MGN_ERR_ARG, "%s: null gate", who);
  if (op->gate_ptr && op->n_gates == 0) return fail(MGN_ERR_ARG, "%s: gate_ptr without gates", who);
  if (op->gate_ptr)
    a.gmode = kGateGroup;
  else if (op->n_gates == 0)
    a.gmode = kGateNone;
  else if (op->n_gates == 1)
    a.gmode = kGateOne;
  else if (op->n_gates == op->rows)
    a.gmode = kGateRow;
  else
    return fail(MGN_ERR_ARG, "%s: %lld gates for %lld rows need gate_ptr", who, (long long)op->n_gates,
                (long long)op->rows);
  a.op = *op;
  // vectors of a norm that is not there
  if (op->post == MGN_NORM_NONE) a.op.post_gamma = a.op.post_beta = nullptr;
  if (op->pre == MGN_NORM_NONE) a.op.pre_gamma = a.op.pre_beta = nullptr;
  return MGN_OK;
}

}  // namespace
}  // namespace mgn

using namespace mgn;

extern "C" {

int mgn_quant8_workspace(int64_t rows, int64_t cols, size_t* ws_bytes) {
  if (!ws_bytes || rows < 0 || cols < 0) return fail(MGN_ERR_ARG, "mgn_quant8_workspace: null or negative argument");
  if (rows >= kMost || cols >= kMost) return fail(MGN_ERR_SHAPE, "mgn_quant8_workspace: 2^31 rows or columns");
  *ws_bytes = (size_t)ceil_div(rows, 128) * (size_t)cols * 4;
  return MGN_OK;
}

int mgn_quant8(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx, int32_t format,
               int32_t block_rows, uint8_t* q, int64_t ldq, float* scale, uint8_t* qt, int64_t ldqt, float* scale_t,
               float* colsum, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "mgn_quant8";
  size_t need = 0;
  int rc = mgn_quant8_workspace(rows, cols, &need);
  if (rc != MGN_OK) return rc;
  if (!is_row_type(x_type)) return fail(MGN_ERR_ARG, "%s: unknown type %d", who, x_type);
  if (!is_format(format)) return fail(MGN_ERR_ARG, "%s: unknown 8-bit format %d", who, format);
  if (block_rows != 1 && block_rows != 128) return fail(MGN_ERR_ARG, "%s: blocks of %d rows (1 or 128)", who, block_rows);
  if ((!q) != (!scale) || (!qt) != (!scale_t)) return fail(MGN_ERR_ARG, "%s: numbers without scales, or scales alone", who);
  if (cols == 0) return MGN_OK;
  if (rows > 0 && (!x || ldx < cols || !fits(rows, ldx) || !aligned(x, elem(x_type))))
    return fail(MGN_ERR_ARG, "%s: null or misaligned x, or its leading dimension %lld", who, (long long)ldx);
  if (q && (!aligned(q, 16) || (ldq & 15) != 0 || ldq < up16(cols) || !fits(rows, ldq)))
    return fail(MGN_ERR_ARG, "%s: rows of q have to start at multiples of 16 bytes", who);
  if (qt && (!aligned(qt, 16) || (ldqt & 15) != 0 || ldqt < up16(rows) || !fits(cols, ldqt)))
    return fail(MGN_ERR_ARG, "%s: rows of qt have to start at multiples of 16 bytes", who);
  if (!aligned(scale, 4) || !aligned(scale_t, 4) || !aligned(colsum, 4))
    return fail(MGN_ERR_ARG, "%s: misaligned scales or sums", who);
  if (ceil_div(rows, 16) * ceil_div(cols, 128) >= kMost)
    return fail(MGN_ERR_SHAPE, "%s: x of %lld x %lld is too large for one call", who, (long long)rows, (long long)cols);
  if (colsum && need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  if (!q && !qt && !colsum) return MGN_OK;
  const Quant8 a = {x, x_type, format, block_rows, rows, cols, ldx, q, qt, ldq, ldqt, scale, scale_t, colsum, (float*)ws,
                    accumulate};
  return launched(launch_quant8(a, (hipStream_t)stream), who);
}

int mgn_matmul8_workspace(int64_t a_rows, int64_t b_rows, int64_t cols, size_t* ws_bytes) {
  if (!ws_bytes || a_rows < 0 || b_rows < 0 || cols < 0)
    return fail(MGN_ERR_ARG, "mgn_matmul8_workspace: null or negative argument");
  if (a_rows >= kMost || b_rows >= kMost || cols >= kMost)
    return fail(MGN_ERR_SHAPE, "mgn_matmul8_workspace: 2^31 rows or columns");
  *ws_bytes = matmul8_workspace(a_rows, b_rows, cols);
  return MGN_OK;
}

int mgn_matmul8(const mgn_mat8* a, const mgn_mat8* b, const mgn_epilogue* ep, int32_t c_type, void* c, int64_t ldc,
                void* ws, size_t ws_bytes, void* stream) {
  const char* who = "mgn_matmul8";
  int rc;
  if ((rc = check_mat8(a, who, "a")) != MGN_OK || (rc = check_mat8(b, who, "b")) != MGN_OK) return rc;
  if (a->cols != b->cols)
    return fail(MGN_ERR_SHAPE, "%s: a has %lld columns, b %lld", who, (long long)a->cols, (long long)b->cols);
  if (!is_row_type(c_type)) return fail(MGN_ERR_ARG, "%s: unknown type %d of c", who, c_type);
  Matmul8 m = {*a, *b, {}, c_type, c, ldc, (float*)ws};
  if (ep) m.ep = *ep;
  if (m.ep.act < MGN_ACT_NONE || m.ep.act > MGN_ACT_RELU_GRAD) return fail(MGN_ERR_ARG, "%s: unknown act %d", who, m.ep.act);
  if (a->rows == 0 || b->rows == 0) return MGN_OK;
  if ((rc = check_epilogue(m.ep, c_type, c, ldc, a->rows, b->rows, a->rows > 32, who)) != MGN_OK) return rc;
  const size_t need = matmul8_workspace(a->rows, b->rows, a->cols);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  return launched(launch_matmul8(m, (hipStream_t)stream), who);
}

int mgn_norm_gate_forward(const mgn_norm_gate* op, mgn_rows x, mgn_rows b, mgn_rows y, mgn_rows z, float* stats,
                          void* stream) {
  const char* who = "mgn_norm_gate_forward";
  NormGate a = {};
  int rc = check_norm_gate(op, a, who);
  if (rc != MGN_OK) return rc;
  if (op->rows == 0) return MGN_OK;
  if ((rc = check_rows(x, op->rows, op->cols, op->x_type, who, "x")) != MGN_OK ||
      (rc = check_rows(b, op->rows, op->cols, op->b_type, who, "b")) != MGN_OK ||
      (rc = check_rows(y, op->rows, op->cols, op->x_type, who, "y")) != MGN_OK)
    return rc;
  if (op->pre != MGN_NORM_NONE && (rc = check_rows(z, op->rows, op->cols, op->b_type, who, "z")) != MGN_OK) return rc;
  if (!aligned(stats, 16)) return fail(MGN_ERR_ARG, "%s: stats have to be 16-byte aligned", who);
  if (op->pre != MGN_NORM_NONE && y.data == z.data) return fail(MGN_ERR_ARG, "%s: y and z are the same", who);
  if ((rc = check_in_place(y, x, op->rows, who, "y")) != MGN_OK ||
      (op->pre != MGN_NORM_NONE && (rc = check_in_place(z, b, op->rows, who, "z")) != MGN_OK))
    return rc;
  a.x = x;
  a.b = b;
  a.y = y;
  a.z = z;
  a.stats = stats;
  return launched(launch_norm_gate_forward(a, (hipStream_t)stream), who);
}

int mgn_norm_gate_workspace(int64_t rows, int32_t cols, size_t* ws_bytes) {
  if (!ws_bytes || rows < 0) return fail(MGN_ERR_ARG, "mgn_norm_gate_workspace: null or negative argument");
  if (rows >= kMost || cols < 1 || cols > MGN_NORM_MAX_COLS)
    return fail(MGN_ERR_SHAPE, "mgn_norm_gate_workspace: 2^31 rows, or %d columns (1 to %d)", cols, MGN_NORM_MAX_COLS);
  const NormPlan p = norm_plan(rows, cols, true);
  *ws_bytes = (size_t)(p.blocks * 5 + p.walkers * 2) * (size_t)cols * 4;
  return MGN_OK;
}

int mgn_norm_gate_backward(const mgn_norm_gate* op, mgn_rows x, mgn_rows b, const float* stats, mgn_rows dy,
                           mgn_rows dz, mgn_rows dx, mgn_rows db, const mgn_norm_gate_grads* grads, void* ws,
                           size_t ws_bytes, void* stream) {
  const char* who = "mgn_norm_gate_backward";
  NormGate a = {};
  int rc = check_norm_gate(op, a, who);
  if (rc != MGN_OK) return rc;
  if (grads) a.grads = *grads;
  if (op->post == MGN_NORM_NONE) a.grads.post_gamma = a.grads.post_beta = nullptr;
  if (op->pre == MGN_NORM_NONE) a.grads.pre_gamma = a.grads.pre_beta = nullptr;
  if (op->n_gates == 0) a.grads.gate = nullptr;
  if (!aligned(a.grads.post_gamma, 4) || !aligned(a.grads.post_beta, 4) || !aligned(a.grads.pre_gamma, 4) ||
      !aligned(a.grads.pre_beta, 4) || !aligned(a.grads.gate, 4))
    return fail(MGN_ERR_ARG, "%s: misaligned parameter gradients", who);
  if (op->rows > 0) {
    if ((rc = check_rows(x, op->rows, op->cols, op->x_type, who, "x")) != MGN_OK ||
        (rc = check_rows(b, op->rows, op->cols, op->b_type, who, "b")) != MGN_OK ||
        (rc = check_rows(dx, op->rows, op->cols, op->x_type, who, "dx")) != MGN_OK ||
        (rc = check_rows(db, op->rows, op->cols, op->b_type, who, "db")) != MGN_OK)
      return rc;
    if (dy.data && (rc = check_rows(dy, op->rows, op->cols, op->x_type, who, "dy")) != MGN_OK) return rc;
    if (dz.data && (rc = check_rows(dz, op->rows, op->cols, op->b_type, who, "dz")) != MGN_OK) return rc;
    if (op->pre == MGN_NORM_NONE && dz.data) return fail(MGN_ERR_ARG, "%s: dz without a norm before the next block", who);
    if (!stats || !aligned(stats, 16)) return fail(MGN_ERR_ARG, "%s: null or misaligned stats", who);
  }
  size_t need = 0;
  if ((rc = mgn_norm_gate_workspace(op->rows, op->cols, &need)) != MGN_OK) return rc;
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  if (op->rows > 0) {
    if (dx.data == db.data) return fail(MGN_ERR_ARG, "%s: dx and db are the same", who);
    if ((rc = check_in_place(dx, x, op->rows, who, "dx")) != MGN_OK ||
        (rc = check_in_place(dx, dy, op->rows, who, "dx")) != MGN_OK ||
        (rc = check_in_place(db, b, op->rows, who, "db")) != MGN_OK ||
        (rc = check_in_place(db, dz, op->rows, who, "db")) != MGN_OK)
      return rc;
  }
  const NormPlan p = norm_plan(op->rows, op->cols, true);
  a.x = x;
  a.b = b;
  a.stats = const_cast<float*>(stats);
  a.dy = dy;
  a.dz = dz;
  a.dx = dx;
  a.db = db;
  a.part = (float*)ws;
  a.slots = a.part + p.blocks * 5 * op->cols;
  return launched(launch_norm_gate_backward(a, (hipStream_t)stream), who);
}

int mgn_quant4_workspace(int64_t rows, int64_t cols, size_t* ws_bytes) {
  if (!ws_bytes || rows < 0 || cols < 0) return fail(MGN_ERR_ARG, "mgn_quant4_workspace: null or negative argument");
  if (rows >= kMost || cols >= kMost) return fail(MGN_ERR_SHAPE, "mgn_quant4_workspace: 2^31 rows or columns");
  *ws_bytes = (size_t)ceil_div(rows, 128) * (size_t)cols * 4;
  return MGN_OK;
}

int mgn_quant4(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx, uint8_t* q, int64_t ldq,
               uint8_t* scale, uint8_t* qt, int64_t ldqt, uint8_t* scale_t, float* colsum, int32_t accumulate, void* ws,
               size_t ws_bytes, void* stream) {
  const char* who = "mgn_quant4";
  size_t need = 0;
  int rc = mgn_quant4_workspace(rows, cols, &need);
  if (rc != MGN_OK) return rc;
  if (!is_row_type(x_type)) return fail(MGN_ERR_ARG, "%s: unknown type %d", who, x_type);
  if ((!q) != (!scale) || (!qt) != (!scale_t)) return fail(MGN_ERR_ARG, "%s: numbers without scales, or scales alone", who);
  if (cols == 0) return MGN_OK;
  if (rows > 0 && (!x || ldx < cols || !fits(rows, ldx) || !aligned(x, elem(x_type))))
    return fail(MGN_ERR_ARG, "%s: null or misaligned x, or its leading dimension %lld", who, (long long)ldx);
  if (q && (!aligned(q, 16) || (ldq & 15) != 0 || ldq < half_bytes(cols) || !fits(rows, ldq)))
    return fail(MGN_ERR_ARG, "%s: rows of q have to start at multiples of 16 bytes", who);
  if (qt && (!aligned(qt, 16) || (ldqt & 15) != 0 || ldqt < half_bytes(rows) || !fits(cols, ldqt)))
    return fail(MGN_ERR_ARG, "%s: rows of qt have to start at multiples of 16 bytes", who);
  if (!aligned(scale, 4) || !aligned(scale_t, 4) || !aligned(colsum, 4))
    return fail(MGN_ERR_ARG, "%s: misaligned scales or sums", who);
  if (q && (q == qt || scale == scale_t)) return fail(MGN_ERR_ARG, "%s: x and its transpose in the same place", who);
  if (ceil_div(rows, 16) * ceil_div(cols, 128) >= kMost)
    return fail(MGN_ERR_SHAPE, "%s: x of %lld x %lld is too large for one call", who, (long long)rows, (long long)cols);
  if (colsum && need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  if (!q && !qt && !colsum) return MGN_OK;
  const Quant4 a = {x, x_type, rows, cols, ldx, q, qt, ldq, ldqt, scale, scale_t, colsum, (float*)ws, accumulate};
  return launched(launch_quant4(a, (hipStream_t)stream), who);
}

int mgn_dequant4(const mgn_mat4* a, int32_t y_type, void* y, int64_t ldy, void* stream) {
  const char* who = "mgn_dequant4";
  int rc = check_mat4(a, who, "a");
  if (rc != MGN_OK) return rc;
  if (!is_row_type(y_type)) return fail(MGN_ERR_ARG, "%s: unknown type %d", who, y_type);
  if (a->rows == 0 || a->cols == 0) return MGN_OK;
  if (!y || ldy < a->cols || !fits(a->rows, ldy) || !aligned(y, elem(y_type)))
    return fail(MGN_ERR_ARG, "%s: null or misaligned y, or its leading dimension %lld", who, (long long)ldy);
  if (ceil_div(a->rows, 8) * ceil_div(a->cols, 128) >= kMost)
    return fail(MGN_ERR_SHAPE, "%s: a of %lld x %lld is too large for one call", who, (long long)a->rows,
                (long long)a->cols);
  const Dequant4 d = {*a, y_type, y, ldy};
  return launched(launch_dequant4(d, (hipStream_t)stream), who);
}

int mgn_matmul4_workspace(int64_t a_rows, int64_t b_rows, int64_t cols, size_t* ws_bytes) {
  if (!ws_bytes || a_rows < 0 || b_rows < 0 || cols < 0)
    return fail(MGN_ERR_ARG, "mgn_matmul4_workspace: null or negative argument");
  if (a_rows >= kMost || b_rows >= kMost || cols >= kMost)
    return fail(MGN_ERR_SHAPE, "mgn_matmul4_workspace: 2^31 rows or columns");
  *ws_bytes = matmul4_workspace(a_rows, b_rows, cols);
  return MGN_OK;
}

int mgn_matmul4(const mgn_mat4* a, const mgn_mat4* b, const mgn_epilogue* ep, int32_t c_type, void* c, int64_t ldc,
                void* ws, size_t ws_bytes, void* stream) {
  const char* who = "mgn_matmul4";
  int rc;
  if ((rc = check_mat4(a, who, "a")) != MGN_OK || (rc = check_mat4(b, who, "b")) != MGN_OK) return rc;
  if (a->cols != b->cols)
    return fail(MGN_ERR_SHAPE, "%s: a has %lld columns, b %lld", who, (long long)a->cols, (long long)b->cols);
  if (!is_row_type(c_type)) return fail(MGN_ERR_ARG, "%s: unknown type %d of c", who, c_type);
  Matmul4 m = {*a, *b, {}, c_type, c, ldc, (float*)ws};
  if (ep) m.ep = *ep;
  if (m.ep.act < MGN_ACT_NONE || m.ep.act > MGN_ACT_RELU_GRAD) return fail(MGN_ERR_ARG, "%s: unknown act %d", who, m.ep.act);
  if (a->rows == 0 || b->rows == 0) return MGN_OK;
  if ((rc = check_epilogue(m.ep, c_type, c, ldc, a->rows, b->rows, true, who)) != MGN_OK) return rc;
  const size_t need = matmul4_workspace(a->rows, b->rows, a->cols);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  return launched(launch_matmul4(m, (hipStream_t)stream), who);
}

int mgn_group_norm_workspace(const mgn_group_norm* op, int32_t backward, size_t* ws_bytes) {
  const char* who = "mgn_group_norm_workspace";
  if (!ws_bytes) return fail(MGN_ERR_ARG, "%s: null argument", who);
  int rc = check_group_norm(op, who);
  if (rc != MGN_OK) return rc;
  *ws_bytes = group_norm_workspace(*op, backward != 0);
  return MGN_OK;
}

int mgn_group_norm_forward(const mgn_group_norm* op, mgn_rows x, mgn_rows y, float* stats, void* ws, size_t ws_bytes,
                           void* stream) {
  const char* who = "mgn_group_norm_forward";
  int rc = check_group_norm(op, who);
  if (rc != MGN_OK) return rc;
  if (op->rows > 0) {
    if ((rc = check_rows(x, op->rows, op->cols, op->type, who, "x")) != MGN_OK ||
        (rc = check_rows(y, op->rows, op->cols, op->type, who, "y")) != MGN_OK ||
        (rc = check_in_place(y, x, op->rows, who, "y")) != MGN_OK)
      return rc;
  }
  if (!aligned(stats, 8)) return fail(MGN_ERR_ARG, "%s: stats have to be 8-byte aligned", who);
  const size_t need = group_norm_workspace(*op, false);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  GroupNorm a = {};
  a.op = *op;
  a.x = x;
  a.y = y;
  a.stats = stats;
  a.ws = ws;
  return launched(launch_group_norm_forward(a, (hipStream_t)stream), who);
}

int mgn_group_norm_backward(const mgn_group_norm* op, mgn_rows x, const float* stats, mgn_rows dy, mgn_rows dx,
                            float* dgamma, float* dbeta, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "mgn_group_norm_backward";
  int rc = check_group_norm(op, who);
  if (rc != MGN_OK) return rc;
  if (op->rows > 0) {
    if ((rc = check_rows(x, op->rows, op->cols, op->type, who, "x")) != MGN_OK ||
        (rc = check_rows(dy, op->rows, op->cols, op->type, who, "dy")) != MGN_OK ||
        (rc = check_rows(dx, op->rows, op->cols, op->type, who, "dx")) != MGN_OK ||
        (rc = check_in_place(dx, x, op->rows, who, "dx")) != MGN_OK ||
        (rc = check_in_place(dx, dy, op->rows, who, "dx")) != MGN_OK)
      return rc;
  }
  if (op->n_samples > 0 && (!stats || !aligned(stats, 8)))
    return fail(MGN_ERR_ARG, "%s: null or misaligned stats", who);
  if (!aligned(dgamma, 4) || !aligned(dbeta, 4)) return fail(MGN_ERR_ARG, "%s: misaligned parameter gradients", who);
  if (dgamma && dgamma == dbeta) return fail(MGN_ERR_ARG, "%s: dgamma and dbeta are the same", who);
  const size_t need = group_norm_workspace(*op, true);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  GroupNorm a = {};
  a.op = *op;
  a.x = x;
  a.dy = dy;
  a.dx = dx;
  a.stats = const_cast<float*>(stats);
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  a.accumulate = accumulate;
  a.ws = ws;
  return launched(launch_group_norm_backward(a, (hipStream_t)stream), who);
}

int32_t mgn_grad_piece(void) { return kPiece; }

int mgn_grad_pieces(const mgn_tensor* t, int64_t n, mgn_piece* pieces, int64_t* n_pieces) {
  const char* who = "mgn_grad_pieces";
  if (n < 0 || (n > 0 && !t) || !n_pieces) return fail(MGN_ERR_ARG, "%s: null or negative argument", who);
  // bytes that are read, and those that are written, by tensor
  struct Span {
    uintptr_t lo, hi;
    int64_t i;
    bool out;
  };
  int64_t count = 0;
  try {
    std::vector<Span> spans;
    for (int64_t i = 0; i < n; ++i) {
      const mgn_tensor& x = t[i];
      if (x.n < 0) return fail(MGN_ERR_ARG, "%s: tensor %lld: negative size", who, (long long)i);
      if (!is_row_type(x.in_type) || (x.out && !is_row_type(x.out_type)))
        return fail(MGN_ERR_ARG, "%s: tensor %lld: unknown type", who, (long long)i);
      if (x.n == 0) continue;
      if (!x.in || !aligned(x.in, elem(x.in_type)) || !aligned(x.out, elem(x.out_type)) || !fits(x.n, 4))
        return fail(MGN_ERR_ARG, "%s: tensor %lld: null or misaligned, or too large", who, (long long)i);
      if (x.in == x.out && x.in_type != x.out_type)
        return fail(MGN_ERR_ARG, "%s: tensor %lld: clipped in place into another type", who, (long long)i);
      count += ceil_div(x.n, kPiece);
      if (count >= kMost) return fail(MGN_ERR_SHAPE, "%s: 2^31 pieces", who);
      const uintptr_t in = (uintptr_t)x.in, out = (uintptr_t)x.out;
      spans.push_back({in, in + (uintptr_t)(x.n * elem(x.in_type)), i, false});
      if (x.out) spans.push_back({out, out + (uintptr_t)(x.n * elem(x.out_type)), i, true});
    }
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    // the furthest end so far of what is written, and of what is read
    const Span* written = nullptr;
    const Span *read = nullptr, *second = nullptr;  // of two tensors, so that a tensor's own place can be told
    for (const Span& s : spans) {
      auto same = [&](const Span* o) { return o->i == s.i && t[s.i].in == t[s.i].out; };
      if ((written && written->hi > s.lo && !(same(written) && !s.out)) ||
          (s.out && read && read->hi > s.lo && !same(read)) || (s.out && second && second->hi > s.lo && !same(second)))
        return fail(MGN_ERR_ARG, "%s: the place of a clipped gradient overlaps another tensor's (%lld)", who, (long long)s.i);
      if (s.out) {
        if (!written || s.hi > written->hi) written = &s;
      } else if (!read || s.hi > read->hi) {
        second = read;
        read = &s;
      } else if (!second || s.hi > second->hi) {
        second = &s;
      }
    }
  } catch (const std::bad_alloc&) {
    return fail(MGN_ERR_NOMEM, "%s: host memory", who);
  }
  if (pieces) {
    int64_t k = 0;
    for (int64_t i = 0; i < n; ++i) {
      const mgn_tensor& x = t[i];
      for (int64_t at = 0; at < x.n; at += kPiece) {
        mgn_piece& p = pieces[k++];
        p.in = (const char*)x.in + at * elem(x.in_type);
        p.out = x.out ? (char*)x.out + at * elem(x.out_type) : nullptr;
        p.n = (int32_t)std::min<int64_t>(kPiece, x.n - at);
        p.types = x.in_type + (x.out ? 2 * x.out_type : 0);
      }
    }
  }
  *n_pieces = count;
  return MGN_OK;
}

int mgn_grad_norm_workspace(int64_t n_pieces, size_t* ws_bytes) {
  if (!ws_bytes || n_pieces < 0) return fail(MGN_ERR_ARG, "mgn_grad_norm_workspace: null or negative argument");
  *ws_bytes = grad_norm_workspace(n_pieces);
  return MGN_OK;
}

namespace {
int grad_clip(GradClip a, void* ws, size_t ws_bytes, void* stream, const char* who) {
  if (a.n < 0 || a.n >= kMost || (a.n > 0 && (!a.pieces || !aligned(a.pieces, 8))))
    return fail(MGN_ERR_ARG, "%s: null or misaligned pieces, or their number", who);
  if (!a.norm || !aligned(a.norm, 4)) return fail(MGN_ERR_ARG, "%s: null or misaligned norm", who);
  const size_t need = a.given ? 0 : grad_norm_workspace(a.n);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16)))
    return fail(MGN_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  a.part = (double*)ws;
  return launched(launch_grad_clip(a, (hipStream_t)stream), who);
}
}  // namespace

int mgn_grad_norm(const mgn_piece* pieces, int64_t n_pieces, float* norm, void* ws, size_t ws_bytes, void* stream) {
  return grad_clip({pieces, n_pieces, 0.0, norm, false, false, nullptr}, ws, ws_bytes, stream, "mgn_grad_norm");
}

int mgn_grad_clip(const mgn_piece* pieces, int64_t n_pieces, double max_norm, float* norm, int32_t given, void* ws,
                  size_t ws_bytes, void* stream) {
  if (!(max_norm >= 0.0)) return fail(MGN_ERR_ARG, "mgn_grad_clip: a largest norm of %g", max_norm);
  return grad_clip({pieces, n_pieces, max_norm, norm, given != 0, true, nullptr}, ws, ws_bytes, stream, "mgn_grad_clip");
}

}  // extern "C"
