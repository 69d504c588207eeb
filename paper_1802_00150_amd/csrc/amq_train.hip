// C ABI of the training operators (declared in include/amq.h): argument validation on the host, then kernel launches on
// the caller's stream.
#include "amq_train.h"

#include <algorithm>
#include <memory>
#include <new>

#include "../../include/amq.h"

namespace {

bool type_ok(int t) { return t == AMQ_F32 || t == AMQ_BF16 || t == AMQ_F16; }
size_t size_of(int t) { return t == AMQ_F32 ? 4 : 2; }
// a tensor of elements of `type` lies on its elements
bool on_elements(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (size_of(type) - 1)) == 0; }
bool workspace_ok(const void* ws, size_t bytes, size_t need) {
  return need == 0 || (ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0 && bytes >= need);
}

// Limits of the operators below: rows and columns, row strides (a tile's rows lie within 32-bit byte offsets), and what the
// launch grids can count.
constexpr int64_t kMaxSize = 1 << 20, kMaxRows = 1 << 22, kMaxStride = 1 << 22, kMaxEntries = 1LL << 38;

bool linear_sizes_ok(int64_t rows, int64_t k, int64_t n) { return rows > 0 && k > 0 && n > 0; }
bool linear_sizes_supported(int64_t rows, int64_t k, int64_t n) {
  return rows <= kMaxRows && k <= kMaxSize && n <= kMaxSize && rows * k <= kMaxEntries && rows * n <= kMaxEntries && n * k <= kMaxEntries;
}

// ---- overlap.  A result's entries are written while other workgroups still read the operands.
// A matrix in memory, in bytes: `rows` pieces of `width`, `step` apart.  (p null: none.)
struct Extent {
  uintptr_t p;
  int64_t rows, width, step;
};
Extent matrix(const void* p, int64_t rows, int64_t n, int64_t ld, int type) {
  const int64_t size = (int64_t)size_of(type);
  return {reinterpret_cast<uintptr_t>(p), rows, n * size, (rows > 1 ? ld : n) * size};
}
Extent vector(const void* p, int64_t n, int type) { return matrix(p, 1, n, n, type); }
int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }
// Whether the two have a byte in common.  Columns of one wider matrix (equal steps) take one division, anything else that may meet a division
// per row.
bool overlap(const Extent& a, const Extent& b) {
  if (!a.p || !b.p) return false;
  const int64_t from = (int64_t)(b.p - a.p);  // where b begins, with a at 0
  if (from >= (a.rows - 1) * a.step + a.width || from + (b.rows - 1) * b.step + b.width <= 0) return false;
  if (a.step == b.step && a.rows > 1 && b.rows > 1) {
    // row i of a meets row i + d of b where -b.width < from + d step < a.width
    const int64_t d = floor_div(-b.width - from, a.step) + 1;
    const int64_t last = floor_div(a.width - 1 - from, a.step);
    return d <= last && d < b.rows && last > -a.rows;
  }
  const bool swap = a.rows > b.rows;
  const Extent &few = swap ? b : a, &many = swap ? a : b;
  const int64_t begin = swap ? -from : from;  // of `many`, with `few` at 0
  for (int64_t i = 0; i < few.rows; ++i) {
    const int64_t at = i * few.step - begin;  // of the row, with `many` at 0
    // row j of `many` meets it where at - many.width < j step < at + few.width
    const int64_t j = floor_div(at - many.width, many.step) + 1;
    if ((j > 0 ? j : 0) * many.step < at + few.width && (j > 0 ? j : 0) < many.rows) return true;
  }
  return false;
}
// The same entries, one by one.
bool same(const Extent& a, const Extent& b) { return a.p == b.p && a.rows == b.rows && a.width == b.width && a.step == b.step; }
template <int N>
bool meets(const Extent& result, const Extent (&others)[N]) {
  for (const Extent& o : others)
    if (overlap(result, o)) return true;
  return false;
}

// A tensor [steps][B][n]: `count` matrices, `apart` bytes from one to the next.
struct Volume {
  Extent matrix;
  int64_t count, apart;
};
Volume volume(const void* p, int64_t steps, int64_t B, int64_t n, int64_t step, int64_t batch, int type) {
  const int64_t size = (int64_t)size_of(type), width = n * size;
  int64_t rows[2] = {steps, B}, by[2] = {step * size, batch * size};
  for (int i = 0; i < 2; ++i)
    if (rows[i] == 1 || by[i] == 0) rows[i] = 1, by[i] = width;  // (the same rows again)
  const int large = by[0] >= by[1] ? 0 : 1, small = 1 - large;
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  if (rows[large] == 1) return {{at, rows[small], width, by[small]}, 1, 0};
  if (rows[small] == 1) return {{at, rows[large], width, by[large]}, 1, 0};
  if (by[large] == rows[small] * by[small]) return {{at, rows[0] * rows[1], width, by[small]}, 1, 0};
  // matrices that lie one behind the other meet few others; many of them are taken the other way
  const int outer = rows[large] <= 4096 || rows[large] <= rows[small] ? large : small, inner = 1 - outer;
  return {{at, rows[inner], width, by[inner]}, rows[outer], by[outer]};
}
int64_t extent_bytes(const Extent& e) { return (e.rows - 1) * e.step + e.width; }
bool overlap(const Volume& a, const Volume& b) {
  if (!a.matrix.p || !b.matrix.p) return false;
  const int64_t room_a = extent_bytes(a.matrix), room_b = extent_bytes(b.matrix);
  for (int64_t i = 0; i < a.count; ++i) {
    const Extent m{a.matrix.p + i * a.apart, a.matrix.rows, a.matrix.width, a.matrix.step};
    const int64_t from = (int64_t)(m.p - b.matrix.p);
    int64_t j = b.count > 1 ? floor_div(from - room_b, b.apart) : 0;  // the first that may reach m
    for (j = j > 0 ? j : 0; j < b.count && j * b.apart < from + room_a; ++j)
      if (overlap(m, {b.matrix.p + j * b.apart, b.matrix.rows, b.matrix.width, b.matrix.step})) return true;
  }
  return false;
}
Volume of(const Extent& e) { return {e, 1, 0}; }
template <int N>
bool meets(const Volume& result, const Volume (&others)[N]) {
  for (const Volume& o : others)
    if (overlap(result, o)) return true;
  return false;
}

// Tensors [steps][B][n] of a recurrence: rows are told apart by steps in batch entries or by batch entries in steps.
bool apart(int64_t steps, int64_t B, int64_t n, int64_t step, int64_t batch) {
  if (steps == 1) return B == 1 || batch >= n;
  if (B == 1) return step >= n;
  return (batch >= n && step >= (B - 1) * batch + n) || (step >= n && batch >= (steps - 1) * step + n);
}
bool recurrence_sizes_ok(int64_t steps, int64_t B, int64_t n) { return steps > 0 && B > 0 && n > 0; }
bool recurrence_sizes_supported(int64_t steps, int64_t B, int64_t n) {
  return steps <= (1 << 24) && B <= (1 << 22) && n <= kMaxSize && B * n <= (1 << 30);
}
bool strides_ok(int64_t step, int64_t batch) { return step >= 0 && batch >= 0; }
bool strides_supported(int64_t step, int64_t batch) { return step <= (1LL << 36) && batch <= (1LL << 36); }
int64_t states_of(int64_t steps) { return (steps - 1) / AMQ_STATE_STEPS; }

// Limits of the joined norms: a row stays in the registers of one workgroup.
constexpr int64_t kMaxJoined = 16384;
bool gate_act_ok(int act) { return act == AMQ_ACT_NONE || act == AMQ_ACT_SIGMOID || act == AMQ_ACT_SILU; }

struct Interval {
  uintptr_t begin, end;
  int64_t index;
};

}  // namespace

extern "C" {

int amq_layer_norm(const void* x, int64_t ld_x, int64_t rows, int64_t n, int type, const void* weight, const void* bias,
                   int param_type, float eps, void* y, int64_t ld_y, float* mean, float* rstd, void* stream) {
  if (!x || !y || !type_ok(type) || (param_type != AMQ_F32 && param_type != type)) return AMQ_ERR_INVALID;
  if (rows <= 0 || n <= 0 || ld_x < n || ld_y < n || !(eps >= 0.0f)) return AMQ_ERR_INVALID;
  if (!on_elements(x, type) || !on_elements(y, type) || !on_elements(weight, param_type) || !on_elements(bias, param_type) ||
      !on_elements(mean, AMQ_F32) || !on_elements(rstd, AMQ_F32))
    return AMQ_ERR_INVALID;
  if (rows > 0x7fffffffLL || n > kMaxSize) return AMQ_ERR_UNSUPPORTED;
  const Extent in = matrix(x, rows, n, ld_x, type), out = matrix(y, rows, n, ld_y, type), m = vector(mean, rows, AMQ_F32), r = vector(rstd, rows, AMQ_F32);
  const Extent params[] = {vector(weight, n, param_type), vector(bias, n, param_type)};
  if ((!same(in, out) && overlap(in, out)) || meets(out, params) || meets(m, params) || meets(r, params) || meets(m, {in, out, r}) || meets(r, {in, out}))
    return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_norm({x, weight, bias, y, mean, rstd, rows, ld_x, ld_y, (int)n, type, param_type, eps},
                                         static_cast<hipStream_t>(stream)));
}

size_t amq_layer_norm_backward_workspace_bytes(int64_t rows, int64_t n) {
  if (rows <= 0 || n <= 0 || rows > 0x7fffffffLL || n > kMaxSize) return 0;
  return (sizeof(float) * 2 * (size_t)amq::norm_grad_parts(rows, (int)n) * n + 255) & ~size_t(255);
}

int amq_layer_norm_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, int64_t rows, int64_t n, int type,
                            const void* weight, int param_type, const float* mean, const float* rstd, void* dx,
                            int64_t ld_dx, void* dweight, void* dbias, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (!dy || !x || !mean || !rstd || !dx || !type_ok(type) || (param_type != AMQ_F32 && param_type != type)) return AMQ_ERR_INVALID;
  if (rows <= 0 || n <= 0 || ld_dy < n || ld_x < n || ld_dx < n) return AMQ_ERR_INVALID;
  if (!on_elements(dy, type) || !on_elements(x, type) || !on_elements(dx, type) || !on_elements(weight, param_type) ||
      !on_elements(dweight, param_type) || !on_elements(dbias, param_type) || !on_elements(mean, AMQ_F32) || !on_elements(rstd, AMQ_F32))
    return AMQ_ERR_INVALID;
  if (rows > 0x7fffffffLL || n > kMaxSize) return AMQ_ERR_UNSUPPORTED;
  const Extent d = matrix(dy, rows, n, ld_dy, type), in = matrix(x, rows, n, ld_x, type), out = matrix(dx, rows, n, ld_dx, type);
  const Extent m = vector(mean, rows, AMQ_F32), r = vector(rstd, rows, AMQ_F32), w = vector(weight, n, param_type);
  const Extent dw = vector(dweight, n, param_type), db = vector(dbias, n, param_type);
  if ((!same(d, out) && overlap(d, out)) || (!same(in, out) && overlap(in, out)) || meets(out, {m, r, w, dw, db}) || meets(dw, {d, in, m, r, w, db}) ||
      meets(db, {d, in, m, r, w}))
    return AMQ_ERR_INVALID;
  if ((dweight || dbias) && !workspace_ok(workspace, workspace_bytes, amq_layer_norm_backward_workspace_bytes(rows, n)))
    return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_norm_grad({dy, x, weight, mean, rstd, dx, dweight, dbias, static_cast<float*>(workspace), rows,
                                               ld_dy, ld_x, ld_dx, (int)n, type, param_type},
                                              static_cast<hipStream_t>(stream)));
}

size_t amq_linear_workspace_bytes(int64_t rows, int64_t k, int64_t n, int type) {
  if (!linear_sizes_ok(rows, k, n) || !linear_sizes_supported(rows, k, n) || !type_ok(type)) return 0;
  return amq::linear_workspace(rows, k, n, type);
}

int amq_linear(const void* x, int64_t ld_x, const void* W, int64_t ld_w, int64_t rows, int64_t k, int64_t n, int type,
               const void* bias, int activation, const void* residual, int64_t ld_r, void* y, int64_t ld_y, void* pre,
               int64_t ld_pre, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !W || !y || !type_ok(type) || activation < AMQ_ACT_NONE || activation > AMQ_ACT_TANH) return AMQ_ERR_INVALID;
  if (!linear_sizes_ok(rows, k, n) || ld_x < k || ld_w < k || ld_y < n || (residual && ld_r < n) || (pre && ld_pre < n))
    return AMQ_ERR_INVALID;
  if (!on_elements(x, type) || !on_elements(W, type) || !on_elements(y, type) || !on_elements(bias, type) ||
      !on_elements(residual, type) || !on_elements(pre, type))
    return AMQ_ERR_INVALID;
  if (!linear_sizes_supported(rows, k, n) || ld_x > kMaxStride || ld_w > kMaxStride) return AMQ_ERR_UNSUPPORTED;
  const Extent ex = matrix(x, rows, k, ld_x, type), eW = matrix(W, n, k, ld_w, type), eb = vector(bias, n, type), er = matrix(residual, rows, n, ld_r, type);
  const Extent ey = matrix(y, rows, n, ld_y, type), ep = matrix(pre, rows, n, ld_pre, type);
  if (meets(ey, {ex, eW, eb, ep}) || meets(ep, {ex, eW, eb, er}) || (!same(ey, er) && overlap(ey, er))) return AMQ_ERR_INVALID;
  if (!workspace_ok(workspace, workspace_bytes, amq::linear_workspace(rows, k, n, type))) return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_linear({x, W, bias, residual, y, pre, ld_x, ld_w, ld_r, ld_y, ld_pre, (int)rows, (int)k, (int)n,
                                            type, activation, workspace},
                                           static_cast<hipStream_t>(stream)));
}

size_t amq_linear_backward_workspace_bytes(int64_t rows, int64_t k, int64_t n, int type) {
  if (!linear_sizes_ok(rows, k, n) || !linear_sizes_supported(rows, k, n) || !type_ok(type)) return 0;
  return amq::linear_grad_workspace(rows, k, n, type);
}

int amq_linear_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* W, int64_t ld_w,
                        const void* pre, int64_t ld_pre, int64_t rows, int64_t k, int64_t n, int type, int activation,
                        void* dx, int64_t ld_dx, void* dW, int64_t ld_dw, void* dbias, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!dy || !type_ok(type) || activation < AMQ_ACT_NONE || activation > AMQ_ACT_TANH) return AMQ_ERR_INVALID;
  if ((dx && !W) || (dW && !x) || (activation != AMQ_ACT_NONE && !pre) || (!dx && !dW && !dbias)) return AMQ_ERR_INVALID;
  if (!linear_sizes_ok(rows, k, n) || ld_dy < n || (activation != AMQ_ACT_NONE && ld_pre < n) || (dW && (ld_x < k || ld_dw < k)) ||
      (dx && (ld_w < k || ld_dx < k)))
    return AMQ_ERR_INVALID;
  if (!on_elements(dy, type) || !on_elements(x, type) || !on_elements(W, type) || !on_elements(pre, type) || !on_elements(dx, type) ||
      !on_elements(dW, type) || !on_elements(dbias, type))
    return AMQ_ERR_INVALID;
  if (!linear_sizes_supported(rows, k, n) || ld_dy > kMaxStride || (dW && ld_x > kMaxStride) || (dx && ld_w > kMaxStride)) return AMQ_ERR_UNSUPPORTED;
  // (x and W are read for dW and dx alone)
  const Extent none{}, ed = matrix(dy, rows, n, ld_dy, type), ep = activation != AMQ_ACT_NONE ? matrix(pre, rows, n, ld_pre, type) : none;
  const Extent ex = dW ? matrix(x, rows, k, ld_x, type) : none, eW = dx ? matrix(W, n, k, ld_w, type) : none;
  const Extent edx = matrix(dx, rows, k, ld_dx, type), edW = matrix(dW, n, k, ld_dw, type), edb = vector(dbias, n, type);
  if (meets(edx, {ed, ep, ex, eW, edW, edb}) || meets(edW, {ed, ep, ex, eW, edb}) || meets(edb, {ed, ep, ex, eW})) return AMQ_ERR_INVALID;
  if (!workspace_ok(workspace, workspace_bytes, amq::linear_grad_workspace(rows, k, n, type))) return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_linear_grad({dy, x, W, pre, dx, dW, dbias, ld_dy, ld_x, ld_w, ld_pre, ld_dx, ld_dw, (int)rows, (int)k,
                                                 (int)n, type, activation, workspace},
                                                static_cast<hipStream_t>(stream)));
}

static bool ortho_supported(int64_t batch, int64_t rows, int64_t cols) { return batch <= 65535 && rows <= kMaxSize && cols <= kMaxSize; }

size_t amq_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, int type) {
  if (batch <= 0 || rows <= 0 || cols <= 0 || !type_ok(type) || !ortho_supported(batch, rows, cols)) return 0;
  return amq::ortho_workspace(batch, rows, cols);
}

int amq_orthogonalize(const void* G, int64_t batch, int64_t batch_stride, int64_t rows, int64_t cols, int64_t ld, int type,
                      int steps, const float* coef, float eps, void* out, int64_t batch_stride_out, int64_t ld_out,
                      void* workspace, size_t workspace_bytes, void* stream) {
  if (!G || !out || !coef || !type_ok(type) || batch <= 0 || rows <= 0 || cols <= 0 || ld < cols || ld_out < cols) return AMQ_ERR_INVALID;
  if (steps < 0 || !(eps >= 0.0f) || !on_elements(G, type) || !on_elements(out, type)) return AMQ_ERR_INVALID;
  if (!ortho_supported(batch, rows, cols)) return AMQ_ERR_UNSUPPORTED;
  if (batch_stride == 0) batch_stride = rows * ld;
  if (batch_stride_out == 0) batch_stride_out = rows * ld_out;
  // (matrices of the output must not share entries)
  if (batch_stride < 0 || (batch > 1 && batch_stride_out < (rows - 1) * ld_out + cols)) return AMQ_ERR_INVALID;
  // (with steps G is read to its end before the result is written)
  if (steps == 0 && !(G == out && ld == ld_out && (batch == 1 || batch_stride == batch_stride_out))) {
    const int64_t size = (int64_t)size_of(type), apart = batch_stride_out * size, room = ((rows - 1) * ld_out + cols) * size;
    for (int64_t z = 0; z < batch; ++z) {
      const Extent g = matrix(static_cast<const char*>(G) + z * batch_stride * size, rows, cols, ld, type);
      const int64_t from = (int64_t)(g.p - reinterpret_cast<uintptr_t>(out));
      int64_t w = batch > 1 ? floor_div(from - room, apart) : 0;  // the first whose room may reach g
      for (w = w > 0 ? w : 0; w < batch && w * apart < from + (rows - 1) * g.step + g.width; ++w)
        if (overlap(g, matrix(static_cast<const char*>(out) + w * apart, rows, cols, ld_out, type))) return AMQ_ERR_INVALID;
    }
  }
  if (!workspace_ok(workspace, workspace_bytes, amq::ortho_workspace(batch, rows, cols))) return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_ortho({G, out, batch_stride, ld, batch_stride_out, ld_out, (int)batch, (int)rows, (int)cols, type, steps,
                                           coef[0], coef[1], coef[2], eps, workspace},
                                          static_cast<hipStream_t>(stream)));
}

size_t amq_linear_recurrence_workspace_bytes(int64_t steps, int64_t B, int64_t n, int type) {
  if (!recurrence_sizes_ok(steps, B, n) || !recurrence_sizes_supported(steps, B, n) || !type_ok(type)) return 0;
  return amq::recurrence_workspace(steps, B, n, type);
}

int amq_linear_recurrence(const void* gate, int64_t gate_step, int64_t gate_batch, const void* x, int64_t x_step, int64_t x_batch,
                          int64_t steps, int64_t B, int64_t n, int type, int mode, const int64_t* lengths, const float* h0,
                          void* hs, int64_t hs_step, int64_t hs_batch, float* h_last, float* states, void* workspace,
                          size_t workspace_bytes, void* stream) {
  if (!gate || !x || !hs || !type_ok(type) || (mode != AMQ_RECURRENCE_BLEND && mode != AMQ_RECURRENCE_DECAY)) return AMQ_ERR_INVALID;
  if (!recurrence_sizes_ok(steps, B, n) || !strides_ok(gate_step, gate_batch) || !strides_ok(x_step, x_batch) || !strides_ok(hs_step, hs_batch))
    return AMQ_ERR_INVALID;
  if (!on_elements(gate, type) || !on_elements(x, type) || !on_elements(hs, type) || !on_elements(h0, AMQ_F32) || !on_elements(h_last, AMQ_F32) ||
      !on_elements(states, AMQ_F32) || (reinterpret_cast<uintptr_t>(lengths) & 7))
    return AMQ_ERR_INVALID;
  if (!recurrence_sizes_supported(steps, B, n) || !strides_supported(gate_step, gate_batch) || !strides_supported(x_step, x_batch) ||
      !strides_supported(hs_step, hs_batch))
    return AMQ_ERR_UNSUPPORTED;
  if (!apart(steps, B, n, hs_step, hs_batch)) return AMQ_ERR_INVALID;
  if (states_of(steps) == 0) states = nullptr;
  const Volume eg = volume(gate, steps, B, n, gate_step, gate_batch, type), ex = volume(x, steps, B, n, x_step, x_batch, type);
  const Volume out = volume(hs, steps, B, n, hs_step, hs_batch, type);
  const Extent h = vector(h0, B * n, AMQ_F32), last = vector(h_last, B * n, AMQ_F32);
  const Volume st = of(vector(states, states_of(steps) * B * n, AMQ_F32)), len = of(vector(lengths, 2 * B, AMQ_F32));
  if (meets(out, {eg, ex, of(h), of(last), st, len}) || meets(of(last), {eg, ex, st, len}) || meets(st, {eg, ex, of(h), len}) ||
      (!same(h, last) && overlap(h, last)))
    return AMQ_ERR_INVALID;
  if (!workspace_ok(workspace, workspace_bytes, amq::recurrence_workspace(steps, B, n, type))) return AMQ_ERR_INVALID;
  // batch entries side by side are channels of one wider entry
  if (!lengths && B > 1 && gate_batch == n && x_batch == n && hs_batch == n && amq::recurrence_entries_join(steps, B * n, type, false)) n *= B, B = 1;
  return amq::status_of(amq::launch_recurrence({gate, x, hs, gate_step, gate_batch, x_step, x_batch, hs_step, hs_batch, steps, B, (int)n, type, mode,
                                                lengths, h0, h_last, states, workspace},
                                               static_cast<hipStream_t>(stream)));
}

size_t amq_linear_recurrence_backward_workspace_bytes(int64_t steps, int64_t B, int64_t n, int type) {
  if (!recurrence_sizes_ok(steps, B, n) || !recurrence_sizes_supported(steps, B, n) || !type_ok(type)) return 0;
  return amq::recurrence_grad_workspace(steps, B, n, type);
}

int amq_linear_recurrence_backward(const void* dhs, int64_t dhs_step, int64_t dhs_batch, const void* gate, int64_t gate_step,
                                   int64_t gate_batch, const void* x, int64_t x_step, int64_t x_batch, int64_t steps, int64_t B,
                                   int64_t n, int type, int mode, const int64_t* lengths, const float* h0, const float* states,
                                   const float* dh_last, void* dgate, int64_t dgate_step, int64_t dgate_batch, void* dx,
                                   int64_t dx_step, int64_t dx_batch, float* dh0, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  if (!dhs || !gate || !x || !dgate || !dx || !type_ok(type) || (mode != AMQ_RECURRENCE_BLEND && mode != AMQ_RECURRENCE_DECAY)) return AMQ_ERR_INVALID;
  if (!recurrence_sizes_ok(steps, B, n) || !strides_ok(dhs_step, dhs_batch) || !strides_ok(gate_step, gate_batch) || !strides_ok(x_step, x_batch) ||
      !strides_ok(dgate_step, dgate_batch) || !strides_ok(dx_step, dx_batch) || (states_of(steps) > 0 && !states))
    return AMQ_ERR_INVALID;
  if (!on_elements(dhs, type) || !on_elements(gate, type) || !on_elements(x, type) || !on_elements(dgate, type) || !on_elements(dx, type) ||
      !on_elements(h0, AMQ_F32) || !on_elements(states, AMQ_F32) || !on_elements(dh_last, AMQ_F32) || !on_elements(dh0, AMQ_F32) ||
      (reinterpret_cast<uintptr_t>(lengths) & 7))
    return AMQ_ERR_INVALID;
  if (!recurrence_sizes_supported(steps, B, n) || !strides_supported(dhs_step, dhs_batch) || !strides_supported(gate_step, gate_batch) ||
      !strides_supported(x_step, x_batch) || !strides_supported(dgate_step, dgate_batch) || !strides_supported(dx_step, dx_batch))
    return AMQ_ERR_UNSUPPORTED;
  if (!apart(steps, B, n, dgate_step, dgate_batch) || !apart(steps, B, n, dx_step, dx_batch)) return AMQ_ERR_INVALID;
  if (states_of(steps) == 0) states = nullptr;
  const Volume ed = volume(dhs, steps, B, n, dhs_step, dhs_batch, type), eg = volume(gate, steps, B, n, gate_step, gate_batch, type);
  const Volume ex = volume(x, steps, B, n, x_step, x_batch, type), rg = volume(dgate, steps, B, n, dgate_step, dgate_batch, type);
  const Volume rx = volume(dx, steps, B, n, dx_step, dx_batch, type), r0 = of(vector(dh0, B * n, AMQ_F32));
  const Volume h = of(vector(h0, B * n, AMQ_F32)), st = of(vector(states, states_of(steps) * B * n, AMQ_F32));
  const Volume dl = of(vector(dh_last, B * n, AMQ_F32)), len = of(vector(lengths, 2 * B, AMQ_F32));
  if (meets(rg, {ed, eg, ex, h, st, dl, len, rx, r0}) || meets(rx, {ed, eg, ex, h, st, dl, len, r0}) || meets(r0, {ed, eg, ex, h, st, dl, len}))
    return AMQ_ERR_INVALID;
  if (!workspace_ok(workspace, workspace_bytes, amq::recurrence_grad_workspace(steps, B, n, type))) return AMQ_ERR_INVALID;
  if (!lengths && B > 1 && dhs_batch == n && gate_batch == n && x_batch == n && dgate_batch == n && dx_batch == n &&
      amq::recurrence_entries_join(steps, B * n, type, true))
    n *= B, B = 1;
  return amq::status_of(amq::launch_recurrence_grad({dhs, gate, x, dgate, dx, dhs_step, dhs_batch, gate_step, gate_batch, x_step, x_batch, dgate_step,
                                                     dgate_batch, dx_step, dx_batch, steps, B, (int)n, type, mode, lengths, h0, states, dh_last,
                                                     dh0, workspace},
                                                    static_cast<hipStream_t>(stream)));
}

int amq_block_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_r, const void* gate, int64_t ld_g, int64_t rows,
                   int64_t n, int type, int residual_type, int param_type, int activation, const void* weight, const void* bias,
                   const void* scale, const void* next_weight, const void* next_bias, float eps, void* y, int64_t ld_y,
                   void* normed, int64_t ld_n, float* stats, void* stream) {
  if (!x || !residual || !y || !type_ok(type) || (residual_type != AMQ_F32 && residual_type != type) || (param_type != AMQ_F32 && param_type != type) ||
      !gate_act_ok(activation))
    return AMQ_ERR_INVALID;
  if (rows <= 0 || n <= 0 || ld_x < n || ld_r < n || (gate && ld_g < n) || ld_y < n || (normed && ld_n < n) || !(eps >= 0.0f)) return AMQ_ERR_INVALID;
  if (!on_elements(x, type) || !on_elements(residual, residual_type) || !on_elements(gate, type) || !on_elements(y, residual_type) ||
      !on_elements(normed, type) || !on_elements(weight, param_type) || !on_elements(bias, param_type) || !on_elements(scale, param_type) ||
      !on_elements(next_weight, param_type) || !on_elements(next_bias, param_type) || !on_elements(stats, AMQ_F32))
    return AMQ_ERR_INVALID;
  if (rows > 0x7fffffffLL || n > kMaxJoined) return AMQ_ERR_UNSUPPORTED;
  const Extent ex = matrix(x, rows, n, ld_x, type), er = matrix(residual, rows, n, ld_r, residual_type), eg = matrix(gate, rows, n, ld_g, type);
  const Extent ey = matrix(y, rows, n, ld_y, residual_type), en = matrix(normed, rows, n, ld_n, type), es = vector(stats, 4 * rows, AMQ_F32);
  const Extent params[] = {vector(weight, n, param_type), vector(bias, n, param_type), vector(scale, n, param_type),
                           vector(next_weight, n, param_type), vector(next_bias, n, param_type)};
  if (meets(ey, params) || meets(en, params) || meets(es, params) || meets(ey, {ex, eg, en, es}) || (!same(ey, er) && overlap(ey, er)) ||
      meets(en, {ex, er, eg, es}) || meets(es, {ex, er, eg}))
    return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_block_norm({x, residual, gate, weight, bias, scale, next_weight, next_bias, y, normed, stats, rows, ld_x, ld_r, ld_g,
                                                ld_y, ld_n, (int)n, type, residual_type, param_type, activation, eps},
                                               static_cast<hipStream_t>(stream)));
}

size_t amq_block_norm_backward_workspace_bytes(int64_t rows, int64_t n) {
  if (rows <= 0 || n <= 0 || rows > 0x7fffffffLL || n > kMaxJoined) return 0;
  return (sizeof(float) * 4 * (size_t)amq::block_norm_grad_parts(rows, (int)n) * n + 255) & ~size_t(255);
}

int amq_block_norm_backward(const void* dy, int64_t ld_dy, const void* dnormed, int64_t ld_dn, const void* x, int64_t ld_x,
                            const void* y, int64_t ld_y, const void* gate, int64_t ld_g, int64_t rows, int64_t n, int type,
                            int residual_type, int param_type, int activation, const void* weight, const void* bias,
                            const void* scale, const void* next_weight, const float* stats, void* dx, int64_t ld_dx,
                            void* dresidual, int64_t ld_dr, void* dgate, int64_t ld_dg, void* dweight, void* dbias, void* dscale,
                            void* dnext_weight, void* dnext_bias, void* workspace, size_t workspace_bytes, void* stream) {
  if ((!dy && !dnormed) || !x || (dnormed && !y) || !stats || !dx || (dgate && !gate) || !type_ok(type) ||
      (residual_type != AMQ_F32 && residual_type != type) || (param_type != AMQ_F32 && param_type != type) || !gate_act_ok(activation))
    return AMQ_ERR_INVALID;
  if (rows <= 0 || n <= 0 || (dy && ld_dy < n) || (dnormed && (ld_dn < n || ld_y < n)) || ld_x < n || (gate && ld_g < n) || ld_dx < n ||
      (dresidual && ld_dr < n) || (dgate && ld_dg < n))
    return AMQ_ERR_INVALID;
  if (!on_elements(dy, residual_type) || !on_elements(dnormed, type) || !on_elements(x, type) || !on_elements(y, residual_type) ||
      !on_elements(gate, type) || !on_elements(dx, type) || !on_elements(dresidual, residual_type) || !on_elements(dgate, type) ||
      !on_elements(weight, param_type) || !on_elements(bias, param_type) || !on_elements(scale, param_type) ||
      !on_elements(next_weight, param_type) || !on_elements(stats, AMQ_F32) || !on_elements(dweight, param_type) || !on_elements(dbias, param_type) ||
      !on_elements(dscale, param_type) || !on_elements(dnext_weight, param_type) || !on_elements(dnext_bias, param_type))
    return AMQ_ERR_INVALID;
  if (rows > 0x7fffffffLL || n > kMaxJoined) return AMQ_ERR_UNSUPPORTED;
  const Extent none{}, ed = matrix(dy, rows, n, ld_dy, residual_type), en = matrix(dnormed, rows, n, ld_dn, type), ex = matrix(x, rows, n, ld_x, type);
  const Extent ey = dnormed ? matrix(y, rows, n, ld_y, residual_type) : none, eg = matrix(gate, rows, n, ld_g, type), es = vector(stats, 4 * rows, AMQ_F32);
  const Extent operands[] = {en, ex, ey, eg, es, vector(weight, n, param_type), vector(bias, n, param_type), vector(scale, n, param_type),
                             vector(next_weight, n, param_type)};
  const Extent rx = matrix(dx, rows, n, ld_dx, type), rr = matrix(dresidual, rows, n, ld_dr, residual_type), rg = matrix(dgate, rows, n, ld_dg, type);
  const Extent sums[] = {vector(dweight, n, param_type), vector(dbias, n, param_type), vector(dscale, n, param_type),
                         vector(dnext_weight, n, param_type), vector(dnext_bias, n, param_type)};
  if (meets(rx, operands) || meets(rr, operands) || meets(rg, operands) || meets(rx, sums) || meets(rr, sums) || meets(rg, sums) ||
      meets(rx, {ed, rr, rg}) || meets(rg, {ed, rr}) || (!same(rr, ed) && overlap(rr, ed)))
    return AMQ_ERR_INVALID;
  for (int i = 0; i < 5; ++i) {
    if (meets(sums[i], operands) || overlap(sums[i], ed)) return AMQ_ERR_INVALID;
    for (int j = 0; j < i; ++j)
      if (overlap(sums[i], sums[j])) return AMQ_ERR_INVALID;
  }
  if ((dweight || dbias || dscale || dnext_weight || dnext_bias) &&
      !workspace_ok(workspace, workspace_bytes, amq_block_norm_backward_workspace_bytes(rows, n)))
    return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_block_norm_grad({dy, dnormed, x, y, gate, weight, bias, scale, next_weight, stats, dx, dresidual, dgate, dweight, dbias,
                                                     dscale, dnext_weight, dnext_bias, static_cast<float*>(workspace), rows, ld_dy, ld_dn, ld_x, ld_y,
                                                     ld_g, ld_dx, ld_dr, ld_dg, (int)n, type, residual_type, param_type, activation},
                                                    static_cast<hipStream_t>(stream)));
}

size_t amq_clip_gradients_workspace_bytes(int64_t count) {
  if (count < 0 || count > kMaxSize) return 0;
  return amq::clip_workspace(count);
}

int amq_clip_gradients(int64_t count, const void* const* tensors, const int64_t* sizes, const int* types, float max_norm,
                       void* const* out, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  return amq_clip_gradients_double(count, tensors, sizes, types, max_norm, out, norm, workspace, workspace_bytes, stream);
}

int amq_clip_gradients_double(int64_t count, const void* const* tensors, const int64_t* sizes, const int* types, double max_norm,
                              void* const* out, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (count < 0 || (count > 0 && (!tensors || !sizes || !types)) || !norm || !on_elements(norm, AMQ_F32) || (out && !(max_norm >= 0.0)))
    return AMQ_ERR_INVALID;
  if (count > kMaxSize) return AMQ_ERR_UNSUPPORTED;
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] < 0 || !type_ok(types[i])) return AMQ_ERR_INVALID;
    if (sizes[i] == 0) continue;
    if (!tensors[i] || !on_elements(tensors[i], types[i]) || (out && (!out[i] || !on_elements(out[i], types[i])))) return AMQ_ERR_INVALID;
    if (sizes[i] > (1LL << 40)) return AMQ_ERR_UNSUPPORTED;
  }
  // results in the order of their addresses: none may meet the next one, the norm, or a tensor that is not its own
  std::unique_ptr<Interval[]> results(new (std::nothrow) Interval[count + 1]);
  if (!results) return amq::status_of(hipErrorOutOfMemory);
  int64_t n = 0;
  const uintptr_t at_norm = reinterpret_cast<uintptr_t>(norm);
  results[n++] = {at_norm, at_norm + sizeof(float), -1};
  for (int64_t i = 0; out && i < count; ++i)
    if (sizes[i] > 0) {
      const uintptr_t p = reinterpret_cast<uintptr_t>(out[i]);
      results[n++] = {p, p + sizes[i] * size_of(types[i]), i};
    }
  std::sort(results.get(), results.get() + n, [](const Interval& a, const Interval& b) { return a.begin < b.begin; });
  for (int64_t i = 1; i < n; ++i)
    if (results[i].begin < results[i - 1].end) return AMQ_ERR_INVALID;
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] == 0) continue;
    const uintptr_t begin = reinterpret_cast<uintptr_t>(tensors[i]), end = begin + sizes[i] * size_of(types[i]);
    const Interval* r = std::lower_bound(results.get(), results.get() + n, begin, [](const Interval& a, uintptr_t b) { return a.end <= b; });
    if (r != results.get() + n && r->begin < end && !(r->index == i && r->begin == begin)) return AMQ_ERR_INVALID;
  }
  if (!workspace_ok(workspace, workspace_bytes, amq::clip_workspace(count))) return AMQ_ERR_INVALID;
  return amq::status_of(amq::launch_clip_gradients({tensors, out, sizes, types, count}, max_norm, norm, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
