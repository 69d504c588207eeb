// C ABI of the training operators (declared in include/amq.h): argument validation on the host, then kernel launches on
// the caller's stream.
#include "amq_train.h"

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

}  // extern "C"
