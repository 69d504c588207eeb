// Host-side interface between the C ABI of the training operators (amq_train.hip) and their kernels: layer
// normalization, linear layers, orthogonalized updates, linear recurrences, joined norms, gradient clipping.  Plain data and launch functions; arguments are checked
// in the C ABI before any of these is called.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace amq {

// A status for the caller of the C ABI, remembered for amq_last_hip_error (amq_api.hip).
int status_of(hipError_t e);

// ---- layer normalization (amq_norm.hip)
struct NormArgs {
  const void *x, *weight, *bias;  // weight, bias: null for 1 and 0
  void* y;
  float *mean, *rstd;
  int64_t rows, ld_x, ld_y;
  int n, type, param_type;
  float eps;
};
hipError_t launch_norm(const NormArgs& a, hipStream_t s);

struct NormGradArgs {
  const void *dy, *x, *weight;
  const float *mean, *rstd;
  void *dx, *dweight, *dbias;  // dweight, dbias: null where not wanted
  float* part;                 // [norm_grad_parts][2][n] partial sums over rows
  int64_t rows, ld_dy, ld_x, ld_dx;
  int n, type, param_type;
};
int norm_grad_parts(int64_t rows, int n);
hipError_t launch_norm_grad(const NormGradArgs& a, hipStream_t s);

// ---- linear layers (amq_linear.hip)
struct LinearArgs {
  const void *x, *W, *bias, *residual;
  void *y, *pre;
  int64_t ld_x, ld_w, ld_r, ld_y, ld_pre;
  int rows, k, n, type, act;
  void* ws;
};
size_t linear_workspace(int64_t rows, int64_t k, int64_t n, int type);
hipError_t launch_linear(const LinearArgs& a, hipStream_t s);

struct LinearGradArgs {
  const void *dy, *x, *W, *pre;
  void *dx, *dW, *dbias;
  int64_t ld_dy, ld_x, ld_w, ld_pre, ld_dx, ld_dw;
  int rows, k, n, type, act;
  void* ws;
};
size_t linear_grad_workspace(int64_t rows, int64_t k, int64_t n, int type);
hipError_t launch_linear_grad(const LinearGradArgs& a, hipStream_t s);

// ---- orthogonalized updates (amq_ortho.hip)
struct OrthoArgs {
  const void* G;
  void* out;
  int64_t stride_g, ld_g, stride_out, ld_out;
  int batch, rows, cols, type, steps;
  float a, b, c, eps;
  void* ws;
};
size_t ortho_workspace(int64_t batch, int64_t rows, int64_t cols);
hipError_t launch_ortho(const OrthoArgs& a, hipStream_t s);

// ---- linear recurrences (amq_recurrence.hip).  Tensors [steps][batch][n] with strides of steps and batch entries.
struct RecurrenceArgs {
  const void *gate, *x;
  void* hs;
  int64_t gate_step, gate_batch, x_step, x_batch, hs_step, hs_batch, steps, batch;
  int n, type, mode;
  const int64_t* lengths;         // null: all steps count
  const float* h0;                // null: zeros
  float *h_last, *states;         // null where not wanted
  void* ws;
};
// Whether one launch has room for `channels`, so that batch entries side by side may count as channels of one wider entry.
bool recurrence_entries_join(int64_t steps, int64_t channels, int type, bool backward);
size_t recurrence_workspace(int64_t steps, int64_t batch, int64_t n, int type);
hipError_t launch_recurrence(const RecurrenceArgs& a, hipStream_t s);

struct RecurrenceGradArgs {
  const void *dhs, *gate, *x;
  void *dgate, *dx;
  int64_t dhs_step, dhs_batch, gate_step, gate_batch, x_step, x_batch, dgate_step, dgate_batch, dx_step, dx_batch, steps, batch;
  int n, type, mode;
  const int64_t* lengths;
  const float *h0, *states, *dh_last;  // h0, dh_last: null for zeros; states: null up to AMQ_STATE_STEPS steps
  float* dh0;                          // null where not wanted
  void* ws;
};
size_t recurrence_grad_workspace(int64_t steps, int64_t batch, int64_t n, int type);
hipError_t launch_recurrence_grad(const RecurrenceGradArgs& a, hipStream_t s);

// ---- joined norms (amq_block_norm.hip)
struct BlockNormArgs {
  const void *x, *residual, *gate;  // gate: null for none
  const void *weight, *bias, *scale, *next_weight, *next_bias;  // null for 1 and 0
  void *y, *normed;                 // normed: null where not wanted
  float* stats;                     // [4][rows]: mean and rstd of x, of y; null where not wanted
  int64_t rows, ld_x, ld_r, ld_g, ld_y, ld_n;
  int n, type, residual_type, param_type, act;
  float eps;
};
hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s);

struct BlockNormGradArgs {
  const void *dy, *dnormed;  // null for zeros (one of them)
  const void *x, *y, *gate, *weight, *bias, *scale, *next_weight;
  const float* stats;
  void *dx, *dresidual, *dgate;                                    // dresidual, dgate: null where not wanted
  void *dweight, *dbias, *dscale, *dnext_weight, *dnext_bias;      // null where not wanted
  float* part;                                                     // [block_norm_grad_parts][4][n] partial sums over rows
  int64_t rows, ld_dy, ld_dn, ld_x, ld_y, ld_g, ld_dx, ld_dr, ld_dg;
  int n, type, residual_type, param_type, act;
};
int block_norm_grad_parts(int64_t rows, int n);
hipError_t launch_block_norm_grad(const BlockNormGradArgs& a, hipStream_t s);

// ---- gradient norm and clipping (amq_clip.hip).  Arrays on the host.
struct ClipTensors {
  const void* const* tensors;
  void* const* out;  // null: the norm alone
  const int64_t* sizes;
  const int* types;
  int64_t count;
};
size_t clip_workspace(int64_t count);
hipError_t launch_clip_gradients(const ClipTensors& c, double max_norm, float* norm, void* ws, hipStream_t s);

}  // namespace amq
