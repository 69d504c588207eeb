// Host-side interface between the C ABI of the training operators (amq_train.hip) and their kernels: layer
// normalization, linear layers, orthogonalized updates.  Plain data and launch functions; arguments are checked
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

}  // namespace amq
