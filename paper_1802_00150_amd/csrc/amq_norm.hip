// Layer normalization, forward and backward.
//
//   mu = sum x / n,  var = sum (x - mu)^2 / n,  r = 1 / sqrt(var + eps),  y = (x - mu) r w + b
//   g = dy w,  z = (x - mu) r,  dx = r (g - mean(g) - z mean(g z)),  dw = sum_rows dy z,  db = sum_rows dy
//
// About 10 operations per entry against 4 to 12 bytes: bound by memory, or by latency for few rows.  So every entry is read
// once and kept in registers between the sums and the output: a row belongs to one wave (up to 2048 entries; its sums need
// no barrier) or to one workgroup of 4 or 16 waves (up to 8192, 16384).  The variance is formed from x - mu, not from the sum
// of squares, since the entries are there anyway.  Workgroups walk over rows, with the parameters, and in the backward pass
// the columns' sums of dy z and dy, in registers; those leave one partial row of sums per workgroup, added up by a second
// launch in a fixed order, so results do not depend on the order of execution.  Statistics and sums are binary32.
// Longer rows are read once per sum (general kernels at the end).
#include "../../include/amq.h"

#include <type_traits>

#include "amq_device.h"
#include "amq_train.h"
#include "amq_typed.h"



namespace amq {
namespace {

__device__ __forceinline__ float sum64(float v) { return group_sum(v, 6); }

// Sums of two values over the W waves that share a row.  One barrier: the slots of consecutive calls alternate.
template <int W>
__device__ __forceinline__ void row_sum2(float& a, float& b, float (*slots)[2], int& turn) {
  a = sum64(a);
  b = sum64(b);
  if constexpr (W > 1) {
    float(*s)[2] = slots + turn * W;
    turn ^= 1;
    if (lane_id() == 0) {
      s[wave_id()][0] = a;
      s[wave_id()][1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      a += s[i][0];
      b += s[i][1];
    }
  }
}
template <int W>
__device__ __forceinline__ float row_sum(float a, float (*slots)[2], int& turn) {
  float b = 0.0f;
  row_sum2<W>(a, b, slots, turn);
  return a;
}

// W waves per row, NV times 16 bytes per lane; workgroups of max(W, 4) waves.
template <typename T, typename P, int W, int NV>
__global__ __launch_bounds__(W > 4 ? W * 64 : 256) void norm_kernel(NormArgs a) {
  constexpr int V = kPer16<T>, kRows = W >= 4 ? 1 : 4;
  __shared__ float slots[2 * W][2];
  int turn = 0;
  const int tid = W == 1 ? lane_id() : (int)threadIdx.x;
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * W * 64 + tid) * V;
    load_params<P, V>((const P*)a.weight, c, a.n - c, 1.0f, w[j]);
    load_params<P, V>((const P*)a.bias, c, a.n - c, 0.0f, b[j]);
  }
  const float inv_n = 1.0f / (float)a.n;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (W == 1 ? wave_id() : 0); row < a.rows; row += (int64_t)gridDim.x * kRows) {
    const T* px = (const T*)a.x + row * a.ld_x;
    float x[NV][V], s = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * W * 64 + tid) * V;
      load16(px + c, a.n - c, x[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) s += x[j][i];
    const float mean = row_sum<W>(s, slots, turn) * inv_n;
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int left = a.n - (j * W * 64 + tid) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[j][i] -= mean;
        q = fmaf(i < left ? x[j][i] : 0.0f, x[j][i], q);
      }
    }
    const float rstd = 1.0f / sqrtf(row_sum<W>(q, slots, turn) * inv_n + a.eps);
    T* py = (T*)a.y + row * a.ld_y;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * W * 64 + tid) * V;
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = fmaf(x[j][i] * rstd, w[j][i], b[j][i]);
      store16(py + c, a.n - c, y);
    }
    if (tid == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <typename T, typename P, int W, int NV>
__global__ __launch_bounds__(W > 4 ? W * 64 : 256) void norm_grad_kernel(NormGradArgs a) {
  constexpr int V = kPer16<T>, kRows = W >= 4 ? 1 : 4, kEntries = W * 64 * NV * V;
  __shared__ float slots[2 * W][2];
  __shared__ float shared_sums[W == 1 ? 2 * kEntries : 1];
  int turn = 0;
  const int tid = W == 1 ? lane_id() : (int)threadIdx.x;
  float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * W * 64 + tid) * V;
    load_params<P, V>((const P*)a.weight, c, a.n - c, 1.0f, w[j]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[j][i] = db[j][i] = 0.0f;
  }
  const float inv_n = 1.0f / (float)a.n;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (W == 1 ? wave_id() : 0); row < a.rows; row += (int64_t)gridDim.x * kRows) {
    const T *px = (const T*)a.x + row * a.ld_x, *pd = (const T*)a.dy + row * a.ld_dy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float x[NV][V], d[NV][V], s = 0.0f, q = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * W * 64 + tid) * V;
      load16(px + c, a.n - c, x[j]);
      load16(pd + c, a.n - c, d[j]);  // 0 past the row's end: nothing there counts in any sum
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[j][i] = (x[j][i] - mean) * rstd;
        dw[j][i] = fmaf(d[j][i], x[j][i], dw[j][i]);
        db[j][i] += d[j][i];
        d[j][i] *= w[j][i];
        s += d[j][i];
        q = fmaf(d[j][i], x[j][i], q);
      }
    row_sum2<W>(s, q, slots, turn);
    s *= inv_n;
    q *= inv_n;
    T* po = (T*)a.dx + row * a.ld_dx;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * W * 64 + tid) * V;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = rstd * (d[j][i] - s - x[j][i] * q);
      store16(po + c, a.n - c, o);
    }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.n;
  if constexpr (W == 1) {
    // the waves add their sums in their order
    for (int turn_of = 0; turn_of < 4; ++turn_of) {
      if (wave_id() == turn_of) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            // [j][i][lane]: consecutive lanes on consecutive banks
            const int at = (j * V + i) * 64 + lane_id();
            if (turn_of) {
              dw[j][i] += shared_sums[at];
              db[j][i] += shared_sums[kEntries + at];
            }
            if (turn_of < 3) {
              shared_sums[at] = dw[j][i];
              shared_sums[kEntries + at] = db[j][i];
            }
          }
      }
      __syncthreads();
    }
    if (wave_id() != 3) return;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * W * 64 + tid) * V;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (c + i < a.n) {
        part[c + i] = dw[j][i];
        part[a.n + c + i] = db[j][i];
      }
  }
}

// Rows of any length, one workgroup per row, the row read once per sum and once for the output.
template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  __shared__ float slots[32][2];
  int turn = 0;
  const T* px = (const T*)a.x + (int64_t)blockIdx.x * a.ld_x;
  T* py = (T*)a.y + (int64_t)blockIdx.x * a.ld_y;
  float s = 0.0f;
  for (int c = threadIdx.x; c < a.n; c += 1024) s += (float)px[c];
  const float mean = row_sum<16>(s, slots, turn) / (float)a.n;
  s = 0.0f;
  for (int c = threadIdx.x; c < a.n; c += 1024) {
    const float d = (float)px[c] - mean;
    s = fmaf(d, d, s);
  }
  const float rstd = 1.0f / sqrtf(row_sum<16>(s, slots, turn) / (float)a.n + a.eps);
  for (int c = threadIdx.x; c < a.n; c += 1024) {
    const float w = a.weight ? (float)((const P*)a.weight)[c] : 1.0f, b = a.bias ? (float)((const P*)a.bias)[c] : 0.0f;
    py[c] = (T)fmaf(((float)px[c] - mean) * rstd, w, b);
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[blockIdx.x] = mean;
    if (a.rstd) a.rstd[blockIdx.x] = rstd;
  }
}

template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs a) {
  __shared__ float slots[32][2];
  int turn = 0;
  const int64_t row = blockIdx.x;
  const T *px = (const T*)a.x + row * a.ld_x, *pd = (const T*)a.dy + row * a.ld_dy;
  T* po = (T*)a.dx + row * a.ld_dx;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float s = 0.0f, q = 0.0f;
  for (int c = threadIdx.x; c < a.n; c += 1024) {
    const float g = (float)pd[c] * (a.weight ? (float)((const P*)a.weight)[c] : 1.0f);
    s += g;
    q = fmaf(g, ((float)px[c] - mean) * rstd, q);
  }
  row_sum2<16>(s, q, slots, turn);
  s /= (float)a.n;
  q /= (float)a.n;
  for (int c = threadIdx.x; c < a.n; c += 1024) {
    const float g = (float)pd[c] * (a.weight ? (float)((const P*)a.weight)[c] : 1.0f);
    po[c] = (T)(rstd * (g - s - ((float)px[c] - mean) * rstd * q));
  }
}

// Column sums of dy z and dy over every gridDim.y-th row, for rows of any length.
template <typename T>
__global__ __launch_bounds__(256) void norm_grad_columns_kernel(NormGradArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.n) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float d = (float)((const T*)a.dy)[row * a.ld_dy + c];
    dw = fmaf(d, ((float)((const T*)a.x)[row * a.ld_x + c] - a.mean[row]) * a.rstd[row], dw);
    db += d;
  }
  float* part = a.part + (int64_t)blockIdx.y * 2 * a.n;
  part[c] = dw;
  part[a.n + c] = db;
}

// Adds up the partial rows: 32 columns per workgroup, 32 groups of partial rows side by side.
template <typename P>
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(const float* part, int parts, int n, P* dweight, P* dbias) {
  __shared__ float sums[32][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane, width = 2 * (int64_t)n;
  float s = 0.0f;
  if (c < width)
#pragma unroll 8
    for (int p = group; p < parts; p += 32) s += part[p * width + c];
  sums[group][lane] = s;
  __syncthreads();
  if (group == 0 && c < width) {
    s = 0.0f;
#pragma unroll
    for (int g = 0; g < 32; ++g) s += sums[g][lane];
    P* out = c < n ? dweight : dbias;
    if (out) out[c < n ? c : c - n] = (P)s;
  }
}

// Waves per row and 16-byte pieces per lane.
struct Shape {
  int waves, pieces;  // waves 0: the general kernels
};
// Few rows go to four waves each from 512 entries on, where the row's latency counts and not the reduction's.
Shape shape_of(int64_t rows, int n, int per16) {
  const int most = 32 / per16;  // 32 entries per lane
  for (int p = 1; p <= most; p *= 2)
    if (n <= 64 * p * per16 && (rows > 512 || n <= 512)) return {1, p};
  for (int p = 1; p <= most; p *= 2)
    if (n <= 256 * p * per16) return {4, p};
  if (n <= 1024 * 16) return {16, most / 2};
  return {0, 0};
}

template <typename F>
hipError_t with_types(int type, int param_type, F f) {
  if (type == AMQ_F32) return f(float(), float());
  if (type == AMQ_BF16) return param_type == AMQ_F32 ? f(bf16(), float()) : f(bf16(), bf16());
  return param_type == AMQ_F32 ? f(f16(), float()) : f(f16(), f16());
}
template <typename T, typename F>
hipError_t with_shape(Shape h, F f) {
  constexpr int most = 32 / kPer16<T>;
#define AMQ_SHAPE(W, NV) \
  if (h.waves == W && h.pieces == NV) return f(std::integral_constant<int, W>(), std::integral_constant<int, NV>())
  AMQ_SHAPE(1, 1);
  AMQ_SHAPE(1, 2);
  AMQ_SHAPE(1, 4);
  if constexpr (most == 8) AMQ_SHAPE(1, 8);
  AMQ_SHAPE(4, 1);
  AMQ_SHAPE(4, 2);
  AMQ_SHAPE(4, 4);
  if constexpr (most == 8) AMQ_SHAPE(4, 8);
  AMQ_SHAPE(16, most / 2);
#undef AMQ_SHAPE
  return hipErrorInvalidValue;
}

// Rows that a grid of at most `most` workgroups takes at a time, spread evenly over its rounds.
int64_t even_blocks(int64_t tasks, int64_t most) {
  const int64_t rounds = (tasks + most - 1) / most;
  return (tasks + rounds - 1) / rounds;
}

constexpr int64_t kMostParts = 512;  // two workgroups per compute unit; more partial rows cost more than they hide

}  // namespace

int norm_grad_parts(int64_t rows, int n) {
  // (the widest and the narrowest types may take different forms; the larger number of either)
  int64_t parts = 1;
  for (int per16 : {4, 8}) {
    const Shape h = shape_of(rows, n, per16);
    const int64_t tasks = h.waves == 1 ? (rows + 3) / 4 : rows;
    const int64_t p = h.waves ? even_blocks(tasks, kMostParts) : (tasks < 64 ? tasks : 64);
    parts = p > parts ? p : parts;
  }
  return (int)parts;
}

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  return with_types(a.type, a.param_type, [&](auto t, auto p) {
    using T = decltype(t);
    using P = decltype(p);
    const Shape h = shape_of(a.rows, a.n, kPer16<T>);
    if (!h.waves) {
      norm_long_kernel<T, P><<<dim3((unsigned)a.rows), dim3(1024), 0, s>>>(a);
      return hipGetLastError();
    }
    return with_shape<T>(h, [&](auto w, auto nv) {
      constexpr int W = decltype(w)::value;
      const int64_t tasks = W == 1 ? (a.rows + 3) / 4 : a.rows;
      norm_kernel<T, P, W, decltype(nv)::value>
          <<<dim3((unsigned)even_blocks(tasks, W == 16 ? 512 : 2048)), dim3(W > 4 ? W * 64 : 256), 0, s>>>(a);
      return hipGetLastError();
    });
  });
}

hipError_t launch_norm_grad(const NormGradArgs& a0, hipStream_t s) {
  NormGradArgs a = a0;
  const bool sums = a.dweight || a.dbias;
  if (!sums) a.part = nullptr;
  return with_types(a.type, a.param_type, [&](auto t, auto p) {
    using T = decltype(t);
    using P = decltype(p);
    const Shape h = shape_of(a.rows, a.n, kPer16<T>);
    int64_t parts = 0;
    hipError_t e;
    if (!h.waves) {
      norm_grad_long_kernel<T, P><<<dim3((unsigned)a.rows), dim3(1024), 0, s>>>(a);
      e = hipGetLastError();
      if (e == hipSuccess && sums) {
        parts = a.rows < 64 ? a.rows : 64;
        norm_grad_columns_kernel<T><<<dim3((unsigned)((a.n + 255) / 256), (unsigned)parts), dim3(256), 0, s>>>(a);
        e = hipGetLastError();
      }
    } else {
      e = with_shape<T>(h, [&](auto w, auto nv) {
        constexpr int W = decltype(w)::value;
        parts = even_blocks(W == 1 ? (a.rows + 3) / 4 : a.rows, kMostParts);
        norm_grad_kernel<T, P, W, decltype(nv)::value><<<dim3((unsigned)parts), dim3(W > 4 ? W * 64 : 256), 0, s>>>(a);
        return hipGetLastError();
      });
    }
    if (e != hipSuccess || !sums) return e;
    norm_grad_sum_kernel<P><<<dim3((unsigned)((2 * (int64_t)a.n + 31) / 32)), dim3(1024), 0, s>>>(a.part, (int)parts, a.n,
                                                                                                  (P*)a.dweight, (P*)a.dbias);
    return hipGetLastError();
  });
}

}  // namespace amq
