// Linear layers: y = act(x W^T + b) + residual, and the backward pass dx = d W, dW = d^T x, db = sum_rows d with
// d = dy act'(z).
//
// The products run on the 16-bit matrix cores (amq_matmul_body.h), which take an operand's k along rows or down columns: W in
// dx, d and x in dW are never transposed.  bfloat16 and half operands whose rows lie on 16 bytes and hold a multiple of 8
// values are read where they are.  Anything else is laid out first: rows padded with zeros, d multiplied out, and
// float values scaled by a power of two per row of the operand and split into two halves, 22 bits together.  (A binary32 matrix
// instruction has 1/16 of the rate of a half one; three half products of split operands have 1/3.)  The scale puts the row's
// largest value into [2^14, 2^15), so no product overflows.  The first half is off by 2^-11 of a value at most; the second holds that to 2^-12 of
// the most it can be, or to half of half's smallest step, 2^-25: a value is held to 2^-23 of itself, but to no less than 2^-39 of its row's largest.  In the
// norm of a result that is the error of binary32 products; a result that only small entries enter has the fewer digits of those.
//
// d of 16-bit data is a value of binary32 behind a slope.  It is laid out as two values of the type, the second what the first leaves (16 bits together in
// bfloat16, 22 in half), and each product takes two passes over its contraction, one for either.  Rounded to one value it cost the gradients
// 1.4 times the error that their own rounding leaves (and the backward pass of 8960 x 4096 by 1024 bfloat16 with gelu 207 us; so 357).
// relu's slopes are 0 and 1 and leave dy as exact as it was: one value, one pass.
// d in half is scaled too before it is rounded, by one power of two: gradients divided by a batch's size lie where half has few digits.
//
// A few rows (a token's vector) are multiplied on the vector units where the matrix cores' layout would cost more than it gives.
#include "../../include/amq.h"

#include <math.h>

#include "amq_device.h"
#include "amq_matmul_body.h"
#include "amq_train.h"

namespace amq {
namespace {

// The activations and their slopes through the hardware's exponential and reciprocal (1 ulp each).  Each passes a NaN on.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
// (1 - e) / (1 + e) with e = exp(-2 |z|) loses digits near 0; there the series to z^9, 2e-9 off at 1/4.
__device__ __forceinline__ float tanh_of(float z) {
  const float s = z * z;
  const float series = fmaf(fmaf(fmaf(fmaf(s, 62.0f / 2835.0f, -17.0f / 315.0f), s, 2.0f / 15.0f), s, -1.0f / 3.0f), s * z, z);
  const float e = __expf(-2.0f * fabsf(z));
  return fabsf(z) < 0.25f ? series : copysignf((1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e), z);
}
// The normal distribution Phi(z) by Abramowitz and Stegun 7.1.26, erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + p x),
// 1.5e-7 off at most; `density` receives exp(-z^2 / 2).
__device__ __forceinline__ float normal_of(float z, float& density) {
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
  density = __expf(-x * x);
  const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f) * density;
  return z < 0.0f ? 0.5f * q : 1.0f - 0.5f * q;
}
// One of the functions below on V values: the choice is made once for all of them, so that they run side by side.
template <int V, typename F>
__device__ __forceinline__ void each(float (&v)[V], F f) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = f(v[i]);
}
template <int V>
__device__ __forceinline__ void activate(float (&v)[V], int act) {
  switch (act) {
    case AMQ_ACT_RELU: return each(v, [](float z) { return z <= 0.0f ? 0.0f : z; });
    case AMQ_ACT_GELU:
      return each(v, [](float z) {
        float density;
        return z * normal_of(z, density);
      });
    case AMQ_ACT_SILU: return each(v, [](float z) { return z * logistic(z); });
    case AMQ_ACT_SIGMOID: return each(v, [](float z) { return logistic(z); });
    case AMQ_ACT_TANH: return each(v, [](float z) { return tanh_of(z); });
  }
}
template <int V>
__device__ __forceinline__ void slopes(float (&v)[V], int act) {
  switch (act) {
    case AMQ_ACT_RELU: return each(v, [](float z) { return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z; });
    case AMQ_ACT_GELU:
      return each(v, [](float z) {
        float density;
        const float phi = normal_of(z, density);
        return fmaf(z * 0.39894228040143268f, density, phi);
      });
    case AMQ_ACT_SILU:
      return each(v, [](float z) {
        const float s = logistic(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
      });
    case AMQ_ACT_SIGMOID:
      return each(v, [](float z) {
        const float s = logistic(z);
        return s * (1.0f - s);
      });
    case AMQ_ACT_TANH:
      return each(v, [](float z) {
        const float t = tanh_of(z);
        return fmaf(-t, t, 1.0f);
      });
  }
  each(v, [](float) { return 1.0f; });
}

// Scales, bias, activation, residual: what becomes of a product's values.
template <typename T>
struct LinearStore {
  static constexpr bool kTransposed = false;
  T *y, *pre;
  const T *bias, *residual;
  const int *exp_r, *exp_c, *exp_all;  // scales of the operands' rows, or of one operand, or null
  int64_t ld_y, ld_pre, ld_r;
  int M, N, act;

  struct Column {
    float bias[4];
    int exp[4];
  };
  struct Extra {
    float residual[4];
    int exp;
  };
  __device__ __forceinline__ Column column(int, int n) const {
    Column c;
    load_params<T, 4>(bias, n, N - n, 0.0f, c.bias);
    const int all = exp_all ? *exp_all : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) c.exp[i] = exp_c && n + i < N ? exp_c[n + i] : all;
    return c;
  }
  __device__ __forceinline__ Extra fetch(int, int m, int n) const {
    Extra e;
    load_params<T, 4>(residual, m * ld_r + n, m < M ? N - n : 0, 0.0f, e.residual);
    e.exp = exp_r && m < M ? exp_r[m] : 0;
    return e;
  }
  __device__ __forceinline__ void put(int, int m, int n, f32x4 v4, const Column& c, const Extra& e) const {
    if (m >= M || n >= N) return;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (exp_r || exp_all ? ldexpf(v4[i], -(e.exp + c.exp[i])) : v4[i]) + c.bias[i];
    if (pre) store<T, 4>(pre + m * ld_pre + n, N - n, v);
    activate(v, act);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += e.residual[i];
    store<T, 4>(y + m * ld_y + n, N - n, v);
  }
  // one value
  __device__ __forceinline__ void put1(int m, int n, float v) const {
    if (bias) v += (float)bias[n];
    if (pre) pre[m * ld_pre + n] = (T)v;
    float one[1] = {v};
    activate(one, act);
    if (residual) one[0] += (float)residual[m * ld_r + n];
    y[m * ld_y + n] = (T)one[0];
  }
};

// ---- a few rows: workgroup = 4 rows of W, its waves share the row's k.  Bound by reading W once, or for small W by latency: one row
// of 1024 float numbers by 4096 5.3 us (of which a launch alone 2), 3.2 TB/s from the last-level cache.
//
// Which rows come here: the matrix cores take 16 rows for the price of one, but float operands and those that do not lie as they need them
// have to be laid out first.  us here with 1 / 2 / 4 / 8 rows, and there:
//   float     1024 x 4096 4.1 / 4.9 / 6.4 / 9.3, 19;  1024 x 42000 25 / 26 / 32 / 63, 93              up to 8
//   16 bits, to be laid out: 300 x 300 3.9 / 4.6 / 5.9 / 8.6, 7.4                                      up to 4
//   16 bits, in place: 1024 x 1024 3.5 / 4.1 / 5.3 / 7.6, 5.0;  4096 x 4096 11.6 / 13.9 / 18.6 / 36, 8.8    rows k n below 2^22
constexpr int kFewRows = 8, kFewLaid = 4;
constexpr int64_t kFewInPlace = int64_t(1) << 22;
template <typename T, int M>
__global__ __launch_bounds__(256) void linear_few_kernel(const T* x, int64_t ld_x, const T* W, int64_t ld_w, int k, LinearStore<T> out) {
  constexpr int V = kPer16<T>, R = 4;
  __shared__ float sums[4][R * M];
  const int n0 = blockIdx.x * R;
  float acc[R][M];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int m = 0; m < M; ++m) acc[r][m] = 0.0f;
  const T* w[R];
#pragma unroll
  for (int r = 0; r < R; ++r) w[r] = W + (int64_t)(n0 + r < out.N ? n0 + r : out.N - 1) * ld_w;
  for (int c = threadIdx.x * V; c < k; c += 256 * V) {
    float b[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) load16(w[r] + c, k - c, b[r]);
#pragma unroll
    for (int m = 0; m < M; ++m) {
      float a[V];
      load16(x + (m < out.M ? m : 0) * ld_x + c, k - c, a);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[r][m] = fmaf(a[i], b[r][i], acc[r][m]);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const float s = group_sum(acc[r][m], 6);
      if (lane_id() == 0) sums[wave_id()][m * R + r] = s;
    }
  __syncthreads();
  if (threadIdx.x < R * M) {
    const int m = threadIdx.x / R, n = n0 + threadIdx.x % R;
    if (m < out.M && n < out.N)
      out.put1(m, n, sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] + sums[3][threadIdx.x]);
  }
}

// ---- laying operands out
// One matrix as it lies in memory; with `pre`, times the slope of the activation there.  (SLOPED: whether the launch has such a
// matrix.  The activations' code, once per piece of a row, takes the time to fetch it even where it does not run.)
template <typename T>
struct Source {
  const T* p;
  int64_t ld;
  const T* pre;
  int64_t ld_pre;
  int rows, cols, act;
  template <bool SLOPED, int V>
  __device__ __forceinline__ void load(int64_t row, int col, float (&v)[V]) const {
    load_params<T, V>(p, row * ld + col, cols - col, 0.0f, v);
    if (SLOPED && pre) {
      float z[V];
      load_params<T, V>(pre, row * ld_pre + col, cols - col, 0.0f, z);
      slopes(z, act);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= z[i];
    }
  }
  // N rows `step` apart, zeros past the last.
  template <bool SLOPED, int V, int N>
  __device__ __forceinline__ void load_rows(int64_t row, int64_t step, int col, float (&v)[N][V]) const {
    float z[N][V];
#pragma unroll
    for (int b = 0; b < N; ++b) load_params<T, V>(p, (row + b * step) * ld + col, row + b * step < rows ? cols - col : 0, 0.0f, v[b]);
    if (!SLOPED || !pre) return;
#pragma unroll
    for (int b = 0; b < N; ++b) load_params<T, V>(pre, (row + b * step) * ld_pre + col, row + b * step < rows ? cols - col : 0, 0.0f, z[b]);
#pragma unroll
    for (int b = 0; b < N; ++b) {
      slopes(z[b], act);
#pragma unroll
      for (int i = 0; i < V; ++i) v[b][i] *= z[b][i];
    }
  }
};
// One matrix in the layout of the product kernel: rows of `padded` values (a multiple of 64, zeros past the end), in two halves
// for float.
struct Laid {
  uint16_t* p;
  int* exps;    // scales: per row, per column, or one
  int64_t ld;
  int64_t low;  // 16 bits: where what the values leave of binary32 ones lies behind them, 0 where that is not kept
  int rows, padded;
};
enum Scale { kAsIs, kPerRow, kPerColumn, kOne };  // per row (found and left here) or column (read): float; as is, or all by one: 16 bits
template <typename T>
struct Job {
  Source<T> from;
  Laid to, also;  // also: the same once more, scaled per column (p null: not wanted)
  Scale scale;
  const float* tops;  // kOne: what the scale is found from, left in to.exps
  int top_count;
};
constexpr int kMaxJobs = 3;
template <typename T>
struct Jobs {
  Job<T> job[kMaxJobs];
  int first[kMaxJobs + 1];  // workgroups of job j: first[j] .. first[j + 1]
  int count;
};

// Scales go by the largest finite value: an infinity or NaN spoils the results that it enters, and no others.
__device__ __forceinline__ float magnitude(float v) {
  const float a = fabsf(v);
  return a < INFINITY ? a : 0.0f;
}
__device__ __forceinline__ int scale_exponent(float largest) { return largest > 0.0f ? 14 - ilogbf(largest) : 0; }
// 8 values of a row as the products take them.
template <typename T>
__device__ __forceinline__ void put8(const Laid& to, int64_t row, int at, const float (&v)[8]) {
  Elements<uint16_t, 8> hi, lo;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 4) {
      const f16 h = (f16)v[i];
      hi.v[i] = __builtin_bit_cast(uint16_t, h);
      lo.v[i] = __builtin_bit_cast(uint16_t, (f16)(v[i] - (float)h));
    } else {
      hi.v[i] = __builtin_bit_cast(uint16_t, (T)v[i]);
    }
  }
  uint16_t* q = to.p + row * to.ld + (sizeof(T) == 4 ? high_part(at) : at);
  *reinterpret_cast<uint4*>(q) = __builtin_bit_cast(uint4, hi);
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<uint4*>(q + 32) = __builtin_bit_cast(uint4, lo);
  } else if (to.low) {
#pragma unroll
    for (int i = 0; i < 8; ++i) lo.v[i] = __builtin_bit_cast(uint16_t, (T)(v[i] - (float)__builtin_bit_cast(T, hi.v[i])));
    *reinterpret_cast<uint4*>(q + to.low) = __builtin_bit_cast(uint4, lo);
  }
}

// One wave per row.  Rows of up to 4096 values stay in registers between the search for the scale and the output.  Bound by
// memory or, for few rows, latency: 700 + 1300 rows of 650 float numbers (10 MB read and written) 8 us, of 2048 11 us = 3 TB/s.
template <typename T, bool SLOPED>
__device__ __forceinline__ void lay(const Jobs<T>& jobs, int block) {
  int k = 0;
  while (k + 1 < jobs.count && block >= jobs.first[k + 1]) ++k;
  const Job<T>& j = jobs.job[k];
  const int64_t row = (int64_t)(block - jobs.first[k]) * 4 + wave_id();
  if (row >= j.to.rows) return;
  constexpr bool kFloat = sizeof(T) == 4;
  constexpr int kHeld = 8;
  float held[kHeld][8];
  const int pieces = (j.to.padded + 511) / 512;
#pragma unroll
  for (int p = 0; p < kHeld; ++p)
    if (p < pieces) j.from.template load<SLOPED, 8>(row, p * 512 + lane_id() * 8, held[p]);  // zeros past the end
  int e = 0;
  if (kFloat && j.scale == kPerRow) {
    float largest = 0.0f;
#pragma unroll
    for (int p = 0; p < kHeld; ++p)
      if (p < pieces)
#pragma unroll
        for (int i = 0; i < 8; ++i) largest = fmaxf(largest, magnitude(held[p][i]));
    for (int p = kHeld; p < pieces; ++p) {
      float v[8];
      j.from.template load<SLOPED, 8>(row, p * 512 + lane_id() * 8, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) largest = fmaxf(largest, magnitude(v[i]));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) largest = fmaxf(largest, __shfl_xor(largest, o, 64));
    e = scale_exponent(largest);
    if (lane_id() == 0) j.to.exps[row] = e;
  } else if (!kFloat && j.scale == kOne) {
    // (each row's wave for itself, of a quarter of a row's length: less than a launch in between costs)
    float largest = 0.0f;
#pragma unroll 4
    for (int i = lane_id(); i < j.top_count; i += 64) largest = fmaxf(largest, j.tops[i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) largest = fmaxf(largest, __shfl_xor(largest, o, 64));
    e = scale_exponent(largest);
    if (row == 0 && lane_id() == 0) *j.to.exps = e;
  }
  auto by_columns = [&](const Laid& to, int at, const float (&v)[8]) __attribute__((always_inline)) {
    const Elements<int, 8> exps = fetch<int, 8>(to.exps + at, j.from.cols - at);
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = ldexpf(v[i], exps.v[i]);
    put8<T>(to, row, at, o);
  };
  auto put = [&](int p, float (&v)[8]) __attribute__((always_inline)) {
    const int at = p * 512 + lane_id() * 8;
    if (at >= j.to.padded) return;
    if (kFloat && j.scale == kPerColumn) return by_columns(j.to, at, v);
    if (kFloat && j.also.p) by_columns(j.also, at, v);
    if (kFloat || j.scale != kAsIs) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = ldexpf(v[i], e);
    }
    put8<T>(j.to, row, at, v);
  };
#pragma unroll
  for (int p = 0; p < kHeld; ++p)
    if (p < pieces) put(p, held[p]);
  for (int p = kHeld; p < pieces; ++p) {
    float v[8];
    j.from.template load<SLOPED, 8>(row, p * 512 + lane_id() * 8, v);
    put(p, v);
  }
}

// ---- columns: sums and largest values, and on the way d itself where it needs no scale.  Bound by memory, or where slopes are
// formed by those: d of 8960 x 1024 bfloat16 with relu's slopes (55 MB) 14.9 us = 3.7 TB/s, with gelu's and in two values (73 MB) 20.0, and 5 us
// for the second launch.  Many rows of few columns are
// dealt to more parts, three workgroups per compute unit (with one, 64 parts, 22.7 us for 14.5).  A workgroup takes 32 groups of V
// columns and every 8 * parts-th row of them; what it finds are partial results, which a second launch puts together.  Of at
// most 128 rows one part is all (16 rows per thread; a launch costs more).
constexpr int kColumnParts = 64, kMostColumnParts = 192;
int column_parts(int64_t rows, int64_t blocks) {  // blocks: workgroups per part, of all jobs
  if (rows <= 128) return 1;
  const int64_t parts = 768 / blocks & ~int64_t(7);
  return (int)(rows <= 32 * kMostColumnParts || parts < kColumnParts ? kColumnParts : parts < kMostColumnParts ? parts : kMostColumnParts);
}
template <typename T>
struct ColumnJob {
  Source<T> from;
  float *sums, *largest;  // [parts][cols], or null; of one scale for all columns [parts][blocks]
  Laid to;                // p null: not wanted
  T* total;               // [cols]: the sums, or null
  int* exps;              // scales per column, or one, or null
  bool one;
};
template <typename T>
struct ColumnJobs {
  ColumnJob<T> job[3];
  int blocks;  // workgroups per part
  int parts, count;
};
// The column jobs, and behind them what is to be laid out and does not depend on them (d itself is not among it).
template <typename T, bool SLOPED>
__global__ __launch_bounds__(256) void columns_kernel(ColumnJobs<T> jobs, Jobs<T> beside) {
  const int own = jobs.blocks * jobs.parts * jobs.count;
  if ((int)blockIdx.x >= own) return lay<T, false>(beside, blockIdx.x - own);
  constexpr int V = kPer16<T>;
  __shared__ float part[2][8][32 * V + 4];
  const int block = blockIdx.x % jobs.blocks, part_of = blockIdx.x / jobs.blocks % jobs.parts;
  const ColumnJob<T>& j = jobs.job[blockIdx.x / (jobs.blocks * jobs.parts)];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, c = (block * 32 + lane) * V;
  const int width = j.to.p ? j.to.padded : j.from.cols;
  if (block * 32 * V >= width) return;
  float s[V], largest[V];
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = largest[i] = 0.0f;
  // four rows at a time, so that their loads are under way together
  constexpr int kBatch = 4;
  const int64_t step = 8 * jobs.parts;
  if (c < width)
    for (int64_t row0 = part_of * 8 + group; row0 < j.from.rows; row0 += kBatch * step) {
      float v[kBatch][V];
      j.from.template load_rows<SLOPED, V, kBatch>(row0, step, c, v);
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s[i] += v[b][i];
          largest[i] = fmaxf(largest[i], magnitude(v[b][i]));
        }
        if constexpr (V == 8)
          if (j.to.p && row0 + b * step < j.from.rows) put8<T>(j.to, row0 + b * step, c, v[b]);
      }
    }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    part[0][group][lane * V + i] = s[i];
    part[1][group][lane * V + i] = largest[i];
  }
  __syncthreads();
  float all = 0.0f;
  for (int i = threadIdx.x; i < 32 * V; i += 256) {
    const int at = block * 32 * V + i;
    if (at >= j.from.cols) continue;
    float sum = 0.0f, top = 0.0f;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      sum += part[0][q][i];
      top = fmaxf(top, part[1][q][i]);
    }
    if (jobs.parts == 1) {
      if (j.total) j.total[at] = (T)sum;
      if (j.exps && !j.one) j.exps[at] = scale_exponent(top);
    } else if (j.sums) {
      j.sums[(int64_t)part_of * j.from.cols + at] = sum;
    }
    if (j.largest && jobs.parts > 1 && !j.one) j.largest[(int64_t)part_of * j.from.cols + at] = top;
    all = top;
  }
  if (!j.one) return;
  __shared__ float tops[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor(all, o, 64));
  if (lane_id() == 0) tops[wave_id()] = all;
  __syncthreads();
  if (threadIdx.x == 0) j.largest[part_of * jobs.blocks + block] = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
}
// 32 columns per workgroup.
template <typename T>
__device__ __forceinline__ void add_columns(const ColumnJobs<T>& jobs, const ColumnJob<T>& j, int block) {
  __shared__ float sums[8][33], tops[8][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, cols = j.from.cols;
  const int c = block * 32 + lane;
  if (block * 32 >= cols) return;
  float s = 0.0f, top = 0.0f;
  if (c < cols) {
    if (j.total)
#pragma unroll 8
      for (int p = 0; p < jobs.parts; p += 8) s += j.sums[(int64_t)(p + group) * cols + c];
    if (j.exps && !j.one)
#pragma unroll 8
      for (int p = 0; p < jobs.parts; p += 8) top = fmaxf(top, j.largest[(int64_t)(p + group) * cols + c]);
  }
  sums[group][lane] = s;
  tops[group][lane] = top;
  __syncthreads();
  if (group || c >= cols) return;
  s = top = 0.0f;
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    s += sums[g][lane];
    top = fmaxf(top, tops[g][lane]);
  }
  if (j.total) j.total[c] = (T)s;
  if (j.exps && !j.one) j.exps[c] = scale_exponent(top);
}
template <typename T>
__global__ __launch_bounds__(256) void columns_sum_kernel(ColumnJobs<T> jobs) {
  add_columns(jobs, jobs.job[blockIdx.y], blockIdx.x);
}
template <typename T, bool SLOPED>
__global__ __launch_bounds__(256) void lay_kernel(Jobs<T> jobs) {
  lay<T, SLOPED>(jobs, blockIdx.x);
}
// The same for d in half, and behind it the sums of its columns.  (A launch in between that finds the scale and adds the columns cost the backward pass
// of 700 x 650 by 1300 14.5 us, 2240 x 1024 by 1024 10 of now 64.)
template <typename T>
__global__ __launch_bounds__(256) void lay_and_add_kernel(Jobs<T> jobs, ColumnJobs<T> beside) {
  const int own = jobs.first[jobs.count];
  if ((int)blockIdx.x >= own) return add_columns(beside, beside.job[0], blockIdx.x - own);
  lay<T, true>(jobs, blockIdx.x);
}

// ---- workspaces
struct Carve {
  char* base;
  size_t off = 0;
  explicit Carve(void* p) : base(static_cast<char*>(p)) {}
  void* take(size_t bytes) {
    void* p = base ? base + off : nullptr;
    off += (bytes + 255) & ~size_t(255);
    return p;
  }
};
int planes_of(int type) { return type == AMQ_F32 ? 2 : 1; }
Laid lay_room(Carve& w, int64_t rows, int64_t cols, int type, int64_t scales, bool low = false) {
  Laid l;
  l.rows = (int)rows;
  l.padded = (int)pad64(cols);
  l.ld = planes_of(type) * (int64_t)l.padded;
  l.low = low ? rows * l.ld : 0;
  l.p = (uint16_t*)w.take(2 * (size_t)(rows * l.ld + l.low));
  l.exps = scales ? (int*)w.take(sizeof(int) * (size_t)scales) : nullptr;
  return l;
}

struct ForwardRoom {
  Laid x, W;
  float* part;
  size_t total;
};
ForwardRoom forward_room(void* ws, int64_t rows, int64_t k, int64_t n, int type) {
  Carve w(ws);
  ForwardRoom r{};
  const bool scaled = type == AMQ_F32;
  if (rows > (scaled ? kFewRows : kFewLaid)) {
    r.x = lay_room(w, rows, k, type, scaled ? rows : 0);
    r.W = lay_room(w, n, k, type, scaled ? n : 0);
  }
  if (!scaled || rows > kFewRows) r.part = (float*)w.take(plan_product(rows, n, k, planes_of(type), 1, false).part_bytes);
  r.total = w.off;
  return r;
}

struct BackwardRoom {
  Laid d, d_columns, x, W;  // d for dx and (float: scaled otherwise; 16 bits: the same) for dW
  float *sums, *tops[3];
  float* part;
  size_t total;
};
BackwardRoom backward_room(void* ws, int64_t rows, int64_t k, int64_t n, int type) {
  Carve w(ws);
  BackwardRoom r{};
  const bool wide = type == AMQ_F32;
  r.d = lay_room(w, rows, n, type, wide ? rows : type == AMQ_F16 ? 1 : 0, !wide);
  r.d_columns = wide ? lay_room(w, rows, n, type, n) : r.d;
  r.x = lay_room(w, rows, k, type, wide ? k : 0);
  r.W = lay_room(w, n, k, type, wide ? k : 0);
  r.sums = (float*)w.take(sizeof(float) * kMostColumnParts * (size_t)n);
  if (type != AMQ_BF16) r.tops[0] = (float*)w.take(sizeof(float) * kMostColumnParts * (size_t)n);
  if (wide)
    for (int i = 1; i < 3; ++i) r.tops[i] = (float*)w.take(sizeof(float) * kMostColumnParts * (size_t)k);
  size_t most = 0;
  for (int passes = 1; passes <= (wide ? 1 : 2); ++passes)  // (either, whatever the activation)
    for (size_t b : {plan_product(rows, k, n, planes_of(type), 1, false, passes).part_bytes, plan_product(n, k, rows, planes_of(type), 1, false, passes).part_bytes})
      most = b > most ? b : most;
  r.part = (float*)w.take(most);
  r.total = w.off;
  return r;
}

template <typename F>
hipError_t with_type(int type, F f) {
  return type == AMQ_F32 ? f(float()) : type == AMQ_BF16 ? f(bf16()) : f(f16());
}

// Whether the product kernel can read a matrix where it is.
template <typename T>
bool in_place(const Source<T>& m) {
  return sizeof(T) == 2 && !m.pre && m.cols % 8 == 0 && m.ld % 8 == 0 && (reinterpret_cast<uintptr_t>(m.p) & 15) == 0;
}
template <typename T>
void add_job(Jobs<T>& jobs, const Source<T>& from, const Laid& to, Scale scale, const Laid& also = Laid{}) {
  jobs.job[jobs.count] = {from, to, also, scale, nullptr, 0};
  jobs.first[jobs.count + 1] = jobs.first[jobs.count] + (int)div_up(from.rows, 4);
  ++jobs.count;
}
template <typename T, bool SLOPED>
hipError_t run_jobs(const Jobs<T>& jobs, hipStream_t s) {
  if (!jobs.count) return hipSuccess;
  lay_kernel<T, SLOPED><<<dim3((unsigned)jobs.first[jobs.count]), dim3(256), 0, s>>>(jobs);
  return hipGetLastError();
}

// A matrix as an operand: its rows, or (`columns`) its columns.
template <typename T>
MatmulOperand operand(const Source<T>& m, bool columns) {
  return {m.p, m.ld, 0, columns ? m.cols : m.rows, 0};
}
MatmulOperand operand(const Laid& l, bool columns) { return {l.p, l.ld, 0, columns ? l.padded : l.rows, l.low}; }

template <typename T>
MatmulArgs product_args(const MatmulOperand& r, const MatmulOperand& c, int64_t k, const LinearStore<T>& out) {
  MatmulArgs g{};
  g.r = r;
  g.c = c;
  g.M = out.M;
  g.N = out.N;
  g.k = (int)k;
  return g;
}
template <typename T, bool RC, bool CC>
hipError_t product(const MatmulArgs& g, const LinearStore<T>& out, float* part, hipStream_t s, int passes = 1) {
  const ProductPlan p = plan_product(out.M, out.N, g.k, sizeof(T) == 4 ? 2 : 1, 1, false, passes);
  if constexpr (sizeof(T) == 4) {
    return launch_product<f16, 2, RC, CC>(g, p, 1, out, part, s);
  } else {
    if constexpr (CC)
      if (passes == 2) return launch_product<T, 1, RC, CC, true>(g, p, 1, out, part, s);
    return launch_product<T, 1, RC, CC>(g, p, 1, out, part, s);
  }
}

template <typename T>
hipError_t linear_few(const LinearArgs& a, const LinearStore<T>& out, hipStream_t s) {
  const dim3 grid((unsigned)div_up(a.n, 4));
  const T *x = (const T*)a.x, *W = (const T*)a.W;
  if (a.rows == 1) linear_few_kernel<T, 1><<<grid, dim3(256), 0, s>>>(x, a.ld_x, W, a.ld_w, a.k, out);
  else if (a.rows == 2) linear_few_kernel<T, 2><<<grid, dim3(256), 0, s>>>(x, a.ld_x, W, a.ld_w, a.k, out);
  else if (a.rows <= 4) linear_few_kernel<T, 4><<<grid, dim3(256), 0, s>>>(x, a.ld_x, W, a.ld_w, a.k, out);
  else linear_few_kernel<T, kFewRows><<<grid, dim3(256), 0, s>>>(x, a.ld_x, W, a.ld_w, a.k, out);
  return hipGetLastError();
}

}  // namespace

// The form of a product that takes the least time by these estimates, in us, with `load` tiles per compute unit and `stages`
// stages each.  Fitted to 22 shapes from 64 x 1024 x 1024 to 8960 x 4096 x 1024, bfloat16 and float, within 15 %; examples
// (bfloat16 with gelu, tile 256 / 128 / 64 / 64 with four groups): 8960 x 4096 x 1024 134 / 120 / 145 / 247, 4096^3 116 / 138 /
// 205 / 260, 2240 x 1024 x 1024 41 / 23 / 15 / 22, 1024 x 1024 x 2240 61 / 33 / 18 / 13, 300 x 300 x 1216 43 / 23 / 12 / 9.
//   256 (one workgroup per unit): a round 24 + 1.3 per stage
//   192 (one): a round 16 + 1.07 per stage (one round over 16384, 136 tiles of 256 or 253 of 192: 338 and 287)
//   128 (two): 10 + a tile 4 + 0.55 per stage, and a last round that is not full counts half as one
//   128 with two groups (one): 2 + a round 7.5 + 0.47 per stage (2048^3 24.6 against 29.7, 1024 x 4096 x 8960 75 against 88)
//   64 (three): 6.5 + a tile 0.9 + 0.2 per stage, alone 5.5 + 0.32 per stage
//   64 with four groups (one): 2 + a round 3.4 + 0.17 per stage
//   32 with eight groups (one): 0.5 + a round 3.7 + 0.085 per stage (64 x 1024 x 1024 5.3 against 8.0, 512^3 4.9 against 6.6)
// Numbers of two halves take half of a stage's steps, and 1.15 to 1.3 times its time.  A contraction split among workgroups
// costs a second launch of 6 us and the partial results twice through memory at 3 TB/s.
static double form_us(int tile, int groups, int planes, int64_t tiles, double s) {
  const double load = (double)tiles / 256.0, rounds = (double)div_up(tiles, 256);
  if (tile == 256) return rounds * (24.0 + 1.3 * s);
  if (tile == 192) return rounds * (16.0 + 1.07 * s);
  if (tile == 128 && groups == 2) return 2.0 + rounds * (7.5 + (planes == 1 ? 0.47 : 0.65) * s);
  if (tile == 128) return 10.0 + 0.5 * (rounds + load) * (4.0 + (planes == 1 ? 0.55 : 0.68) * s);
  if (tile == 32) return 0.5 + rounds * (3.7 + (planes == 1 ? 0.085 : 0.1) * s);
  if (groups == 4) return 2.0 + rounds * (3.4 + (planes == 1 ? 0.17 : 0.22) * s);
  return fmax(5.5 + (planes == 1 ? 0.32 : 0.4) * s, 6.5 + load * (0.9 + (planes == 1 ? 0.2 : 0.23) * s));
}

ProductPlan plan_product(int64_t M, int64_t N, int64_t k, int planes, int64_t batch, bool lower, int passes) {
  const int64_t stages = passes * div_up(k, stage_of(planes));
  ProductPlan best{};
  auto consider = [&](int tile, int groups, int64_t splits) {
    const int64_t a = div_up(M, tile), b = div_up(N, tile);
    const int64_t tiles = batch * (lower ? a * (a + 1) / 2 : a * b);
    ProductPlan p{};
    p.tile = tile;
    p.groups = groups;
    // (a whole number of stages for each group)
    p.tiles_per_split = (int)(splits == 1 ? stages : div_up(stages, groups * splits) * groups);
    p.splits = (int)div_up(stages, p.tiles_per_split);
    p.us = form_us(tile, groups, planes, tiles * p.splits, p.tiles_per_split);
    if (p.splits > 1) {
      p.part_bytes = sizeof(float) * (size_t)batch * p.splits * M * ((N + 3) & ~int64_t(3));
      p.us += 6.0 + 2.0 * (double)p.part_bytes / 3e6;
    }
    if (best.tile == 0 || p.us < best.us) best = p;
  };
  if (planes == 1) {
    consider(256, 1, 1);
    consider(192, 1, 1);
  }
  for (int64_t splits = 1; splits <= 32 && (splits == 1 || stages >= 16 * splits); splits *= 2) {
    consider(128, 1, splits);
    if (stages >= 4) consider(128, 2, splits);
    consider(64, 1, splits);
    if (stages >= 4) consider(64, 4, splits);
    consider(32, 8, splits);
  }
  return best;
}

ProductPlan plan_pair(int64_t M, int64_t N, int64_t k, int64_t M2, int64_t N2, int64_t k2, int planes, int passes) {
  const double s = (double)(passes * div_up(k, stage_of(planes))), s2 = (double)(passes * div_up(k2, stage_of(planes)));
  const struct {
    int tile, groups;
  } forms[] = {{128, 1}, {128, 2}, {64, 1}, {64, 4}, {32, 8}};
  ProductPlan best{};
  for (const auto& f : forms) {
    const int64_t tiles = div_up(M, f.tile) * div_up(N, f.tile), tiles2 = div_up(M2, f.tile) * div_up(N2, f.tile), all = tiles + tiles2;
    // one round takes as long as the longer of both, several as their mean
    const double mean = (s * tiles + s2 * tiles2) / all, longest = s > s2 ? s : s2;
    ProductPlan p{};
    p.tile = f.tile;
    p.groups = f.groups;
    p.splits = 1;
    p.us = fmax(form_us(f.tile, f.groups, planes, all, mean), form_us(f.tile, f.groups, planes, 256, longest));
    if (best.tile == 0 || p.us < best.us) best = p;
  }
  return best;
}

size_t linear_workspace(int64_t rows, int64_t k, int64_t n, int type) { return forward_room(nullptr, rows, k, n, type).total; }

hipError_t launch_linear(const LinearArgs& a, hipStream_t s) {
  return with_type(a.type, [&](auto t) {
    using T = decltype(t);
    LinearStore<T> out{(T*)a.y, (T*)a.pre, (const T*)a.bias, (const T*)a.residual, nullptr, nullptr, nullptr, a.ld_y, a.ld_pre, a.ld_r, a.rows, a.n, a.act};
    const Source<T> x{(const T*)a.x, a.ld_x, nullptr, 0, a.rows, a.k, 0}, W{(const T*)a.W, a.ld_w, nullptr, 0, a.n, a.k, 0};
    const bool as_is = in_place(x) && in_place(W);
    if (a.rows <= (sizeof(T) == 4 || as_is ? kFewRows : kFewLaid) && (!as_is || (int64_t)a.rows * a.k * a.n < kFewInPlace)) return linear_few(a, out, s);
    const ForwardRoom room = forward_room(a.ws, a.rows, a.k, a.n, a.type);
    Jobs<T> jobs{};
    const Scale scale = sizeof(T) == 4 ? kPerRow : kAsIs;
    if (!in_place(x)) add_job(jobs, x, room.x, scale);
    if (!in_place(W)) add_job(jobs, W, room.W, scale);
    const hipError_t e = run_jobs<T, false>(jobs, s);
    if (e != hipSuccess) return e;
    if (sizeof(T) == 4) {
      out.exp_r = room.x.exps;
      out.exp_c = room.W.exps;
    }
    return product<T, false, false>(product_args(in_place(x) ? operand(x, false) : operand(room.x, false),
                                                 in_place(W) ? operand(W, false) : operand(room.W, false), a.k, out),
                                    out, room.part, s);
  });
}

size_t linear_grad_workspace(int64_t rows, int64_t k, int64_t n, int type) { return backward_room(nullptr, rows, k, n, type).total; }

hipError_t launch_linear_grad(const LinearGradArgs& a, hipStream_t s) {
  return with_type(a.type, [&](auto t) {
    using T = decltype(t);
    constexpr bool kFloat = sizeof(T) == 4;
    BackwardRoom room = backward_room(a.ws, a.rows, a.k, a.n, a.type);
    const bool sloped = a.act != AMQ_ACT_NONE;
    const int passes = !kFloat && sloped && a.act != AMQ_ACT_RELU ? 2 : 1;
    if (passes == 1) room.d.low = room.d_columns.low = 0;
    const Source<T> d{(const T*)a.dy, a.ld_dy, sloped ? (const T*)a.pre : nullptr, a.ld_pre, a.rows, a.n, a.act};
    const Source<T> x{(const T*)a.x, a.ld_x, nullptr, 0, a.rows, a.k, 0}, W{(const T*)a.W, a.ld_w, nullptr, 0, a.n, a.k, 0};
    const bool scaled = kFloat || (a.type == AMQ_F16 && sloped);  // d, before it is rounded
    const bool products = a.dx || a.dW, d_laid = products && !in_place(d);
    hipError_t e = hipSuccess;
    // what goes by columns: sums of d; scales of float operands whose k runs down them, and of d in half; d itself without any
    ColumnJobs<T> columns{};
    int count = 0, widest = 0;
    auto column_job = [&](const ColumnJob<T>& job) {
      columns.job[count++] = job;
      const int width = job.to.p ? job.to.padded : job.from.cols;
      widest = width > widest ? width : widest;
    };
    const bool d_scales = kFloat ? a.dW != nullptr : scaled && products, d_here = d_laid && !scaled, one = d_scales && !kFloat;
    if (a.dbias || d_scales || d_here)
      column_job({d, a.dbias ? room.sums : nullptr, d_scales ? room.tops[0] : nullptr, d_here ? room.d : Laid{}, (T*)a.dbias,
                  d_scales ? room.d_columns.exps : nullptr, one});
    if (kFloat && a.dW) column_job({x, nullptr, room.tops[1], Laid{}, nullptr, room.x.exps, false});
    if (kFloat && a.dx) column_job({W, nullptr, room.tops[2], Laid{}, nullptr, room.W.exps, false});
    Jobs<T> jobs{};
    if (d_laid && scaled) {
      if (!kFloat) add_job(jobs, d, room.d, kOne);
      else if (a.dx) add_job(jobs, d, room.d, kPerRow, a.dW ? room.d_columns : Laid{});
      else add_job(jobs, d, room.d_columns, kPerColumn);
    }
    if (a.dx && !in_place(W)) add_job(jobs, W, room.W, kFloat ? kPerColumn : kAsIs);
    if (a.dW && !in_place(x)) add_job(jobs, x, room.x, kFloat ? kPerColumn : kAsIs);
    if (count) {
      const int64_t longest = kFloat && a.dx && a.n > a.rows ? a.n : a.rows;
      columns.count = count;
      columns.blocks = (int)div_up(widest, 32 * kPer16<T>);
      columns.parts = column_parts(longest, (int64_t)columns.blocks * count);
      const Jobs<T> beside = scaled ? Jobs<T>{} : jobs;
      const dim3 grid((unsigned)(columns.blocks * columns.parts * count + beside.first[beside.count]));
      if (sloped) columns_kernel<T, true><<<grid, dim3(256), 0, s>>>(columns, beside);
      else columns_kernel<T, false><<<grid, dim3(256), 0, s>>>(columns, beside);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      const bool to_add = columns.parts > 1 && (a.dbias || scaled);
      if (one) {
        if constexpr (std::is_same<T, f16>::value) {
          jobs.job[0].tops = room.tops[0];
          jobs.job[0].top_count = columns.parts * columns.blocks;
          const int64_t sum_blocks = to_add && a.dbias ? div_up(a.n, 32) : 0;
          lay_and_add_kernel<T><<<dim3((unsigned)(jobs.first[jobs.count] + sum_blocks)), dim3(256), 0, s>>>(jobs, columns);
          if ((e = hipGetLastError()) != hipSuccess) return e;
        }
      } else if (to_add) {
        columns_sum_kernel<T><<<dim3((unsigned)div_up(widest, 32), (unsigned)count), dim3(256), 0, s>>>(columns);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
    }
    // (what was not laid out beside the columns; of 16 bits that is without an activation)
    if (!count || (scaled && !one)) {
      if constexpr (kFloat) e = sloped ? run_jobs<T, true>(jobs, s) : run_jobs<T, false>(jobs, s);
      else e = run_jobs<T, false>(jobs, s);
      if (e != hipSuccess) return e;
    }
    if (!products) return hipSuccess;
    auto store_of = [&](void* y, int64_t ld, int M, const int* exp_r, const int* exp_c) {
      LinearStore<T> out{};
      out.act = AMQ_ACT_NONE;
      out.y = (T*)y;
      out.ld_y = ld;
      out.M = M;
      out.N = a.k;
      if (kFloat) {
        out.exp_r = exp_r;
        out.exp_c = exp_c;
      } else if (scaled) {
        out.exp_all = room.d.exps;
      }
      return out;
    };
    const LinearStore<T> to_x = store_of(a.dx, a.ld_dx, a.rows, room.d.exps, room.W.exps);
    const LinearStore<T> to_W = store_of(a.dW, a.ld_dw, a.n, room.d_columns.exps, room.x.exps);
    const MatmulArgs for_x = product_args(d_laid ? operand(room.d, false) : operand(d, false), in_place(W) ? operand(W, true) : operand(room.W, true), a.n, to_x);
    const MatmulArgs for_W = product_args(d_laid ? operand(room.d_columns, true) : operand(d, true), in_place(x) ? operand(x, true) : operand(room.x, true),
                                          a.rows, to_W);
    if (a.dx && a.dW) {
      const int planes = planes_of(a.type);
      const ProductPlan pair = plan_pair(a.rows, a.k, a.n, a.n, a.k, a.rows, planes, passes);
      if (pair.us < plan_product(a.rows, a.k, a.n, planes, 1, false, passes).us + plan_product(a.n, a.k, a.rows, planes, 1, false, passes).us) {
        if constexpr (kFloat) return launch_pair<f16, 2, false>(for_x, to_x, for_W, to_W, pair, s);
        else if (passes == 2) return launch_pair<T, 1, true>(for_x, to_x, for_W, to_W, pair, s);
        else return launch_pair<T, 1, false>(for_x, to_x, for_W, to_W, pair, s);
      }
    }
    if (a.dx) e = product<T, false, true>(for_x, to_x, room.part, s, passes);
    if (e == hipSuccess && a.dW) e = product<T, true, true>(for_W, to_W, room.part, s, passes);
    return e;
  });
}

}  // namespace amq
