// Linear layers: y = act(x W^T + b) + residual, and the backward pass dx = d W, dW = d^T x, db = sum_rows d with
// d = dy act'(z).
//
// The products run on the 16-bit matrix cores (amq_matmul_body.h).  bfloat16 and half operands whose rows lie on 16 bytes
// and hold a multiple of 64 values are read where they are.  Anything else is laid out first: rows padded with zeros;
// transposed where the contraction runs along columns (W in dx, d and x in dW); float values scaled by a power of two
// per row of the operand and split into two halves, 22 bits together.  (A binary32 matrix instruction has 1/16 of the rate
// of a half one; three half products of split operands have 1/3, with the error of binary32 products.)  The scale puts the
// row's largest value into [2^14, 2^15), so no product overflows, and half's smallest step is 2^-38 of that value.  d in
// half is scaled the same way before it is rounded: gradients divided by a batch's size lie where half has few digits.
//
// A few rows (a token's vector) are multiplied on the vector units: there W is read once, and nothing else matters.
#include "../../include/amq.h"

#include "amq_device.h"
#include "amq_matmul_body.h"
#include "amq_train.h"

namespace amq {
namespace {

__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case AMQ_ACT_RELU: return z > 0.0f ? z : 0.0f;
    case AMQ_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    case AMQ_ACT_SILU: return z / (1.0f + expf(-z));
    case AMQ_ACT_SIGMOID: return 1.0f / (1.0f + expf(-z));
    case AMQ_ACT_TANH: return tanhf(z);
  }
  return z;
}
__device__ __forceinline__ float slope(float z, int act) {
  switch (act) {
    case AMQ_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case AMQ_ACT_GELU:
      return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * (0.39894228040143268f * expf(-0.5f * z * z));
    case AMQ_ACT_SILU: {
      const float s = 1.0f / (1.0f + expf(-z));
      return s * (1.0f + z * (1.0f - s));
    }
    case AMQ_ACT_SIGMOID: {
      const float s = 1.0f / (1.0f + expf(-z));
      return s * (1.0f - s);
    }
    case AMQ_ACT_TANH: {
      const float t = tanhf(z);
      return 1.0f - t * t;
    }
  }
  return 1.0f;
}

template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Group {
  T v[V];
};

// bias, activation, residual: what becomes of a product's values.
template <typename T>
struct LinearStore {
  static constexpr bool kTransposed = false;
  T *y, *pre;
  const T *bias, *residual;
  const int *exp_r, *exp_c;  // scales of the operands' rows, or null
  int64_t ld_y, ld_pre, ld_r;
  int M, N, act;

  template <int V>
  __device__ __forceinline__ void values(int m, int n, float (&v)[V]) const {
    const int valid = N - n;
    float b[V];
    load_params<T, V>(bias, n, valid, 0.0f, b);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += b[i];
    if (pre) put<V>(pre + m * ld_pre + n, valid, v);
    if (act != AMQ_ACT_NONE)
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = activate(v[i], act);
    if (residual) {
      load_params<T, V>(residual, m * ld_r + n, valid, 0.0f, b);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += b[i];
    }
    put<V>(y + m * ld_y + n, valid, v);
  }
  template <int V>
  static __device__ __forceinline__ void put(T* p, int valid, const float (&v)[V]) {
    if (valid >= V) {
      Group<T, V> o;
#pragma unroll
      for (int i = 0; i < V; ++i) o.v[i] = (T)v[i];
      *reinterpret_cast<Group<T, V>*>(p) = o;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < valid) p[i] = (T)v[i];
    }
  }
  __device__ __forceinline__ void along_n(int, int m, int n, f32x4 v4) const {
    if (m >= M || n >= N) return;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = v4[i];
    if (exp_r || exp_c) {
      const int e = exp_r ? exp_r[m] : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < N) v[i] = ldexpf(v[i], -(e + (exp_c ? exp_c[n + i] : 0)));
    }
    values<4>(m, n, v);
  }
  __device__ __forceinline__ void along_m(int, int, int, f32x4) const {}
};

// ---- a few rows: workgroup = 4 rows of W, its waves share the row's k
constexpr int kFewRows = 8;
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
    if (m < out.M && n < out.N) {
      float v[1] = {sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] + sums[3][threadIdx.x]};
      out.template values<1>(m, n, v);
    }
  }
}

// ---- laying operands out
// One matrix as it lies in memory; with `pre`, times the slope of the activation there.
template <typename T>
struct Source {
  const T* p;
  int64_t ld;
  const T* pre;
  int64_t ld_pre;
  int rows, cols, act;
  template <int V>
  __device__ __forceinline__ void load(int64_t row, int col, float (&v)[V]) const {
    load_params<T, V>(p, row * ld + col, cols - col, 0.0f, v);
    if (pre) {
      float z[V];
      load_params<T, V>(pre, row * ld_pre + col, cols - col, 0.0f, z);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= slope(z[i], act);
    }
  }
};
// One operand in the layout of the product kernel: rows of kp values (a multiple of 64), in two halves for float.
struct Laid {
  uint16_t* p;
  int* exps;      // scale per row of the operand, or null: values as they are
  int64_t ld;     // 16-bit values per row
  int rows, kp;
};
template <typename T>
struct Job {
  Source<T> from;
  Laid to;
  bool columns;  // the operand's rows are the matrix's columns
};
constexpr int kMaxJobs = 4;
template <typename T>
struct Jobs {
  Job<T> job[kMaxJobs];
  int first[kMaxJobs + 1];  // workgroups of job j: first[j] .. first[j + 1]
  int count;
};

__device__ __forceinline__ int scale_exponent(float largest) { return largest > 0.0f ? 14 - ilogbf(largest) : 0; }
__device__ __forceinline__ void split(float v, uint16_t& hi, uint16_t& lo) {
  const f16 h = (f16)v;
  const f16 l = (f16)(v - (float)h);
  hi = __builtin_bit_cast(uint16_t, h);
  lo = __builtin_bit_cast(uint16_t, l);
}
// 8 values of an operand's row as the products take them.
template <typename T>
__device__ __forceinline__ void put8(const Laid& to, int row, int at, float (&v)[8], int e) {
  constexpr bool kFloat = sizeof(T) == 4;
  Group<uint16_t, 8> hi, lo;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (to.exps) v[i] = ldexpf(v[i], e);
    if constexpr (kFloat) split(v[i], hi.v[i], lo.v[i]);
    else hi.v[i] = __builtin_bit_cast(uint16_t, (T)v[i]);
  }
  uint16_t* q = to.p + row * to.ld + (kFloat ? high_part(at) : at);
  *reinterpret_cast<uint4*>(q) = __builtin_bit_cast(uint4, hi);
  if constexpr (kFloat) *reinterpret_cast<uint4*>(q + 32) = __builtin_bit_cast(uint4, lo);
}

// Operand rows = matrix rows: one wave per row (16 rows per workgroup).
template <typename T>
__device__ __forceinline__ void lay_rows(const Job<T>& j, int block) {
  for (int r = 0; r < 4; ++r) {
    const int row = block * 16 + r * 4 + wave_id();
    if (row >= j.to.rows) return;
    int e = 0;
    if (j.to.exps) {
      float largest = 0.0f;
      for (int c = lane_id() * 4; c < j.from.cols; c += 256) {
        float v[4];
        j.from.template load<4>(row, c, v);
        largest = fmaxf(largest, fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))));
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) largest = fmaxf(largest, __shfl_xor(largest, o, 64));
      e = scale_exponent(largest);
      if (lane_id() == 0) j.to.exps[row] = e;
    }
    for (int c = lane_id() * 8; c < j.to.kp; c += 512) {
      float v[8];
      j.from.template load<8>(row, c, v);  // zeros past the end
      put8<T>(j.to, row, c, v, e);
    }
  }
}

// Operand rows = matrix columns: 64 x 64 values per workgroup, turned in LDS.
template <typename T>
__device__ __forceinline__ void lay_columns(const Job<T>& j, int block, float (*t)[65]) {
  const int across = (j.from.cols + 63) / 64;
  const int r0 = block / across * 64, c0 = block % across * 64;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 16 + (threadIdx.x >> 4), col = (threadIdx.x & 15) * 4;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (r0 + row < j.from.rows) j.from.template load<4>(r0 + row, c0 + col, v);
#pragma unroll
    for (int q = 0; q < 4; ++q) t[row][col + q] = v[q];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = i * 32 + (threadIdx.x >> 3), row = (threadIdx.x & 7) * 8;
    if (c0 + col < j.from.cols) {
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = t[row + q][col];
      put8<T>(j.to, c0 + col, r0 + row, v, j.to.exps ? j.to.exps[c0 + col] : 0);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void lay_kernel(Jobs<T> jobs) {
  __shared__ float t[64][65];
  int j = 0;
  while (j + 1 < jobs.count && (int)blockIdx.x >= jobs.first[j + 1]) ++j;
  const int block = blockIdx.x - jobs.first[j];
  if (jobs.job[j].columns) lay_columns(jobs.job[j], block, t);
  else lay_rows(jobs.job[j], block);
}

// ---- sums and largest values of columns: partial ones over every gridDim.y-th row, then over those
constexpr int kMaxColumnParts = 64;
template <typename T>
struct ColumnJob {
  Source<T> from;
  float *sums, *largest;  // [gridDim.y][cols], or null
  void* total;            // T [cols]: the sums
  int* exps;              // [cols]: scales
};
template <typename T>
struct ColumnJobs {
  ColumnJob<T> job[3];
};
template <typename T>
__global__ __launch_bounds__(256) void columns_kernel(ColumnJobs<T> jobs) {
  const ColumnJob<T>& j = jobs.job[blockIdx.z];
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= j.from.cols) return;
  float s = 0.0f, largest = 0.0f;
#pragma unroll 4
  for (int64_t row = blockIdx.y; row < j.from.rows; row += gridDim.y) {
    float v = (float)j.from.p[row * j.from.ld + c];
    if (j.from.pre) v *= slope((float)j.from.pre[row * j.from.ld_pre + c], j.from.act);
    s += v;
    largest = fmaxf(largest, fabsf(v));
  }
  if (j.sums) j.sums[(int64_t)blockIdx.y * j.from.cols + c] = s;
  if (j.largest) j.largest[(int64_t)blockIdx.y * j.from.cols + c] = largest;
}
template <typename T>
__global__ __launch_bounds__(256) void columns_sum_kernel(ColumnJobs<T> jobs, int parts) {
  const ColumnJob<T>& j = jobs.job[blockIdx.y];
  __shared__ float sums[8][33], tops[8][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, cols = j.from.cols;
  if (blockIdx.x * 32 >= (unsigned)cols) return;
  float s = 0.0f, top = 0.0f;
  if (c < cols)
    for (int p = group; p < parts; p += 8) {
      if (j.sums) s += j.sums[(int64_t)p * cols + c];
      if (j.largest) top = fmaxf(top, j.largest[(int64_t)p * cols + c]);
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
  if (j.total) ((T*)j.total)[c] = (T)s;
  if (j.exps) j.exps[c] = scale_exponent(top);
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
Laid lay_room(Carve& w, int64_t rows, int64_t k, int type, bool scaled) {
  Laid l;
  l.rows = (int)rows;
  l.kp = (int)pad64(k);
  l.ld = planes_of(type) * (int64_t)l.kp;
  l.p = (uint16_t*)w.take(2 * (size_t)(rows * l.ld));
  l.exps = scaled ? (int*)w.take(sizeof(int) * (size_t)rows) : nullptr;
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
  if (rows > kFewRows) {
    r.x = lay_room(w, rows, k, type, type == AMQ_F32);
    r.W = lay_room(w, n, k, type, type == AMQ_F32);
    r.part = (float*)w.take(plan_product(rows, n, pad64(k), planes_of(type), 1, false).part_bytes);
  }
  r.total = w.off;
  return r;
}

struct BackwardRoom {
  Laid d, d_cols, W_cols, x_cols;
  float *sums, *tops[3];
  float* part;
  int column_parts;
  size_t total;
};
BackwardRoom backward_room(void* ws, int64_t rows, int64_t k, int64_t n, int type) {
  Carve w(ws);
  BackwardRoom r{};
  r.d = lay_room(w, rows, n, type, type != AMQ_BF16);
  r.W_cols = lay_room(w, k, n, type, type == AMQ_F32);
  r.d_cols = lay_room(w, n, rows, type, type != AMQ_BF16);
  r.x_cols = lay_room(w, k, rows, type, type == AMQ_F32);
  const int64_t most = rows > n ? rows : n;  // the longest column: of d and x, of W
  r.column_parts = (int)(most < kMaxColumnParts ? most : kMaxColumnParts);
  r.sums = (float*)w.take(sizeof(float) * r.column_parts * (size_t)n);
  if (type != AMQ_BF16) r.tops[0] = (float*)w.take(sizeof(float) * r.column_parts * (size_t)n);
  if (type == AMQ_F32) {
    r.tops[1] = (float*)w.take(sizeof(float) * r.column_parts * (size_t)k);
    r.tops[2] = (float*)w.take(sizeof(float) * r.column_parts * (size_t)k);
  }
  const size_t a = plan_product(rows, k, pad64(n), planes_of(type), 1, false).part_bytes;
  const size_t b = plan_product(n, k, pad64(rows), planes_of(type), 1, false).part_bytes;
  r.part = (float*)w.take(a > b ? a : b);
  r.total = w.off;
  return r;
}

template <typename F>
hipError_t with_type(int type, F f) {
  return type == AMQ_F32 ? f(float()) : type == AMQ_BF16 ? f(bf16()) : f(f16());
}

// Whether the product kernel can read a matrix where it is.
template <typename T>
bool in_place(const void* p, int64_t ld, int64_t k) {
  return sizeof(T) == 2 && k % 64 == 0 && ld % 8 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}
template <typename T>
void add_job(Jobs<T>& jobs, const Source<T>& from, const Laid& to, bool columns) {
  const int64_t blocks = columns ? pad64(from.rows) / 64 * div_up(from.cols, 64) : div_up(from.rows, 16);
  jobs.job[jobs.count] = {from, to, columns};
  jobs.first[jobs.count + 1] = jobs.first[jobs.count] + (int)blocks;
  ++jobs.count;
}
template <typename T>
hipError_t run_jobs(const Jobs<T>& jobs, hipStream_t s) {
  if (!jobs.count) return hipSuccess;
  lay_kernel<T><<<dim3((unsigned)jobs.first[jobs.count]), dim3(256), 0, s>>>(jobs);
  return hipGetLastError();
}
MatmulOperand operand(const Laid& l) { return {l.p, l.ld, 0, l.rows}; }

template <typename T>
hipError_t product(const MatmulOperand& r, const MatmulOperand& c, int64_t k, const LinearStore<T>& out, float* part, hipStream_t s) {
  MatmulArgs g{};
  g.r = r;
  g.c = c;
  g.M = out.M;
  g.N = out.N;
  g.tiles_k = (int)pad64(k);
  const ProductPlan p = plan_product(out.M, out.N, pad64(k), sizeof(T) == 4 ? 2 : 1, 1, false);
  if constexpr (sizeof(T) == 4) return launch_product<f16, 2>(g, p, 1, out, part, s);
  else return launch_product<T, 1>(g, p, 1, out, part, s);
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

ProductPlan plan_product(int64_t M, int64_t N, int64_t k, int planes, int64_t batch, bool lower) {
  auto tiles = [&](int64_t t) {
    const int64_t a = div_up(M, t), b = div_up(N, t);
    return batch * (lower ? a * (a + 1) / 2 : a * b);
  };
  ProductPlan p{};
  p.splits = 1;
  p.tile = planes == 1 && tiles(256) >= 192 ? 256 : tiles(128) >= 192 ? 128 : 64;
  const int64_t steps = k / stage_of(planes);
  p.tiles_per_split = (int)steps;
  if (p.tile == 64 && tiles(64) < 256) {
    int64_t splits = 512 / tiles(64);
    if (splits > steps / 4) splits = steps / 4;
    if (splits > 1) {
      p.tiles_per_split = (int)div_up(steps, 2 * splits) * 2;
      p.splits = (int)div_up(steps, p.tiles_per_split);
      if (p.splits > 1) p.part_bytes = sizeof(float) * (size_t)batch * p.splits * M * ((N + 3) & ~int64_t(3));
    }
  }
  return p;
}

size_t linear_workspace(int64_t rows, int64_t k, int64_t n, int type) { return forward_room(nullptr, rows, k, n, type).total; }

hipError_t launch_linear(const LinearArgs& a, hipStream_t s) {
  return with_type(a.type, [&](auto t) {
    using T = decltype(t);
    LinearStore<T> out{(T*)a.y, (T*)a.pre, (const T*)a.bias, (const T*)a.residual, nullptr, nullptr, a.ld_y, a.ld_pre, a.ld_r, a.rows, a.n, a.act};
    if (a.rows <= kFewRows) return linear_few(a, out, s);
    const ForwardRoom room = forward_room(a.ws, a.rows, a.k, a.n, a.type);
    Jobs<T> jobs{};
    MatmulOperand x{a.x, a.ld_x, 0, a.rows}, W{a.W, a.ld_w, 0, a.n};
    if (!in_place<T>(a.x, a.ld_x, a.k)) {
      add_job(jobs, Source<T>{(const T*)a.x, a.ld_x, nullptr, 0, a.rows, a.k, 0}, room.x, false);
      x = operand(room.x);
    }
    if (!in_place<T>(a.W, a.ld_w, a.k)) {
      add_job(jobs, Source<T>{(const T*)a.W, a.ld_w, nullptr, 0, a.n, a.k, 0}, room.W, false);
      W = operand(room.W);
    }
    const hipError_t e = run_jobs(jobs, s);
    if (e != hipSuccess) return e;
    if (sizeof(T) == 4) {
      out.exp_r = room.x.exps;
      out.exp_c = room.W.exps;
    }
    return product(x, W, a.k, out, room.part, s);
  });
}

size_t linear_grad_workspace(int64_t rows, int64_t k, int64_t n, int type) { return backward_room(nullptr, rows, k, n, type).total; }

hipError_t launch_linear_grad(const LinearGradArgs& a, hipStream_t s) {
  return with_type(a.type, [&](auto t) {
    using T = decltype(t);
    constexpr bool kFloat = sizeof(T) == 4;
    BackwardRoom room = backward_room(a.ws, a.rows, a.k, a.n, a.type);
    const bool sloped = a.act != AMQ_ACT_NONE;
    const bool scaled = kFloat || (a.type == AMQ_F16 && sloped);  // d, before it is rounded
    if (!scaled) room.d.exps = room.d_cols.exps = nullptr;
    const Source<T> d{(const T*)a.dy, a.ld_dy, sloped ? (const T*)a.pre : nullptr, a.ld_pre, a.rows, a.n, a.act};
    const Source<T> x{(const T*)a.x, a.ld_x, nullptr, 0, a.rows, a.k, 0}, W{(const T*)a.W, a.ld_w, nullptr, 0, a.n, a.k, 0};
    hipError_t e = hipSuccess;
    // sums of d's columns, and the scales of operands whose rows are columns
    ColumnJobs<T> columns{};
    int count = 0, widest = 0;
    auto column_job = [&](const Source<T>& from, float* sums, float* tops, void* total, int* exps) {
      columns.job[count++] = {from, sums, tops, total, exps};
      widest = from.cols > widest ? from.cols : widest;
    };
    const bool scaled_columns = scaled && a.dW;
    if (a.dbias || scaled_columns)
      column_job(d, a.dbias ? room.sums : nullptr, scaled_columns ? room.tops[0] : nullptr, a.dbias, scaled_columns ? room.d_cols.exps : nullptr);
    if (kFloat && a.dW) column_job(x, nullptr, room.tops[1], nullptr, room.x_cols.exps);
    if (kFloat && a.dx) column_job(W, nullptr, room.tops[2], nullptr, room.W_cols.exps);
    if (count) {
      columns_kernel<T><<<dim3((unsigned)div_up(widest, 256), (unsigned)room.column_parts, (unsigned)count), dim3(256), 0, s>>>(columns);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      columns_sum_kernel<T><<<dim3((unsigned)div_up(widest, 32), (unsigned)count), dim3(256), 0, s>>>(columns, room.column_parts);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    Jobs<T> jobs{};
    MatmulOperand rows_of_d{a.dy, a.ld_dy, 0, a.rows};
    if (a.dx) {
      if (sloped || !in_place<T>(a.dy, a.ld_dy, a.n)) {
        add_job(jobs, d, room.d, false);
        rows_of_d = operand(room.d);
      }
      add_job(jobs, W, room.W_cols, true);
    }
    if (a.dW) {
      add_job(jobs, d, room.d_cols, true);
      add_job(jobs, x, room.x_cols, true);
    }
    if ((e = run_jobs(jobs, s)) != hipSuccess) return e;
    LinearStore<T> out{};
    out.act = AMQ_ACT_NONE;
    if (a.dx) {
      out.y = (T*)a.dx;
      out.ld_y = a.ld_dx;
      out.M = a.rows;
      out.N = a.k;
      out.exp_r = room.d.exps;
      out.exp_c = room.W_cols.exps;
      if ((e = product(rows_of_d, operand(room.W_cols), a.n, out, room.part, s)) != hipSuccess) return e;
    }
    if (a.dW) {
      out.y = (T*)a.dW;
      out.ld_y = a.ld_dw;
      out.M = a.n;
      out.N = a.k;
      out.exp_r = room.d_cols.exps;
      out.exp_c = room.x_cols.exps;
      e = product(operand(room.d_cols), operand(room.x_cols), a.rows, out, room.part, s);
    }
    return e;
  });
}

}  // namespace amq
