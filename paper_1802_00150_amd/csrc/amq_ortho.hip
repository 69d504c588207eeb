// Orthogonalized updates: X = G / (|G|_F + eps), then `steps` times A = X X^T, B = b A + c A A, X = a X + B X.
//
// n <= m are the sizes of X (the transpose of G where G is tall).  Per step n^2 m + n^3 + 2 n^2 m operations, since A and
// A A are symmetric and only tiles on and below the diagonal are computed: bound by the matrix cores from about n = 512 on,
// by the chain of three dependent launches per step below.  Measured: 16384 x 4096 bfloat16 or half 14.0 to 14.4 ms for 4.5 Tflop, each as three half
// products: per step A 1069 us and B 271 = 770 and 760 TFLOP/s of half products (528 tiles in 512 places: the second round is almost empty, the
// matrix cores busy for 36 % of the cycles), X 1443 = 1140.  Two float matrices of 1200 x 300 135 us, 17 launches of 6 to 10; one half matrix of 2048 x 512 155.
//
// Iterates, A and B are held as half values times 2^12, in two planes (22 bits).  Singular values stay below about 1.2 with the usual coefficients, so
// nothing comes near 65504 / 4096 = 16, and half's smallest step is 2^-36 of an entry of 1.  Two planes lose 3e-7 of the result in the 2-norm
// over five steps.  One plane would lose 1.4e-3, as much as the rounding to bfloat16 (1.7e-3) once more, in a third of the
// products: 16384 x 4096 took 4.4 ms with one.
// X lies as G does: of a wide G, X X^T contracts along rows and B X down the columns of X; of a tall one, which is the
// transpose of X, X X^T contracts down its columns and B X along its rows.
// The norm is summed in binary64, so that no gradient's scale overflows its square.
#include "../../include/amq.h"

#include "amq_device.h"
#include "amq_matmul_body.h"
#include "amq_train.h"

namespace amq {
namespace {

constexpr int kScaleBits = 12;
constexpr float kInvScale = 1.0f / 4096.0f;
constexpr int kNormParts = 1024;  // sums of squares per matrix: four workgroups of 256 per compute unit

struct __attribute__((packed, aligned(8))) Half4 {
  f16 v[4];
};

constexpr int kPlanes = 2;

// A matrix of scaled values of two halves, [batch][rows][ld]; zeros from `cols` to `padded`, a multiple of 64.
struct Planes {
  f16* p;
  int64_t ld, batch;
  int rows, cols, padded;
  __device__ __forceinline__ f16* at(int z, int row, int col) const { return p + z * batch + row * ld + high_part(col); }
  // four values along a row (col a multiple of 4)
  __device__ __forceinline__ f32x4 load(int z, int row, int col) const {
    const f16* q = at(z, row, col);
    const Half4 h = *reinterpret_cast<const Half4*>(q);
    const Half4 l = *reinterpret_cast<const Half4*>(q + 32);
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)h.v[i] + (float)l.v[i];
    return v;
  }
  __device__ __forceinline__ bool has(int row, int col) const { return row < rows && col < padded; }
  __device__ __forceinline__ void store(int z, int row, int col, f32x4 v) const {
    f16* q = at(z, row, col);
    Half4 h, l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float s = col + i < cols ? v[i] : 0.0f;
      h.v[i] = (f16)s;
      l.v[i] = (f16)(s - (float)h.v[i]);
    }
    *reinterpret_cast<Half4*>(q) = h;
    *reinterpret_cast<Half4*>(q + 32) = l;
  }
};

// What the epilogues below have in common: nothing per column, four scaled values of a matrix per call.
struct OrthoStore {
  struct Column {};
  typedef f32x4 Extra;
  __device__ __forceinline__ Column column(int, int) const { return {}; }
};
// A = X X^T, both triangles from the lower tiles.
struct GramStore : OrthoStore {
  static constexpr bool kTransposed = true;
  Planes A;
  explicit GramStore(const Planes& a) : A(a) {}
  __device__ __forceinline__ f32x4 fetch(int, int, int) const { return f32x4{}; }
  __device__ __forceinline__ void put(int z, int m, int n, f32x4 v, const Column&, const f32x4&) const {
    if (A.has(m, n)) A.store(z, m, n, v * kInvScale);
  }
};
// B = b A + c A A, A being symmetric as well.
struct PolynomialStore : OrthoStore {
  static constexpr bool kTransposed = true;
  Planes A, B;
  float b, c;
  PolynomialStore(const Planes& a_, const Planes& b_, float fb, float fc) : A(a_), B(b_), b(fb), c(fc) {}
  __device__ __forceinline__ f32x4 fetch(int z, int m, int n) const { return A.has(m, n) ? A.load(z, m, n) : f32x4{}; }
  __device__ __forceinline__ void put(int z, int m, int n, f32x4 v, const Column&, const f32x4& a) const {
    if (B.has(m, n)) B.store(z, m, n, a * b + v * (c * kInvScale));
  }
};
// X = a X + B X.  (Not in place: X is an operand of the product.)
struct UpdateStore : OrthoStore {
  static constexpr bool kTransposed = false;
  Planes X, next;
  float a;
  UpdateStore(const Planes& x, const Planes& n, float fa) : X(x), next(n), a(fa) {}
  __device__ __forceinline__ f32x4 fetch(int z, int m, int n) const { return X.has(m, n) ? X.load(z, m, n) : f32x4{}; }
  __device__ __forceinline__ void put(int z, int m, int n, f32x4 v, const Column&, const f32x4& x) const {
    if (X.has(m, n)) next.store(z, m, n, x * a + v * kInvScale);
  }
};
// The last X.
template <typename T>
struct ResultStore : OrthoStore {
  static constexpr bool kTransposed = false;
  Planes X;
  T* out;
  int64_t ld, batch;
  float a;
  ResultStore(const Planes& x, T* o, int64_t l, int64_t b, float fa) : X(x), out(o), ld(l), batch(b), a(fa) {}
  __device__ __forceinline__ f32x4 fetch(int z, int m, int n) const { return X.has(m, n) ? X.load(z, m, n) : f32x4{}; }
  __device__ __forceinline__ void put(int z, int m, int n, f32x4 v, const Column&, const f32x4& x) const {
    if (m >= X.rows || n >= X.cols) return;
    v = (x * a + v * kInvScale) * kInvScale;
    T* q = out + z * batch + m * ld + n;
    struct __attribute__((packed, aligned(sizeof(T)))) Four {
      T v[4];
    } o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = (T)v[i];
    if (n + 4 <= X.cols) *reinterpret_cast<Four*>(q) = o;
    else
      for (int i = 0; i < X.cols - n; ++i) q[i] = (T)v[i];
  }
};

template <typename T>
struct Gradient {
  const T* p;
  int64_t ld, batch;
  int rows, cols;
};

// Sums of squares, kNormParts of them per matrix.  Bound by memory: 16384 x 4096 bfloat16 (134 MB) 35 us = 3.8 TB/s (one piece of
// a row under way instead of four, and a quarter of the workgroups: 85).
template <typename T>
__global__ __launch_bounds__(256) void ortho_norm_kernel(Gradient<T> G, double* parts) {
  __shared__ double scratch[4];
  constexpr int V = kPer16<T>;
  const T* p = G.p + blockIdx.y * G.batch;
  double s = 0.0;
  // pieces of 256 x V values of a row, dealt to the workgroups in turn
  const int64_t across = (G.cols + 256 * V - 1) / (256 * V), pieces = across * G.rows;
  constexpr int kAhead = 4;  // pieces under way
  for (int64_t i = blockIdx.x; i < pieces; i += (int64_t)kAhead * gridDim.x) {
    float v[kAhead][V];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t at = i + (int64_t)u * gridDim.x, row = at / across;
      const int col = ((int)(at % across) * 256 + (int)threadIdx.x) * V;
      load16(p + row * G.ld + col, at < pieces ? G.cols - col : 0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int q = 0; q < V; ++q) s += (double)v[u][q] * (double)v[u][q];
  }
  s = block_sum<4>(s, scratch);
  if (threadIdx.x == 0) parts[(int64_t)blockIdx.y * kNormParts + blockIdx.x] = s;
}

// 1 / (|G| + eps) of matrix z from its partial sums, by a whole workgroup of 256: as a number in [1/2, 1) and an exponent, since without
// eps it may be larger than binary32 numbers are.
struct Factor {
  float m;
  int e;
  __device__ __forceinline__ float times(float v) const { return ldexpf(v, e) * m; }
};
__device__ __forceinline__ Factor inverse_norm(const double* parts, int z, int count, float eps, double* scratch) {
  double s = 0.0;
  for (int i = threadIdx.x; i < count; i += 256) s += parts[(int64_t)z * kNormParts + i];
  Factor f;
  f.m = (float)frexp(1.0 / (sqrt(block_sum<4>(s, scratch)) + (double)eps), &f.e);
  return f;
}

// X_0: 8 numbers per lane, rows dealt to the workgroups.  Bound by memory: 16384 x 4096 bfloat16 (403 MB) 110 us = 3.7 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void ortho_begin_kernel(Gradient<T> G, const double* parts, int count, float eps, Planes X) {
  __shared__ double scratch[4];
  const int z = blockIdx.z;
  Factor scale = inverse_norm(parts, z, count, eps, scratch);
  scale.e += kScaleBits;
  const T* p = G.p + z * G.batch;
  const int per_row = X.padded / 8;
  const int64_t total = (int64_t)G.rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per_row;
    const int col = (int)(i % per_row) * 8;
    float v[8];
    load_params<T, 8>(p, row * G.ld + col, G.cols - col, 0.0f, v);
#pragma unroll
    for (float& u : v) u = scale.times(u);
    X.store(z, (int)row, col, f32x4{v[0], v[1], v[2], v[3]});
    X.store(z, (int)row, col + 4, f32x4{v[4], v[5], v[6], v[7]});
  }
}

// No steps: the scaled gradient itself.
template <typename T>
__global__ __launch_bounds__(256) void ortho_scale_kernel(Gradient<T> G, const double* parts, int count, float eps, T* out, int64_t ld, int64_t batch) {
  __shared__ double scratch[4];
  const int z = blockIdx.z;
  const Factor scale = inverse_norm(parts, z, count, eps, scratch);
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= G.cols) return;
  for (int64_t row = blockIdx.y; row < G.rows; row += gridDim.y)
    out[z * batch + row * ld + col] = (T)scale.times((float)G.p[z * G.batch + row * G.ld + col]);
}

struct Room {
  f16 *X[2], *A, *B;
  double* parts;
  float* part;
  int64_t n, m;
  size_t total;
};
ProductPlan gram_plan(const Room& r, int64_t batch) { return plan_product(r.n, r.n, r.m, kPlanes, batch, true); }
ProductPlan polynomial_plan(const Room& r, int64_t batch) { return plan_product(r.n, r.n, r.n, kPlanes, batch, true); }
ProductPlan update_plan(const Room& r, bool tall, int64_t batch) {
  return plan_product(tall ? r.m : r.n, tall ? r.n : r.m, r.n, kPlanes, batch, false);
}

Room room_of(void* ws, int64_t batch, int64_t rows, int64_t cols) {
  Room r{};
  r.n = rows < cols ? rows : cols;
  r.m = rows < cols ? cols : rows;
  char* base = static_cast<char*>(ws);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    void* p = base ? base + off : nullptr;
    off += (bytes + 255) & ~size_t(255);
    return p;
  };
  const size_t value = sizeof(f16) * (size_t)kPlanes * batch;
  for (f16*& x : r.X) x = (f16*)take(value * rows * pad64(cols));
  r.A = (f16*)take(value * r.n * pad64(r.n));
  r.B = (f16*)take(value * r.n * pad64(r.n));
  r.parts = (double*)take(sizeof(double) * kNormParts * (size_t)batch);
  size_t most = gram_plan(r, batch).part_bytes;
  for (size_t b : {polynomial_plan(r, batch).part_bytes, update_plan(r, rows > cols, batch).part_bytes})
    if (b > most) most = b;
  r.part = (float*)take(most);
  r.total = off;
  return r;
}

template <typename T>
hipError_t run(const OrthoArgs& o, hipStream_t s) {
  const Room r = room_of(o.ws, o.batch, o.rows, o.cols);
  const bool tall = o.rows > o.cols;
  const Gradient<T> G{(const T*)o.G, o.ld_g, o.stride_g, o.rows, o.cols};
  T* out = (T*)o.out;
  auto planes = [&](f16* p, int64_t rows, int64_t cols) {
    const int64_t padded = pad64(cols);
    return Planes{p, kPlanes * padded, rows * kPlanes * padded, (int)rows, (int)cols, (int)padded};
  };
  const Planes X[2] = {planes(r.X[0], o.rows, o.cols), planes(r.X[1], o.rows, o.cols)};
  const Planes A = planes(r.A, r.n, r.n), B = planes(r.B, r.n, r.n);

  const int64_t pieces = div_up(o.cols, 256 * kPer16<T>) * o.rows;
  const int count = (int)(pieces < kNormParts ? pieces : kNormParts);
  ortho_norm_kernel<T><<<dim3((unsigned)count, (unsigned)o.batch), dim3(256), 0, s>>>(G, r.parts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (o.steps == 0) {
    ortho_scale_kernel<T><<<dim3((unsigned)div_up(o.cols, 256), (unsigned)(o.rows < 1024 ? o.rows : 1024), (unsigned)o.batch), dim3(256), 0, s>>>(
        G, r.parts, count, o.eps, out, o.ld_out, o.stride_out);
    return hipGetLastError();
  }
  const int64_t begin = div_up(o.rows * (int64_t)(X[0].padded / 8), 256);
  ortho_begin_kernel<T><<<dim3((unsigned)(begin < 2048 ? begin : 2048), 1, (unsigned)o.batch), dim3(256), 0, s>>>(G, r.parts, count, o.eps, X[0]);
  if ((e = hipGetLastError()) != hipSuccess) return e;

  auto args = [&](const Planes& rows, bool rows_down, const Planes& cols, bool cols_down, int64_t k, bool lower) {
    MatmulArgs g{};
    // (of an operand whose k runs down columns the padding counts as rows: zeros, and a multiple of 8)
    g.r = {rows.p, rows.ld, rows.batch, rows_down ? rows.padded : rows.rows};
    g.c = {cols.p, cols.ld, cols.batch, cols_down ? cols.padded : cols.rows};
    g.M = rows_down ? rows.cols : rows.rows;
    g.N = cols_down ? cols.cols : cols.rows;
    g.k = (int)k;
    g.lower = lower;
    return g;
  };
  const ProductPlan gram = gram_plan(r, o.batch), polynomial = polynomial_plan(r, o.batch), update = update_plan(r, tall, o.batch);
  for (int i = 0; i < o.steps; ++i) {
    const Planes&now = X[i & 1], &next = X[(i + 1) & 1];
    const MatmulArgs xx = args(now, tall, now, tall, r.m, true);
    e = tall ? launch_product<f16, kPlanes, true, true>(xx, gram, o.batch, GramStore(A), r.part, s)
             : launch_product<f16, kPlanes, false, false>(xx, gram, o.batch, GramStore(A), r.part, s);
    if (e != hipSuccess) return e;
    e = launch_product<f16, kPlanes, false, false>(args(A, false, A, false, r.n, true), polynomial, o.batch, PolynomialStore(A, B, o.b, o.c), r.part, s);
    if (e != hipSuccess) return e;
    auto multiply = [&](const auto& store) {
      return tall ? launch_product<f16, kPlanes, false, false>(args(now, false, B, false, r.n, false), update, o.batch, store, r.part, s)
                  : launch_product<f16, kPlanes, false, true>(args(B, false, now, true, r.n, false), update, o.batch, store, r.part, s);
    };
    e = i + 1 < o.steps ? multiply(UpdateStore(now, next, o.a)) : multiply(ResultStore<T>(now, out, o.ld_out, o.stride_out, o.a));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t ortho_workspace(int64_t batch, int64_t rows, int64_t cols) { return room_of(nullptr, batch, rows, cols).total; }

hipError_t launch_ortho(const OrthoArgs& a, hipStream_t s) {
  if (a.type == AMQ_F32) return run<float>(a, s);
  return a.type == AMQ_F16 ? run<f16>(a, s) : run<bf16>(a, s);
}

}  // namespace amq
