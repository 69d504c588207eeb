// Layer normalization, forward and backward.
//
//   mu = sum x / n,  var = sum (x - mu)^2 / n,  r = 1 / sqrt(var + eps),  y = (x - mu) r w + b
//   g = dy w,  z = (x - mu) r,  dx = r (g - mean(g) - z mean(g z)),  dw = sum_rows dy z,  db = sum_rows dy
//
// About 10 operations per entry against 4 to 12 bytes: bound by memory, or by latency for few rows.  So every entry is read
// once and kept in registers between the sums and the output: a row belongs to one wave (up to 1024 entries; its sums need
// no barrier) or to one workgroup of 4, 8 or 16 waves (up to 4096, 8192, 16384).  The variance is formed from x - mu, not from the sum
// of squares, since the entries are there anyway.  Workgroups walk over rows, with the parameters, and in the backward pass
// the columns' sums of dy z and dy, in registers; those leave one partial row of sums per workgroup, added up by a second
// launch in a fixed order, so results do not depend on the order of execution.  Statistics and sums are binary32.
// Rows of less than 16 bytes belong to a lane each; rows of more than 16384 entries are read once per sum (kernels at the end).
//
// Measured (bytes read and written once, of a large copy's 5.1 TB/s): forward 8960 x 1024 half 7.7 us = 4.7 TB/s, 35840 x 1024
// float 6.3 TB/s; backward 8960 x 1500 bfloat16 26.9 us = 3.0 TB/s, of which 6.3 are the parameters' sums, 35840 x 1024 float
// 5.1 TB/s; one row of 1024 2 us (and the launch).
#include "../../include/amq.h"

#include <type_traits>

#include "amq_device.h"
#include "amq_train.h"
#include "amq_typed.h"



namespace amq {
namespace {

__device__ __forceinline__ float sum64(float v) { return group_sum(v, 6); }

// Sums of two values over the W waves that share a row.  One barrier, of all groups of W waves in the workgroup: the slots of
// consecutive calls alternate.
template <int W>
__device__ __forceinline__ void row_sum2(float& a, float& b, float (*slots)[2], int& turn) {
  a = sum64(a);
  b = sum64(b);
  if constexpr (W > 1) {
    const int waves = blockDim.x / 64, group = wave_id() / W * W;
    float(*s)[2] = slots + turn * waves;
    turn ^= 1;
    if (lane_id() == 0) {
      s[wave_id()][0] = a;
      s[wave_id()][1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      a += s[group + i][0];
      b += s[group + i][1];
    }
  }
}
template <int W>
__device__ __forceinline__ float row_sum(float a, float (*slots)[2], int& turn) {
  float b = 0.0f;
  row_sum2<W>(a, b, slots, turn);
  return a;
}

// Makes the compiler take the values as new ones.
template <typename T>
__device__ __forceinline__ void forget(Bytes16<T>& b) {
  uint4 v = __builtin_bit_cast(uint4, b);
  asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w));
  b = __builtin_bit_cast(Bytes16<T>, v);
}

// Piece j of a row's 16-byte pieces for thread `tid` of W waves.  The last one ends with the row and overlaps the one before
// it (its first `repeated` entries count there), so that no lane takes a path of its own; threads past the end hold it once more
// with nothing that counts, and store nothing.  (n >= V.)
template <int W, int V>
struct Piece {
  int start, repeated;
  __device__ __forceinline__ Piece(int j, int tid, int n) {
    const int c = (j * W * 64 + tid) * V;
    start = c < n - V ? c : n - V;
    repeated = c - start < V ? c - start : V;
  }
  __device__ __forceinline__ bool counts(int i) const { return i >= repeated; }
  __device__ __forceinline__ bool any() const { return repeated < V; }
};

// Rows that a wave has asked for beside the one at hand: 4 KB of each operand, so that a compute unit's 8 waves have 32 KB or
// more under way (8960 x 1500 bfloat16 backward with one row of 1 KB ahead 58 us, with four 40; and without lanes that take a
// path of their own at the row's end 28).
template <int NV>
constexpr int kAhead = NV >= 4 ? 1 : 4 / NV;

// W waves per row, NV times 16 bytes per lane; workgroups of max(W, 4) waves.
template <typename T, typename P, int W, int NV>
__global__ __launch_bounds__(W > 4 ? W * 64 : 256) void norm_kernel(NormArgs a) {
  constexpr int V = kPer16<T>, kRows = W >= 4 ? 1 : 4, kDeep = (kAhead<NV> + 1) / 2;
  __shared__ float slots[2 * W][2];
  int turn = 0;
  const int tid = W == 1 ? lane_id() : (int)threadIdx.x;
  auto piece = [&](int j) __attribute__((always_inline)) { return Piece<W, V>(j, tid, a.n); };
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    load_params<P, V>((const P*)a.weight, piece(j).start, V, 1.0f, w[j]);
    load_params<P, V>((const P*)a.bias, piece(j).start, V, 0.0f, b[j]);
  }
  const float inv_n = 1.0f / (float)a.n;
  Bytes16<T> ring[kDeep][NV];
  auto fetch = [&](Bytes16<T>(&r)[NV], int64_t row) __attribute__((always_inline)) {
    if (row >= a.rows) return;
    const T* px = (const T*)a.x + row * a.ld_x;
#pragma unroll
    for (int j = 0; j < NV; ++j) r[j] = fetch16(px + piece(j).start, V);
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + (W == 1 ? wave_id() : 0);
#pragma unroll
  for (int u = 0; u < kDeep; ++u) fetch(ring[u], row + u * step);
  while (row < a.rows) {
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      if (row >= a.rows) break;
      float x[NV][V], s = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          x[j][i] = (float)ring[u][j].v[i];
          s += piece(j).counts(i) ? x[j][i] : 0.0f;
        }
      fetch(ring[u], row + kDeep * step);
      const float mean = row_sum<W>(s, slots, turn) * inv_n;
      float q = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          x[j][i] -= mean;
          q = fmaf(piece(j).counts(i) ? x[j][i] : 0.0f, x[j][i], q);
        }
      const float rstd = 1.0f / sqrtf(row_sum<W>(q, slots, turn) * inv_n + a.eps);
      T* py = (T*)a.y + row * a.ld_y;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = fmaf(x[j][i] * rstd, w[j][i], b[j][i]);
        if (piece(j).any()) store16(py + piece(j).start, V, y);
      }
      if (tid == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
      }
      row += step;
    }
  }
}

// Rows that a workgroup of the backward pass has at a time: 16 waves where the registers allow it, which hide each other's sums and barriers
// (8960 x 1500 bfloat16 26.9 us, with 8 waves 28.0).
constexpr int grad_rows(int waves, int entries) {
  const int twice = entries <= 8 ? 2 : 1;
  return waves == 1 ? 8 * twice : waves == 4 ? 2 * twice : 1;
}
template <typename T, typename P, int W, int NV>
__global__ __launch_bounds__(grad_rows(W, NV * kPer16<T>) * W * 64) void norm_grad_kernel(NormGradArgs a) {
  constexpr int V = kPer16<T>, kRows = grad_rows(W, NV * V), kEntries = W * 64 * NV * V;
  __shared__ float slots[2 * kRows * W][2];
  __shared__ float shared_sums[kRows > 1 ? kRows * 2 * kEntries : 1];
  int turn = 0;
  const int group = wave_id() / W, tid = (int)threadIdx.x - group * W * 64;
  auto piece = [&](int j, int t) __attribute__((always_inline)) { return Piece<W, V>(j, t, a.n); };
  // 16 waves have 128 registers each: they read w again for every row, and ask for no row ahead
  constexpr bool kRoom = W < 16;
  constexpr int kDeep = kRoom ? kAhead<NV> : 1;
  float w[NV][V], dw[NV][V], db[NV][V];
  auto load_weights = [&] __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) load_params<P, V>((const P*)a.weight, piece(j, tid).start, V, 1.0f, w[j]);
  };
  if constexpr (kRoom) load_weights();
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) dw[j][i] = db[j][i] = 0.0f;
  const float inv_n = 1.0f / (float)a.n;
  // The entries stay in registers as they came (half the room in 16-bit types) and are widened in either pass.
  struct Row {
    Bytes16<T> x[NV], d[NV];
    float mean, rstd;
  };
  auto fetch = [&](Row& r, int64_t row) __attribute__((always_inline)) {
    if (row >= a.rows) return;
    const T *px = (const T*)a.x + row * a.ld_x, *pd = (const T*)a.dy + row * a.ld_dy;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      r.x[j] = fetch16(px + piece(j, tid).start, V);
      r.d[j] = fetch16(pd + piece(j, tid).start, V);
    }
    r.mean = a.mean[row];
    r.rstd = a.rstd[row];
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t first = (int64_t)blockIdx.x * kRows;  // of the workgroup's rows: its groups meet at barriers, so they leave together
  Row ring[kDeep];
#pragma unroll
  for (int u = 0; u < kDeep; ++u) fetch(ring[u], first + group + u * step);
  while (first < a.rows) {
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      if (first >= a.rows) break;
      const int64_t row = first + group;
      const bool here = row < a.rows;
      Row now = ring[u];
      if constexpr (kRoom) fetch(ring[u], row + kDeep * step);
      else load_weights();
      const float mean = now.mean, rstd = now.rstd;
      float s = 0.0f, q = 0.0f;
      if (here)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float z = ((float)now.x[j].v[i] - mean) * rstd, d = piece(j, tid).counts(i) ? (float)now.d[j].v[i] : 0.0f;
            dw[j][i] = fmaf(d, z, dw[j][i]);
            db[j][i] += d;
            const float g = d * w[j][i];
            s += g;
            q = fmaf(g, z, q);
          }
      row_sum2<W>(s, q, slots, turn);
      s *= inv_n;
      q *= inv_n;
      T* po = (T*)a.dx + row * a.ld_dx;
      if (here)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          // (without this the compiler keeps the widened values of the first pass in registers)
          forget(now.x[j]);
          forget(now.d[j]);
          float o[V];
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = rstd * (fmaf((float)now.d[j].v[i], w[j][i], -s) - ((float)now.x[j].v[i] - mean) * rstd * q);
          if (piece(j, tid).any()) store16(po + piece(j, tid).start, V, o);
        }
      if constexpr (!kRoom) fetch(ring[u], row + step);
      first += step;
    }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.n;
  if constexpr (kRows > 1) {
    // [group][sums of dy z, of dy][j][i][thread]: consecutive lanes on consecutive banks
    constexpr int kThreads = W * 64;
    float* mine = shared_sums + group * 2 * kEntries;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        mine[(j * V + i) * kThreads + tid] = dw[j][i];
        mine[kEntries + (j * V + i) * kThreads + tid] = db[j][i];
      }
    __syncthreads();
    for (int at = threadIdx.x; at < 2 * kEntries; at += kRows * kThreads) {
      const int of = at & (kEntries - 1), ji = of / kThreads, i = ji % V;
      float sum = 0.0f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) sum += shared_sums[r * 2 * kEntries + at];
      const Piece<W, V> p = piece(ji / V, of % kThreads);
      if (p.counts(i)) part[(at >= kEntries ? a.n : 0) + p.start + i] = sum;
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (piece(j, tid).counts(i)) {
          part[piece(j, tid).start + i] = dw[j][i];
          part[a.n + piece(j, tid).start + i] = db[j][i];
        }
  }
}

// Rows of less than 16 bytes, one per lane: 10^6 rows of 4 bfloat16 entries 8.7 us, backward 26.5 (of which 256 workgroups' loads, one row of each lane
// under way, are the most).
template <typename T, typename P>
__global__ __launch_bounds__(256) void norm_short_kernel(NormArgs a) {
  constexpr int V = kPer16<T>;
  float w[V], b[V];
  load_params<P, V>((const P*)a.weight, 0, a.n, 1.0f, w);
  load_params<P, V>((const P*)a.bias, 0, a.n, 0.0f, b);
  const float inv_n = 1.0f / (float)a.n;
  for (int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x; row < a.rows; row += (int64_t)gridDim.x * 256) {
    float x[V], s = 0.0f, q = 0.0f;
    load16((const T*)a.x + row * a.ld_x, a.n, x);  // zeros past the end
#pragma unroll
    for (int i = 0; i < V; ++i) s += x[i];
    const float mean = s * inv_n;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = i < a.n ? x[i] - mean : 0.0f;
      q = fmaf(x[i], x[i], q);
    }
    const float rstd = 1.0f / sqrtf(q * inv_n + a.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = fmaf(x[i] * rstd, w[i], b[i]);
    store16((T*)a.y + row * a.ld_y, a.n, x);
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}
template <typename T, typename P>
__global__ __launch_bounds__(256) void norm_grad_short_kernel(NormGradArgs a) {
  constexpr int V = kPer16<T>;
  __shared__ float sums[4][2 * V];
  float w[V], dw[V], db[V];
  load_params<P, V>((const P*)a.weight, 0, a.n, 1.0f, w);
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.0f;
  const float inv_n = 1.0f / (float)a.n;
  for (int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x; row < a.rows; row += (int64_t)gridDim.x * 256) {
    float z[V], d[V], s = 0.0f, q = 0.0f;
    load16((const T*)a.x + row * a.ld_x, a.n, z);
    load16((const T*)a.dy + row * a.ld_dy, a.n, d);  // zeros past the end: nothing of them counts
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      z[i] = i < a.n ? (z[i] - mean) * rstd : 0.0f;
      dw[i] = fmaf(d[i], z[i], dw[i]);
      db[i] += d[i];
      d[i] *= w[i];
      s += d[i];
      q = fmaf(d[i], z[i], q);
    }
    s *= inv_n;
    q *= inv_n;
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = rstd * (d[i] - s - z[i] * q);
    store16((T*)a.dx + row * a.ld_dx, a.n, d);
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float u = sum64(dw[i]), v = sum64(db[i]);
    if (lane_id() == 0) {
      sums[wave_id()][i] = u;
      sums[wave_id()][V + i] = v;
    }
  }
  __syncthreads();
  const int i = threadIdx.x % V;
  if (threadIdx.x < 2 * V && i < a.n)
    a.part[((int64_t)blockIdx.x * 2 + threadIdx.x / V) * a.n + i] =
        sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] + sums[3][threadIdx.x];
}

// Rows of any length, a workgroup for each, read once per sum and once for the output: 300 x 20011 float 21 us, backward 41; 2100 x 16385 bfloat16
// 75 and 118.
template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  __shared__ float slots[32][2];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* px = (const T*)a.x + row * a.ld_x;
    T* py = (T*)a.y + row * a.ld_y;
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
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <typename T, typename P>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs a) {
  __shared__ float slots[32][2];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
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

// Adds up the partial rows: 16 columns per workgroup, 64 groups of partial rows side by side.
template <typename P>
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(const float* part, int parts, int n, P* dweight, P* dbias) {
  __shared__ float sums[64][17];
  const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
  const int64_t c = (int64_t)blockIdx.x * 16 + lane, width = 2 * (int64_t)n;
  float s = 0.0f;
  if (c < width)
#pragma unroll 4
    for (int p = group; p < parts; p += 64) s += part[p * width + c];
  sums[group][lane] = s;
  __syncthreads();
  if (group < 4) {  // one wave: 16 groups each, then the four of them
    s = 0.0f;
#pragma unroll
    for (int g = 0; g < 16; ++g) s += sums[group * 16 + g][lane];
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if (group == 0 && c < width) {
      P* out = c < n ? dweight : dbias;
      if (out) out[c < n ? c : c - n] = (P)s;
    }
  }
}

// Waves per row and 16-byte pieces per lane.
struct Shape {
  int waves, pieces;  // waves 0: rows read once per sum; pieces 0 too: a row per lane
};
// 16 entries per lane at most: with 32 the backward pass needs more than 256 registers.  Few rows go to four waves each from 512 entries on, where the row's latency counts.
constexpr int kPerLane = 16;
Shape shape_of(int64_t rows, int n, int per16) {
  if (n < per16) return {0, 0};
  const int most = kPerLane / per16;
  for (int p = 1; p <= most; p *= 2)
    if (n <= 64 * p * per16 && (rows > 512 || n <= 512)) return {1, p};
  for (int p = 1; p <= most; p *= 2)
    if (n <= 256 * p * per16) return {4, p};
  if (n <= 512 * kPerLane) return {8, most};
  if (n <= 1024 * kPerLane) return {16, most};
  return {0, 1};
}

template <typename F>
hipError_t with_types(int type, int param_type, F f) {
  if (type == AMQ_F32) return f(float(), float());
  if (type == AMQ_BF16) return param_type == AMQ_F32 ? f(bf16(), float()) : f(bf16(), bf16());
  return param_type == AMQ_F32 ? f(f16(), float()) : f(f16(), f16());
}
template <typename T, typename F>
hipError_t with_shape(Shape h, F f) {
  constexpr int most = kPerLane / kPer16<T>;
#define AMQ_SHAPE(W, NV) \
  if (h.waves == W && h.pieces == NV) return f(std::integral_constant<int, W>(), std::integral_constant<int, NV>())
  AMQ_SHAPE(1, 1);
  AMQ_SHAPE(1, 2);
  if constexpr (most == 4) AMQ_SHAPE(1, 4);
  AMQ_SHAPE(4, 1);
  AMQ_SHAPE(4, 2);
  if constexpr (most == 4) AMQ_SHAPE(4, 4);
  AMQ_SHAPE(8, most);
  AMQ_SHAPE(16, most);
#undef AMQ_SHAPE
  return hipErrorInvalidValue;
}

// Rows that a grid of at most `most` workgroups takes at a time, spread evenly over its rounds.
int64_t even_blocks(int64_t tasks, int64_t most) {
  const int64_t rounds = (tasks + most - 1) / most;
  return (tasks + rounds - 1) / rounds;
}

constexpr int64_t kMostParts = 256;  // one workgroup per compute unit: more partial rows cost more than they hide
constexpr int64_t kMostLong = 2048;  // workgroups of the kernels for long rows: four rounds of the card

}  // namespace

int norm_grad_parts(int64_t rows, int n) {
  // (the widest and the narrowest types may take different forms; the larger number of either)
  int64_t parts = 1;
  for (int per16 : {4, 8}) {
    const Shape h = shape_of(rows, n, per16);
    const int at_a_time = h.waves ? grad_rows(h.waves, h.pieces * per16) : 256;
    const int64_t tasks = (rows + at_a_time - 1) / at_a_time;
    const int64_t p = h.waves || !h.pieces ? even_blocks(tasks, kMostParts) : (rows < 64 ? rows : 64);
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
      if (!h.pieces) norm_short_kernel<T, P><<<dim3((unsigned)even_blocks((a.rows + 255) / 256, 2048)), dim3(256), 0, s>>>(a);
      else norm_long_kernel<T, P><<<dim3((unsigned)even_blocks(a.rows, kMostLong)), dim3(1024), 0, s>>>(a);
      return hipGetLastError();
    }
    return with_shape<T>(h, [&](auto w, auto nv) {
      constexpr int W = decltype(w)::value;
      const int64_t tasks = W == 1 ? (a.rows + 3) / 4 : a.rows;
      norm_kernel<T, P, W, decltype(nv)::value>
          <<<dim3((unsigned)even_blocks(tasks, W >= 8 ? 512 : 2048)), dim3(W > 4 ? W * 64 : 256), 0, s>>>(a);
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
    if (!h.waves && !h.pieces) {
      parts = even_blocks((a.rows + 255) / 256, kMostParts);
      norm_grad_short_kernel<T, P><<<dim3((unsigned)parts), dim3(256), 0, s>>>(a);
      e = hipGetLastError();
    } else if (!h.waves) {
      // (the columns' sums first: dx may lie where dy or x does)
      if (sums) {
        parts = a.rows < 64 ? a.rows : 64;
        norm_grad_columns_kernel<T><<<dim3((unsigned)((a.n + 255) / 256), (unsigned)parts), dim3(256), 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
      norm_grad_long_kernel<T, P><<<dim3((unsigned)even_blocks(a.rows, kMostLong)), dim3(1024), 0, s>>>(a);
      e = hipGetLastError();
    } else {
      e = with_shape<T>(h, [&](auto w, auto nv) {
        constexpr int W = decltype(w)::value, NV = decltype(nv)::value, kRows = grad_rows(W, NV * kPer16<T>);
        parts = even_blocks((a.rows + kRows - 1) / kRows, kMostParts);
        norm_grad_kernel<T, P, W, NV><<<dim3((unsigned)parts), dim3(kRows * W * 64), 0, s>>>(a);
        return hipGetLastError();
      });
    }
    if (e != hipSuccess || !sums) return e;
    norm_grad_sum_kernel<P><<<dim3((unsigned)((2 * (int64_t)a.n + 15) / 16)), dim3(1024), 0, s>>>(a.part, (int)parts, a.n,
                                                                                                  (P*)a.dweight, (P*)a.dbias);
    return hipGetLastError();
  });
}

}  // namespace amq
