// The 2-norm over all entries of many tensors, and the same tensors scaled to a largest norm.
//
//   norm = sqrt(sum of g^2 over all tensors),  out = c g,  c = max / norm where norm is finite and more than max, else 1
//
// Two operations per entry each way: bound by memory, every entry read twice (no entry can be scaled before the last is read) and
// written once; by latency for few.  The tensors' addresses travel in the kernels' arguments, so nothing has to be copied to the
// card and a captured launch keeps its own; every 120 tensors take a launch of each kernel.  A tensor is cut into pieces that
// workgroups take in turn; each leaves one partial sum, and every workgroup of the second kernel adds all of them up again in one
// order (4 KB from L2), which saves a launch and makes the norm the same from run to run.  The second kernel goes through the pieces from the
// last one on, which the card's memory-side cache still holds, and writes past the caches, which leaves that cache to what is still to be read
// (94 million floats 220 us, with such stores 197, from the last one on 190; in 1024 workgroups instead of 512 190 and 185; 47 million
// bfloat16 entries 58 and 51).
//
// Sums are binary64: squares of binary32 gradients neither overflow nor vanish there.
#include "../../include/amq.h"

#include "amq_device.h"
#include "amq_train.h"
#include "amq_typed.h"

namespace amq {
namespace {

constexpr int kTensors = 120;    // of a launch: its arguments stay below 4 KB
constexpr int kThreads = 512;
constexpr int kMostBlocks = 512;  // of a launch: two workgroups of 8 waves per compute unit

struct Table {
  const void* p[kTensors];
  void* out[kTensors];
  int64_t n[kTensors];
  uint32_t first[kTensors];  // piece that a tensor begins with; unused entries: all ones
  uint8_t type[kTensors];
};
struct ClipArgs {
  Table t;
  uint32_t pieces, vectors;  // in all; 16-byte vectors of a thread in a piece
  double* partial;           // of this launch's workgroups
};
struct ScaleArgs {
  Table t;
  uint32_t pieces, vectors;
  const double* partial;  // of all launches
  double max_norm;
  float* norm;  // null: another launch writes it
  int partials;
};

// The tensor that a piece belongs to: the last one that begins at it or before.
__device__ __forceinline__ int tensor_of(const Table& t, uint32_t piece) {
  const int l = lane_id();
  const uint32_t a = t.first[l], b = l + 64 < kTensors ? t.first[l + 64] : ~0u;
  const int n = __popcll(__ballot(a <= piece)) + __popcll(__ballot(b <= piece));
  return __builtin_amdgcn_readfirstlane(n - 1);
}

template <typename T>
__device__ __forceinline__ double squares(const Bytes16<T>& b) {
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kPer16<T>; ++i) {
    const double v = (double)(float)b.v[i];
    s = fma(v, v, s);
  }
  return s;
}
// Calls f(vector, its first entry, valid entries there) for the vectors of a piece that a thread has; four are under way at a time where the
// piece is whole and has as many.
template <typename T, typename F>
__device__ __forceinline__ void vectors_of(const T* p, int64_t n, int64_t piece, uint32_t vectors, F f) {
  constexpr int V = kPer16<T>;
  const int64_t begin = piece * vectors * kThreads * V;
  if (vectors % 4 == 0 && begin + (int64_t)vectors * kThreads * V <= n) {
    const T* q = p + begin;  // (the same in all lanes)
    for (uint32_t v = 0; v < vectors; v += 4, q += 4 * kThreads * V) {
      Bytes16<T> b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) b[u] = *reinterpret_cast<const Bytes16<T>*>(q + u * kThreads * V + threadIdx.x * (uint32_t)V);
#pragma unroll
      for (int u = 0; u < 4; ++u) f(b[u], begin + ((int64_t)(v + u) * kThreads + threadIdx.x) * V, V);
    }
    return;
  }
  int64_t at = begin + (int64_t)threadIdx.x * V;
  for (uint32_t v = 0; v < vectors && at < n; ++v, at += kThreads * V) {
    const int valid = n - at < V ? (int)(n - at) : V;
    f(fetch16(p + at, valid), at, valid);
  }
}

template <typename T>
__device__ __forceinline__ double piece_squares(const Table& t, int i, int64_t piece, uint32_t vectors) {
  double s = 0.0;
  vectors_of((const T*)t.p[i], t.n[i], piece, vectors, [&](const Bytes16<T>& b, int64_t, int) { s += squares<T>(b); });
  return s;
}

__global__ __launch_bounds__(kThreads) void norm_of_tensors_kernel(ClipArgs a) {
  __shared__ double scratch[kThreads / 64];
  double s = 0.0;
  for (uint32_t piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
    const int i = tensor_of(a.t, piece);
    const int64_t of = piece - a.t.first[i];
    const int type = a.t.type[i];
    s += type == AMQ_F32    ? piece_squares<float>(a.t, i, of, a.vectors)
         : type == AMQ_BF16 ? piece_squares<bf16>(a.t, i, of, a.vectors)
                            : piece_squares<f16>(a.t, i, of, a.vectors);
  }
  s = block_sum<kThreads / 64>(s, scratch);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = s;
}

template <typename T>
__device__ __forceinline__ void scale_piece(const Table& t, int i, int64_t piece, uint32_t vectors, float c, double exact, bool small) {
  constexpr int V = kPer16<T>;
  T* q = (T*)t.out[i];
  vectors_of((const T*)t.p[i], t.n[i], piece, vectors, [&](const Bytes16<T>& b, int64_t at, int valid) {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = small ? (float)((double)(float)b.v[j] * exact) : (float)b.v[j] * c;
    if (valid == V) store_streaming<T, V>(q + at, v);
    else store16(q + at, valid, v);
  });
}

__global__ __launch_bounds__(kThreads) void scale_tensors_kernel(ScaleArgs a) {
  __shared__ double scratch[kThreads / 64];
  double s = 0.0;
  for (int i = threadIdx.x; i < a.partials; i += kThreads) s += a.partial[i];
  s = sqrt(block_sum<kThreads / 64>(s, scratch));
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)s;
  const bool finite = s < __builtin_inf();  // (false for NaN)
  const double exact = finite && s > a.max_norm ? a.max_norm / s : 1.0;
  // a factor that binary32 holds to fewer digits takes binary64 products
  const bool small = exact < 0x1p-100;
  const float c = (float)exact;
  for (uint32_t turn = blockIdx.x; turn < a.pieces; turn += gridDim.x) {
    const uint32_t piece = a.pieces - 1 - turn;
    const int i = tensor_of(a.t, piece);
    if (c == 1.0f && a.t.p[i] == a.t.out[i]) continue;
    const int64_t of = piece - a.t.first[i];
    const int type = a.t.type[i];
    if (type == AMQ_F32) scale_piece<float>(a.t, i, of, a.vectors, c, exact, small);
    else if (type == AMQ_BF16) scale_piece<bf16>(a.t, i, of, a.vectors, c, exact, small);
    else scale_piece<f16>(a.t, i, of, a.vectors, c, exact, small);
  }
}

// A launch's tensors: fills the table from `at` on, skipping empty ones, and returns the index behind them.
int64_t fill(const ClipTensors& c, int64_t at, Table& t, uint32_t& pieces, uint32_t& vectors) {
  int used = 0;
  int64_t bytes = 0;
  for (; at < c.count && used < kTensors; ++at)
    if (c.sizes[at] > 0) {
      t.p[used] = c.tensors[at];
      t.out[used] = c.out ? c.out[at] : nullptr;
      t.n[used] = c.sizes[at];
      t.type[used] = (uint8_t)c.types[at];
      bytes += c.sizes[at] * (c.types[at] == AMQ_F32 ? 4 : 2);
      ++used;
    }
  // pieces of 8 KB while they do not fill the card, of up to 64 KB (or more where their number would pass 32 bits)
  vectors = 1;
  while ((vectors < 8 && bytes / (16 * kThreads * vectors) > 2 * kMostBlocks) || bytes / (16 * kThreads * (int64_t)vectors) > (1 << 30)) vectors *= 2;
  int64_t total = 0;
  for (int i = 0; i < kTensors; ++i) {
    if (i < used) {
      const int64_t per = (int64_t)vectors * kThreads * (t.type[i] == AMQ_F32 ? 4 : 8);
      t.first[i] = (uint32_t)total;
      total += (t.n[i] + per - 1) / per;
    } else {
      t.p[i] = t.out[i] = nullptr;
      t.n[i] = 0;
      t.type[i] = 0;
      t.first[i] = ~0u;
    }
  }
  pieces = (uint32_t)total;
  return at;
}
int blocks_of(uint32_t pieces) { return (int)(pieces < kMostBlocks ? pieces : kMostBlocks); }

}  // namespace

size_t clip_workspace(int64_t count) {
  const int64_t launches = (count + kTensors - 1) / kTensors;
  return (size_t)(launches > 0 ? launches : 1) * kMostBlocks * sizeof(double);
}

hipError_t launch_clip_gradients(const ClipTensors& c, double max_norm, float* norm, void* ws, hipStream_t s) {
  double* partial = static_cast<double*>(ws);
  int partials = 0;
  ClipArgs sum;
  for (int64_t at = 0; at < c.count;) {
    at = fill(c, at, sum.t, sum.pieces, sum.vectors);
    if (!sum.pieces) continue;
    sum.partial = partial + partials;
    norm_of_tensors_kernel<<<dim3((unsigned)blocks_of(sum.pieces)), dim3(kThreads), 0, s>>>(sum);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    partials += blocks_of(sum.pieces);
  }
  ScaleArgs scale;
  scale.partial = partial;
  scale.partials = partials;
  scale.max_norm = max_norm;
  scale.norm = norm;
  int64_t at = 0;
  do {
    at = fill(c, at, scale.t, scale.pieces, scale.vectors);
    if (!c.out) scale.pieces = 0, at = c.count;
    if (!scale.pieces && !scale.norm) continue;
    scale_tensors_kernel<<<dim3((unsigned)(scale.pieces ? blocks_of(scale.pieces) : 1)), dim3(kThreads), 0, s>>>(scale);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    scale.norm = nullptr;
  } while (at < c.count);
  return hipSuccess;
}

}  // namespace amq
