// Linear recurrences over whole sequences, forward and backward: every channel has a state of its own,
//
//   blend   f = sigmoid(g), i = 1 - f:  h_t = f h_{t-1} + i x_t
//   decay   h_t = a_t h_{t-1} + x_t, the factor a given
//   back    e_t = dh_t + f_{t+1} e_{t+1} (from dh_last):  dx = i e,  dg = e (h_{t-1} - x) f i;  decay: dx = e, da = e h_{t-1}
//
// About 12 operations per entry forward and 30 backward, against 6 and 10 bytes (16-bit types): bound by memory once enough
// is under way, by latency for few entries.  A step is an affine map of the state, so time is split: the kSpan steps of a
// wave are read at once, turned into one map (factor A, offset B) from a zero state, the waves of a workgroup exchange those
// through LDS, every wave folds the ones before it onto the state and replays its steps, which are still in registers, from
// the state they really start in.  So inputs are read once, and the results' error is that of steps one after the other but for
// the folds'.  A workgroup's tile is up to 16 waves of 8 steps = 128 steps of 64 lanes of V channels; it walks over its tiles.
//
// The backward pass takes h_{t-1} in full precision from the states that the forward pass leaves in front of every 128th
// step (4 / 128 bytes per entry instead of the 2 of reading rounded states): each tile replays the recurrence from there.
//
// States, products of factors and gradients along time are binary32.  1 - i is never rounded by itself: for g >= 0 the kept
// state is fma(-i, h, h), one rounding of the exact (1 - i) h, so that units that hold for 10^5 steps do not drift (a rounded f
// is off by up to 2^-25 the same way in every step), and for g < 0 it is f h with f = sigmoid(g) to its last digits.
#include "../../include/amq.h"

#include <type_traits>

#include "amq_device.h"
#include "amq_train.h"
#include "amq_typed.h"

namespace amq {
namespace {

constexpr int kSpan = 8;                      // steps of a wave in a tile
constexpr int kTileWaves = 16;                // waves of a full tile
constexpr int kTile = kSpan * kTileWaves;     // its steps
static_assert(kTile == AMQ_STATE_STEPS, "a backward tile begins where a state was left");

template <typename T>
constexpr int kWidth = 4 / (int)sizeof(T);  // channels of a lane: 4 bytes, 256 of a row per wave

// What a step does to the state: h -> keep(h) + add.
template <int MODE>
struct Step;
template <>
struct Step<AMQ_RECURRENCE_BLEND> {
  float i, p;  // p: f where g < 0, -i (sign bit set, -0 included) where g >= 0
  __device__ __forceinline__ void set(float g) {
    const float e = __expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.0f + e), small = e * r;  // sigmoid(|g|), sigmoid(-|g|)
    i = g >= 0.0f ? small : r;
    p = g >= 0.0f ? -small : small;
  }
  __device__ __forceinline__ void hold() { i = 0.0f, p = -0.0f; }
  __device__ __forceinline__ float keep(float h) const {
    return fmaf(p, h, __int_as_float((__float_as_int(p) >> 31) & __float_as_int(h)));
  }
  __device__ __forceinline__ float next(float h, float x) const { return fmaf(i, x, keep(h)); }
  __device__ __forceinline__ float dx(float e) const { return i * e; }
  __device__ __forceinline__ float dgate(float e, float h, float x) const {
    const float small = fabsf(p);
    return e * (h - x) * (small * (1.0f - small));
  }
};
template <>
struct Step<AMQ_RECURRENCE_DECAY> {
  float p;
  __device__ __forceinline__ void set(float a) { p = a; }
  __device__ __forceinline__ void hold() { p = 1.0f; }
  __device__ __forceinline__ float keep(float h) const { return p * h; }
  __device__ __forceinline__ float next(float h, float x) const { return fmaf(p, h, x); }
  __device__ __forceinline__ float dx(float e) const { return e; }
  __device__ __forceinline__ float dgate(float e, float h, float) const { return e * h; }
};

// A lane's V channels.  The last ones of a row end with it and overlap the lane before: the first `repeated` are that lane's, and
// stored by it alone (a state may be replaced in place, so that the second copy may be worked out from the wrong one).
template <int V>
struct Channels {
  int start, repeated;
  __device__ __forceinline__ Channels(int c, int n) {
    start = c < n - V ? c : n - V;
    repeated = c - start < V ? c - start : V;
  }
  __device__ __forceinline__ bool any() const { return repeated < V; }
  template <typename T>
  __device__ __forceinline__ void put(T* p, const float (&v)[V]) const {
    if (repeated == 0) {
      store<T, V>(p, V, v);
    } else {
#pragma unroll
      for (int j = 1; j < V; ++j)
        if (j >= repeated) p[j] = (T)v[j];
    }
  }
};

struct Place {  // of a workgroup: its batch entry and first channel, and the steps that count
  int64_t b;
  int c;
  int64_t length;
};
template <int V, typename A>
__device__ __forceinline__ Place place_of(const A& a) {
  const int pieces = (a.n + 64 * V - 1) / (64 * V);
  Place p;
  p.b = blockIdx.x / pieces;
  p.c = (int)(blockIdx.x - p.b * pieces) * 64 * V;
  p.length = a.steps;
  if (a.lengths) {
    const int64_t l = a.lengths[p.b];
    p.length = l < 0 ? 0 : l < a.steps ? l : a.steps;
  }
  return p;
}

template <typename T, int MODE, int V>
__global__ __launch_bounds__(64 * kTileWaves) void recurrence_kernel(RecurrenceArgs a) {
  __shared__ float maps[2][kTileWaves][2][64 * V];
  const int w = wave_id(), waves = blockDim.x / 64, lane = lane_id();
  const Place at = place_of<V>(a);
  const Channels<V> ch(at.c + lane * V, a.n);
  const T* pg = (const T*)a.gate + at.b * a.gate_batch + ch.start;
  const T* px = (const T*)a.x + at.b * a.x_batch + ch.start;
  T* py = (T*)a.hs + at.b * a.hs_batch + ch.start;
  const int64_t state = at.b * a.n + ch.start;
  float carry[V];
#pragma unroll
  for (int j = 0; j < V; ++j) carry[j] = 0.0f;
  if (w == 0 && a.h0) {  // (wave 0 alone: h_last, written behind a barrier, may lie there)
    const Elements<float, V> h = fetch<float, V>(a.h0 + state, V);
#pragma unroll
    for (int j = 0; j < V; ++j) carry[j] = h.v[j];
  }
  Elements<T, V> g[kSpan], x[kSpan];
  auto ask = [&](int64_t t0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
      if (t0 + k < at.length) {
        g[k] = fetch<T, V>(pg + (t0 + k) * a.gate_step, V);
        x[k] = fetch<T, V>(px + (t0 + k) * a.x_step, V);
      }
  };
  int turn = 0;
  ask(w * kSpan);
  for (int64_t first = 0; first < a.steps; first += waves * kSpan, turn ^= 1) {
    const int64_t t0 = first + w * kSpan;
    Step<MODE> s[kSpan][V];
    float v[kSpan][V];
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (t0 + k < at.length) {
          s[k][j].set((float)g[k].v[j]);
          v[k][j] = (float)x[k].v[j];
        } else {
          s[k][j].hold();
          v[k][j] = 0.0f;
        }
      }
    ask(t0 + waves * kSpan);
    float start[V];
    if (waves > 1) {
      // the wave's map; wave 0 knows the state it starts in, and leaves the one that it ends in
      float A[V], B[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        A[j] = w == 0 ? 0.0f : 1.0f;
        B[j] = carry[j];
      }
#pragma unroll
      for (int k = 0; k < kSpan; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          A[j] = s[k][j].keep(A[j]);
          B[j] = s[k][j].next(B[j], v[k][j]);
        }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        maps[turn][w][0][lane * V + j] = A[j];
        maps[turn][w][1][lane * V + j] = B[j];
        start[j] = carry[j];
      }
      lds_barrier();
      float h[V];
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = 0.0f;
      for (int u = 0; u < waves; ++u) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (u == w && w > 0) start[j] = h[j];
          const float fa = maps[turn][u][0][lane * V + j], fb = maps[turn][u][1][lane * V + j];
          h[j] = u == 0 ? fb : fmaf(fa, h[j], fb);
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) carry[j] = w == 0 ? h[j] : 0.0f;
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) start[j] = carry[j];
    }
#pragma unroll
    for (int k = 0; k < kSpan; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) start[j] = s[k][j].next(start[j], v[k][j]);
      const int64_t t = t0 + k;
      if (t < a.steps && ch.any()) {
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = t < at.length ? start[j] : 0.0f;
        ch.put(py + t * a.hs_step, out);
        if (a.h_last && t == a.steps - 1) ch.put(a.h_last + state, start);
        else if (a.states && (t + 1) % kTile == 0) ch.put(a.states + ((t + 1) / kTile - 1) * (int64_t)a.batch * a.n + state, start);
      }
    }
    if (waves == 1)
#pragma unroll
      for (int j = 0; j < V; ++j) carry[j] = start[j];
  }
}

template <typename T, int MODE, int V>
__global__ __launch_bounds__(64 * kTileWaves) void recurrence_grad_kernel(RecurrenceGradArgs a) {
  __shared__ float maps[2][kTileWaves][3][64 * V];
  const int w = wave_id(), waves = blockDim.x / 64, lane = lane_id();
  const Place at = place_of<V>(a);
  const Channels<V> ch(at.c + lane * V, a.n);
  const T* pg = (const T*)a.gate + at.b * a.gate_batch + ch.start;
  const T* px = (const T*)a.x + at.b * a.x_batch + ch.start;
  const T* pd = (const T*)a.dhs + at.b * a.dhs_batch + ch.start;
  T* qg = (T*)a.dgate + at.b * a.dgate_batch + ch.start;
  T* qx = (T*)a.dx + at.b * a.dx_batch + ch.start;
  const int64_t state = at.b * a.n + ch.start;
  float back[V];  // the gradient that reaches a tile's last state from the steps behind it
#pragma unroll
  for (int j = 0; j < V; ++j) back[j] = 0.0f;
  if (a.dh_last) {
    const Elements<float, V> h = fetch<float, V>(a.dh_last + state, V);
#pragma unroll
    for (int j = 0; j < V; ++j) back[j] = h.v[j];
  }
  const int64_t tiles = (a.steps + waves * kSpan - 1) / (waves * kSpan);  // (one tile, or tiles of kTile steps)
  int turn = 0;
  for (int64_t tile = tiles - 1; tile >= 0; --tile, turn ^= 1) {
    const int64_t t0 = tile * waves * kSpan + w * kSpan;
    Elements<T, V> g[kSpan], x[kSpan], d[kSpan];
    Elements<float, V> h0;
    const float* from = tile == 0 ? a.h0 : a.states + (tile - 1) * (int64_t)a.batch * a.n;
#pragma unroll
    for (int j = 0; j < V; ++j) h0.v[j] = 0.0f;
    if (from) h0 = fetch<float, V>(from + state, V);
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
      if (t0 + k < at.length) {
        g[k] = fetch<T, V>(pg + (t0 + k) * a.gate_step, V);
        x[k] = fetch<T, V>(px + (t0 + k) * a.x_step, V);
        d[k] = fetch<T, V>(pd + (t0 + k) * a.dhs_step, V);
      }
    Step<MODE> s[kSpan][V];
    float v[kSpan][V], dh[kSpan][V];
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (t0 + k < at.length) {
          s[k][j].set((float)g[k].v[j]);
          v[k][j] = (float)x[k].v[j];
          dh[k][j] = (float)d[k].v[j];
        } else {
          s[k][j].hold();
          v[k][j] = dh[k][j] = 0.0f;
        }
      }
    // the wave's maps: of the state along time, and of the gradient against it (the same factor)
    float h[V], r[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float A = 1.0f, B = 0.0f, R = 0.0f;
#pragma unroll
      for (int k = 0; k < kSpan; ++k) {
        A = s[k][j].keep(A);
        B = s[k][j].next(B, v[k][j]);
        R = s[kSpan - 1 - k][j].keep(R + dh[kSpan - 1 - k][j]);
      }
      maps[turn][w][0][lane * V + j] = A;
      maps[turn][w][1][lane * V + j] = B;
      maps[turn][w][2][lane * V + j] = R;
      h[j] = h0.v[j];
      r[j] = back[j];
    }
    lds_barrier();
    for (int u = 0; u < w; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = fmaf(maps[turn][u][0][lane * V + j], h[j], maps[turn][u][1][lane * V + j]);
    for (int u = waves - 1; u >= 0; --u)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (u == w) r[j] = back[j];
        back[j] = fmaf(maps[turn][u][0][lane * V + j], back[j], maps[turn][u][2][lane * V + j]);
      }
    float before[kSpan][V];
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        before[k][j] = h[j];
        h[j] = s[k][j].next(h[j], v[k][j]);
      }
#pragma unroll
    for (int k = kSpan - 1; k >= 0; --k) {
      float og[V], ox[V];
      const bool here = t0 + k < at.length;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float e = r[j] + dh[k][j];
        og[j] = here ? s[k][j].dgate(e, before[k][j], v[k][j]) : 0.0f;
        ox[j] = here ? s[k][j].dx(e) : 0.0f;
        r[j] = s[k][j].keep(e);
      }
      if (t0 + k < a.steps && ch.any()) {
        ch.put(qg + (t0 + k) * a.dgate_step, og);
        ch.put(qx + (t0 + k) * a.dx_step, ox);
      }
    }
    if (tile == 0 && w == 0 && a.dh0 && ch.any()) ch.put(a.dh0 + state, r);
  }
}

template <typename F>
hipError_t with_type(int type, int mode, int n, F f) {
  auto modes = [&](auto t, auto v) {
    return mode == AMQ_RECURRENCE_BLEND ? f(t, v, std::integral_constant<int, AMQ_RECURRENCE_BLEND>())
                                        : f(t, v, std::integral_constant<int, AMQ_RECURRENCE_DECAY>());
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  if (type == AMQ_F32) return modes(float(), one);
  if (type == AMQ_BF16) return n >= 2 ? modes(bf16(), two) : modes(bf16(), one);
  return n >= 2 ? modes(f16(), two) : modes(f16(), one);
}

int waves_of(int64_t steps) {
  const int64_t w = (steps + kSpan - 1) / kSpan;
  return (int)(w < kTileWaves ? w : kTileWaves);
}
template <int V>
dim3 grid_of(int64_t batch, int n) { return dim3((unsigned)(batch * ((n + 64 * V - 1) / (64 * V)))); }

}  // namespace

size_t recurrence_workspace(int64_t, int64_t, int64_t, int) { return 0; }
size_t recurrence_grad_workspace(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t launch_recurrence(const RecurrenceArgs& a, hipStream_t s) {
  return with_type(a.type, a.mode, a.n, [&](auto t, auto v, auto m) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value;
    recurrence_kernel<T, decltype(m)::value, V><<<grid_of<V>(a.batch, a.n), dim3(64 * waves_of(a.steps)), 0, s>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_recurrence_grad(const RecurrenceGradArgs& a, hipStream_t s) {
  return with_type(a.type, a.mode, a.n, [&](auto t, auto v, auto m) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value;
    recurrence_grad_kernel<T, decltype(m)::value, V><<<grid_of<V>(a.batch, a.n), dim3(64 * waves_of(a.steps)), 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace amq
