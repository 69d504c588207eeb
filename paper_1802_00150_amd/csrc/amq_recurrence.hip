// Linear recurrences over whole sequences, forward and backward: every channel has a state of its own,
//
//   blend   f = sigmoid(g), i = 1 - f:  h_t = f h_{t-1} + i x_t
//   decay   h_t = a_t h_{t-1} + x_t, the factor a given
//   back    e_t = dh_t + f_{t+1} e_{t+1} (from dh_last):  dx = i e,  dg = e (h_{t-1} - x) f i;  decay: dx = e, da = e h_{t-1}
//
// About 30 vector operations per entry forward and 50 backward (exponential and reciprocal count four each), against 6 and 10 bytes
// (16-bit types): bound by memory once enough is under way, by latency for few entries.  A step is an affine map of the
// state, so time is split: the kSpan steps of a wave are read at once, turned into one map (factor A, offset B) from a zero state, the waves
// of a workgroup exchange those through LDS, every wave folds the ones before it onto the state and replays its steps, which are still
// in registers, from the state they really start in.  So inputs are read once, and the results' error is that of steps one after the
// other but for the folds'.  A tile is up to 16 waves of 8 steps = 128 steps of 64 lanes of V channels.
//
// With channels enough for the card a workgroup walks over the tiles of its channels.  Otherwise every tile has a workgroup: it leaves its
// map in memory, looks back for the nearest tile whose end state is there, folds the maps between and leaves its own end state ("Tiles of
// one sequence" below).
//
// The backward pass takes h_{t-1} in full precision from the states that the forward pass leaves in front of every 128th
// step (4 / 128 bytes per entry instead of the 2 of reading rounded states): each tile replays the recurrence from there.
//
// States, products of factors and gradients along time are binary32.  1 - i is never rounded by itself: for g >= 0 the kept
// state is h - i h in one fused operation, so that units that hold for 10^5 steps do not drift (a rounded f is off by up to
// 2^-25 the same way in every step), and for g < 0 it is f h with f = sigmoid(g) to its last digits.
#include "../../include/amq.h"

#include <type_traits>

#include "amq_device.h"
#include "amq_train.h"
#include "amq_typed.h"

namespace amq {
namespace {

constexpr int kSpan = 8;                   // steps of a wave in a tile
constexpr int kTileWaves = 16;             // waves of a full tile
constexpr int kTile = kSpan * kTileWaves;  // its steps
static_assert(kTile == AMQ_STATE_STEPS, "a backward tile begins where a state was left");

// What a step does to the state: h -> keep(h) + add.
template <int MODE>
struct Step {
  float p, add;  // blend: f where g < 0, -i where g >= 0;  decay: the factor
  bool pos;      // g >= 0
  __device__ __forceinline__ void set(float g, float x) {
    if constexpr (MODE == AMQ_RECURRENCE_BLEND) {
      const float e = __expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.0f + e), small = e * r;  // sigmoid(|g|), sigmoid(-|g|)
      pos = g >= 0.0f;
      p = pos ? -small : small;
      add = (pos ? small : r) * x;
    } else {
      p = g;
      add = x;
    }
  }
  __device__ __forceinline__ void hold() {
    p = MODE == AMQ_RECURRENCE_BLEND ? 0.0f : 1.0f;
    add = 0.0f;
    pos = true;
  }
  __device__ __forceinline__ float keep(float h) const {
    return MODE == AMQ_RECURRENCE_BLEND ? fmaf(p, h, pos ? h : 0.0f) : p * h;
  }
  __device__ __forceinline__ float next(float h) const {
    return MODE == AMQ_RECURRENCE_BLEND ? fmaf(p, h, pos ? add + h : add) : fmaf(p, h, add);
  }
  __device__ __forceinline__ float dx(float e) const { return MODE == AMQ_RECURRENCE_BLEND ? (pos ? -p : 1.0f - p) * e : e; }
  __device__ __forceinline__ float dgate(float e, float h, float x) const {
    if constexpr (MODE == AMQ_RECURRENCE_BLEND) {
      const float small = fabsf(p);
      return e * (h - x) * fmaf(-small, small, small);
    }
    return e * h;
  }
};

// A workgroup's batch entry, the first of its channels, and the steps that count.
struct Place {
  int64_t b;
  int c;
  int64_t length;
};
template <int V, typename A>
__device__ __forceinline__ Place place_of(const A& a, int64_t group) {
  const int pieces = (a.n + 64 * V - 1) / (64 * V);
  Place p;
  p.b = group / pieces;
  p.c = (int)(group - p.b * pieces) * 64 * V;
  p.length = a.steps;
  if (a.lengths) {
    const int64_t l = a.lengths[p.b];
    p.length = l < 0 ? 0 : l < a.steps ? l : a.steps;
  }
  return p;
}
// The V channels of a lane behind `row` (the same address in all lanes).  n is a multiple of V; lanes past the end read the last ones.
template <int V>
struct Lane {
  uint32_t first;
  bool any;
  __device__ __forceinline__ Lane(int c, int n) {
    const uint32_t left = (uint32_t)(n - c), at = lane_id() * V;
    any = at < left;
    first = any ? at : left - V;
  }
  template <typename T>
  __device__ __forceinline__ Elements<T, V> get(const T* row) const {
    return *reinterpret_cast<const Elements<T, V>*>(reinterpret_cast<const char*>(row) + first * (uint32_t)sizeof(T));
  }
  template <typename T>
  __device__ __forceinline__ void put(T* row, const float (&v)[V]) const {
    Elements<T, V> e;
#pragma unroll
    for (int j = 0; j < V; ++j) e.v[j] = (T)v[j];
    *reinterpret_cast<Elements<T, V>*>(reinterpret_cast<char*>(row) + first * (uint32_t)sizeof(T)) = e;
  }
};

// ---- Tiles of one sequence in workgroups of their own.
//
// Tiles are taken in the order of a counter, those that others wait for first, so that a workgroup waits only for ones that have begun
// (and those for earlier ones): every wait ends, whatever part of the grid has room at a time.  A tile leaves {A, B} of every channel, raises its mark to 1,
// and once it knows the state that it starts in leaves the one it ends in and raises it to 2.  The one it starts in is that of the
// nearest earlier tile with mark 2 folded through the maps between: the same operations in the same order wherever that one is,
// so results do not depend on the order of execution.  Up to 64 tiles back are looked at.
// Values go past the caches of the chip's dies as relaxed atomics of device scope; a mark is written when its values have arrived.
struct Chain {
  uint32_t* marks;    // [tiles]
  uint64_t* maps;     // [tiles][64 V]
  uint32_t* ends;     // [tiles][64 V]
};
constexpr unsigned kPollLimit = 1u << 22;  // (seconds; a workgroup that gave up would leave NaN)

__device__ __forceinline__ void leave(uint32_t* p, uint32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void leave(uint64_t* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t look(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t look(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <int V>
__device__ __forceinline__ void leave_map(const Chain& c, int64_t tile, const float (&A)[V], const float (&B)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j)
    leave(c.maps + (tile * 64 + lane_id()) * V + j, (uint64_t)__float_as_uint(B[j]) << 32 | __float_as_uint(A[j]));
  arrived();
  if (lane_id() == 0) leave(c.marks + tile, 1u);
}
template <int V>
__device__ __forceinline__ void leave_end(const Chain& c, int64_t tile, const float (&h)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) leave(c.ends + (tile * 64 + lane_id()) * V + j, __float_as_uint(h[j]));
}
__device__ __forceinline__ void mark_end(const Chain& c, int64_t tile) {
  arrived();
  if (lane_id() == 0) leave(c.marks + tile, 2u);
}
// One wave: the state that tile > 0 starts in.
template <int V>
__device__ __forceinline__ void look_back(const Chain& c, int64_t tile, float (&h)[V]) {
  const int l = lane_id();
  int back = -1;  // the nearest tile whose end is known, and all between have left their maps
  for (unsigned polls = 0; polls < kPollLimit; ++polls) {
    const uint32_t mark = l < tile ? look(c.marks + tile - 1 - l) : 0u;
    const unsigned long long ends = __ballot(mark == 2u), none = __ballot(mark == 0u);
    if (ends) {
      const int at = __ffsll(ends) - 1;
      if ((none & ((1ull << at) - 1)) == 0) {
        back = at;
        break;
      }
    }
    __builtin_amdgcn_s_sleep(1);
  }
  back = __builtin_amdgcn_readfirstlane(back);
  if (back < 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = __builtin_nanf("");
    return;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) h[j] = __uint_as_float(look(c.ends + ((tile - 1 - back) * 64 + l) * V + j));
  constexpr int kAtOnce = 8;
  for (int64_t t = tile - back; t < tile; t += kAtOnce) {
    uint64_t m[kAtOnce][V];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) m[u][j] = look(c.maps + ((t + u < tile ? t + u : tile - 1) * 64 + l) * V + j);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (t + u < tile)
#pragma unroll
        for (int j = 0; j < V; ++j) h[j] = fmaf(__uint_as_float((uint32_t)m[u][j]), h[j], __uint_as_float((uint32_t)(m[u][j] >> 32)));
  }
}
// What a launch with workgroups of their own keeps in the workspace: the counter, then the marks (both cleared first), maps and ends.
struct SplitLayout {
  int64_t groups, tiles;
  size_t marks, maps, ends, bytes;
  SplitLayout(int64_t g, int64_t t, int channels) : groups(g), tiles(t) {
    marks = 256;
    maps = (marks + sizeof(uint32_t) * g * t + 255) & ~size_t(255);
    ends = maps + sizeof(uint64_t) * g * t * channels;
    bytes = (ends + sizeof(uint32_t) * g * t * channels + 255) & ~size_t(255);
  }
};
struct Split {
  uint32_t* counter;
  uint32_t* marks;
  uint64_t* maps;
  uint32_t* ends;
  int64_t tiles;
  uint32_t groups;
};
template <int V>
__device__ __forceinline__ Chain chain_of(const Split& s, int64_t group) {
  return {s.marks + group * s.tiles, s.maps + group * s.tiles * 64 * V, s.ends + group * s.tiles * 64 * V};
}
__global__ __launch_bounds__(256) void split_clear_kernel(uint32_t* p, int64_t words) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// ---- forward

// A wave's steps: asked for, and turned into what they do.
template <typename T, int V>
struct Asked {
  Elements<T, V> g[kSpan], x[kSpan];
};

template <typename T, int MODE, int V, bool SPLIT>
__global__ __launch_bounds__(64 * kTileWaves) void recurrence_kernel(RecurrenceArgs a, Split split) {
  __shared__ float maps[2][kTileWaves][2][64 * V];
  __shared__ float begin[64 * V];
  __shared__ uint32_t ticket;
  const int w = __builtin_amdgcn_readfirstlane(wave_id()), waves = blockDim.x / 64, lane = lane_id();
  int64_t group = blockIdx.x, tile = 0;
  if constexpr (SPLIT) {
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(split.counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const uint32_t t = __builtin_amdgcn_readfirstlane(ticket);
    tile = t / split.groups;
    group = t - (uint32_t)tile * split.groups;
  }
  const Place at = place_of<V>(a, group);
  const Lane<V> ch(at.c, a.n);
  const T* pg = (const T*)a.gate + at.b * a.gate_batch + at.c;
  const T* px = (const T*)a.x + at.b * a.x_batch + at.c;
  T* py = (T*)a.hs + at.b * a.hs_batch + at.c;
  const int64_t state = at.b * a.n + at.c;
  auto first_state = [&](float (&h)[V]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = 0.0f;
    if (a.h0) {
      const Elements<float, V> e = ch.get(a.h0 + state);
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = e.v[j];
    }
  };
  Asked<T, V> in;
  auto ask = [&](int64_t t0) __attribute__((always_inline)) {
    if (t0 + kSpan <= at.length) {
#pragma unroll
      for (int k = 0; k < kSpan; ++k) {
        in.g[k] = ch.get(pg + (t0 + k) * a.gate_step);
        in.x[k] = ch.get(px + (t0 + k) * a.x_step);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kSpan; ++k)
        if (t0 + k < at.length) {
          in.g[k] = ch.get(pg + (t0 + k) * a.gate_step);
          in.x[k] = ch.get(px + (t0 + k) * a.x_step);
        }
    }
  };
  Step<MODE> s[kSpan][V];
  auto turn_into_steps = [&](int64_t t0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) s[k][j].set((float)in.g[k].v[j], (float)in.x[k].v[j]);
    if (t0 + kSpan > at.length)
#pragma unroll
      for (int k = 0; k < kSpan; ++k)
        if (t0 + k >= at.length)
#pragma unroll
          for (int j = 0; j < V; ++j) s[k][j].hold();
  };
  // the wave's steps from the state in front of them
  auto replay = [&](int64_t t0, float (&h)[V]) __attribute__((always_inline)) {
    if (t0 >= a.steps) return;
    const bool whole = t0 + kSpan <= at.length;
    if (ch.any) {
#pragma unroll
      for (int k = 0; k < kSpan; ++k) {
#pragma unroll
        for (int j = 0; j < V; ++j) h[j] = s[k][j].next(h[j]);
        if (whole || t0 + k < a.steps) {
          float out[V];
#pragma unroll
          for (int j = 0; j < V; ++j) out[j] = whole || t0 + k < at.length ? h[j] : 0.0f;
          ch.put(py + (t0 + k) * a.hs_step, out);
        }
      }
      if (a.h_last && t0 + kSpan >= a.steps) ch.put(a.h_last + state, h);
      if (a.states && (t0 + kSpan) % kTile == 0 && t0 + kSpan < a.steps)
        ch.put(a.states + ((t0 + kSpan) / kTile - 1) * (int64_t)a.batch * a.n + state, h);
    }
  };

  if constexpr (SPLIT) {
    const int64_t t0 = tile * kTile + w * kSpan;
    ask(t0);
    turn_into_steps(t0);
    float A[V], B[V], h[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      A[j] = 1.0f;
      B[j] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        A[j] = s[k][j].keep(A[j]);
        B[j] = s[k][j].next(B[j]);
      }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      maps[0][w][0][lane * V + j] = A[j];
      maps[0][w][1][lane * V + j] = B[j];
    }
    lds_barrier();
    // the maps of the waves before it as one; wave 0 takes those of all
#pragma unroll
    for (int j = 0; j < V; ++j) {
      A[j] = 1.0f;
      B[j] = 0.0f;
    }
    const int before = w == 0 ? kTileWaves : w;
#pragma unroll 4
    for (int u = 0; u < before; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float fa = maps[0][u][0][lane * V + j];
        A[j] *= fa;
        B[j] = fmaf(fa, B[j], maps[0][u][1][lane * V + j]);
      }
    if (w == 0) {
      const Chain chain = chain_of<V>(split, group);
      if (tile == 0) {
        first_state(h);
      } else {
        leave_map(chain, tile, A, B);
        look_back(chain, tile, h);
      }
      float end[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        begin[lane * V + j] = h[j];
        end[j] = fmaf(A[j], h[j], B[j]);
      }
      leave_end(chain, tile, end);
      lds_barrier();
      mark_end(chain, tile);
    } else {
      lds_barrier();
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = fmaf(A[j], begin[lane * V + j], B[j]);
    }
    replay(t0, h);
    return;
  }

  float carry[V];  // (wave 0 alone has it, and reads h0: h_last, written behind a barrier, may lie there)
#pragma unroll
  for (int j = 0; j < V; ++j) carry[j] = 0.0f;
  if (w == 0) first_state(carry);
  int turn = 0;
  ask(w * kSpan);
  for (int64_t first = 0; first < a.steps; first += waves * kSpan, turn ^= 1) {
    const int64_t t0 = first + w * kSpan;
    turn_into_steps(t0);
    if (first + waves * kSpan < a.steps) ask(t0 + waves * kSpan);
    float h[V];
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = carry[j];
    if (waves > 1) {
      // the wave's map; wave 0 knows the state it starts in, and leaves the one that it ends in
      float A[V], B[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        A[j] = 1.0f;
        B[j] = carry[j];
      }
#pragma unroll
      for (int k = 0; k < kSpan; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          A[j] = s[k][j].keep(A[j]);
          B[j] = s[k][j].next(B[j]);
        }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        maps[turn][w][0][lane * V + j] = A[j];
        maps[turn][w][1][lane * V + j] = B[j];
      }
      lds_barrier();
      if (w > 0)
#pragma unroll
        for (int j = 0; j < V; ++j) h[j] = maps[turn][0][1][lane * V + j];
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = w == 0 ? B[j] : h[j];
      const int before = w == 0 ? waves : w;
#pragma unroll 4
      for (int u = 1; u < before; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = fmaf(maps[turn][u][0][lane * V + j], f[j], maps[turn][u][1][lane * V + j]);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (w == 0) carry[j] = f[j];
        else h[j] = f[j];
      }
    }
    replay(t0, h);
    if (waves == 1)
#pragma unroll
      for (int j = 0; j < V; ++j) carry[j] = h[j];
  }
}

// ---- backward

template <typename T, int MODE, int V, bool SPLIT>
__global__ __launch_bounds__(64 * kTileWaves) void recurrence_grad_kernel(RecurrenceGradArgs a, Split split) {
  __shared__ float maps[2][kTileWaves][3][64 * V];
  __shared__ float begin[64 * V];
  __shared__ uint32_t ticket;
  const int w = __builtin_amdgcn_readfirstlane(wave_id()), waves = blockDim.x / 64, lane = lane_id();
  const int64_t tiles = (a.steps + waves * kSpan - 1) / (waves * kSpan);  // (one tile, or tiles of kTile steps)
  int64_t group = blockIdx.x, tile = tiles - 1;
  if constexpr (SPLIT) {
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(split.counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const uint32_t t = __builtin_amdgcn_readfirstlane(ticket), order = t / split.groups;
    tile = tiles - 1 - order;
    group = t - order * split.groups;
  }
  const Place at = place_of<V>(a, group);
  const Lane<V> ch(at.c, a.n);
  const T* pg = (const T*)a.gate + at.b * a.gate_batch + at.c;
  const T* px = (const T*)a.x + at.b * a.x_batch + at.c;
  const T* pd = (const T*)a.dhs + at.b * a.dhs_batch + at.c;
  T* qg = (T*)a.dgate + at.b * a.dgate_batch + at.c;
  T* qx = (T*)a.dx + at.b * a.dx_batch + at.c;
  const int64_t state = at.b * a.n + at.c;
  auto last_gradient = [&](float (&r)[V]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = 0.0f;
    if (a.dh_last) {
      const Elements<float, V> e = ch.get(a.dh_last + state);
#pragma unroll
      for (int j = 0; j < V; ++j) r[j] = e.v[j];
    }
  };
  float back[V];  // the gradient that reaches a tile's last state from the steps behind it
  if constexpr (!SPLIT) last_gradient(back);
  int turn = 0;
  for (; tile >= 0; --tile, turn ^= 1) {
    const int64_t t0 = tile * waves * kSpan + w * kSpan;
    const bool whole = t0 + kSpan <= at.length;
    Elements<T, V> g[kSpan], x[kSpan], d[kSpan];
    float h[V], r[V];
    const float* from = tile == 0 ? a.h0 : a.states + (tile - 1) * (int64_t)a.batch * a.n;
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = 0.0f;
    auto ask = [&](int k) __attribute__((always_inline)) {
      g[k] = ch.get(pg + (t0 + k) * a.gate_step);
      x[k] = ch.get(px + (t0 + k) * a.x_step);
      d[k] = ch.get(pd + (t0 + k) * a.dhs_step);
    };
    if (whole) {
#pragma unroll
      for (int k = 0; k < kSpan; ++k) ask(k);
    } else {
#pragma unroll
      for (int k = 0; k < kSpan; ++k)
        if (t0 + k < at.length) ask(k);
    }
    if (from) {
      const Elements<float, V> e = ch.get(from + state);
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = e.v[j];
    }
    Step<MODE> s[kSpan][V];
#pragma unroll
    for (int k = 0; k < kSpan; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) s[k][j].set((float)g[k].v[j], (float)x[k].v[j]);
    if (!whole)
#pragma unroll
      for (int k = 0; k < kSpan; ++k)
        if (t0 + k >= at.length)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            s[k][j].hold();
            d[k].v[j] = (T)0.0f;
          }
    // the wave's maps: of the state along time, and of the gradient against it (the same factor)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float A = 1.0f, B = 0.0f, R = 0.0f;
#pragma unroll
      for (int k = 0; k < kSpan; ++k) {
        A = s[k][j].keep(A);
        B = s[k][j].next(B);
        R = s[kSpan - 1 - k][j].keep(R + (float)d[kSpan - 1 - k].v[j]);
      }
      maps[turn][w][0][lane * V + j] = A;
      maps[turn][w][1][lane * V + j] = B;
      maps[turn][w][2][lane * V + j] = R;
    }
    lds_barrier();
#pragma unroll 4
    for (int u = 0; u < w; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = fmaf(maps[turn][u][0][lane * V + j], h[j], maps[turn][u][1][lane * V + j]);
    if constexpr (SPLIT) {
      // the maps of the waves behind it as one; the last wave takes those of all
      float A[V], R[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        A[j] = 1.0f;
        R[j] = 0.0f;
      }
      const int until = w == kTileWaves - 1 ? 0 : w + 1;
#pragma unroll 4
      for (int u = kTileWaves - 1; u >= until; --u)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float fa = maps[turn][u][0][lane * V + j];
          A[j] *= fa;
          R[j] = fmaf(fa, R[j], maps[turn][u][2][lane * V + j]);
        }
      if (w == kTileWaves - 1) {
        const Chain chain = chain_of<V>(split, group);
        const int64_t order = tiles - 1 - tile;
        if (order == 0) {
          last_gradient(r);
        } else {
          leave_map(chain, order, A, R);
          look_back(chain, order, r);
        }
        float end[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          begin[lane * V + j] = r[j];
          end[j] = fmaf(A[j], r[j], R[j]);
        }
        leave_end(chain, order, end);
        lds_barrier();
        mark_end(chain, order);
      } else {
        lds_barrier();
#pragma unroll
        for (int j = 0; j < V; ++j) r[j] = fmaf(A[j], begin[lane * V + j], R[j]);
      }
    } else {
#pragma unroll 4
      for (int u = waves - 1; u > w; --u)
#pragma unroll
        for (int j = 0; j < V; ++j) back[j] = fmaf(maps[turn][u][0][lane * V + j], back[j], maps[turn][u][2][lane * V + j]);
#pragma unroll
      for (int j = 0; j < V; ++j) r[j] = back[j];
#pragma unroll 4
      for (int u = w; u >= 0; --u)
#pragma unroll
        for (int j = 0; j < V; ++j) back[j] = fmaf(maps[turn][u][0][lane * V + j], back[j], maps[turn][u][2][lane * V + j]);
    }
    if (t0 < a.steps && ch.any) {
      float before[kSpan][V];
#pragma unroll
      for (int k = 0; k < kSpan; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          before[k][j] = h[j];
          h[j] = s[k][j].next(h[j]);
        }
#pragma unroll
      for (int k = kSpan - 1; k >= 0; --k) {
        float og[V], ox[V];
        const bool here = whole || t0 + k < at.length;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float e = r[j] + (float)d[k].v[j];
          og[j] = here ? s[k][j].dgate(e, before[k][j], (float)x[k].v[j]) : 0.0f;
          ox[j] = here ? s[k][j].dx(e) : 0.0f;
          r[j] = s[k][j].keep(e);
        }
        if (whole || t0 + k < a.steps) {
          ch.put(qg + (t0 + k) * a.dgate_step, og);
          ch.put(qx + (t0 + k) * a.dx_step, ox);
        }
      }
      if (tile == 0 && w == 0 && a.dh0) ch.put(a.dh0 + state, r);
    }
    if constexpr (SPLIT) return;
  }
}

// ---- launches

template <typename F>
hipError_t with_type(int type, int mode, int n, F f) {
  auto modes = [&](auto t, auto v) {
    return mode == AMQ_RECURRENCE_BLEND ? f(t, v, std::integral_constant<int, AMQ_RECURRENCE_BLEND>())
                                        : f(t, v, std::integral_constant<int, AMQ_RECURRENCE_DECAY>());
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  if (type == AMQ_F32) return modes(float(), one);
  if (type == AMQ_BF16) return n % 2 == 0 ? modes(bf16(), two) : modes(bf16(), one);
  return n % 2 == 0 ? modes(f16(), two) : modes(f16(), one);
}

int waves_of(int64_t steps) {
  const int64_t w = (steps + kSpan - 1) / kSpan;
  return (int)(w < kTileWaves ? w : kTileWaves);
}
int64_t groups_of(int64_t batch, int64_t n, int V) { return batch * ((n + 64 * V - 1) / (64 * V)); }
// Workgroups of their own for tiles: where the channels alone leave compute units without one.
constexpr int64_t kMostSplit = 512;
bool splits(int64_t groups, int64_t steps) { return steps > kTile && groups <= kMostSplit; }

hipError_t split_of(int64_t groups, int64_t steps, int channels, void* ws, hipStream_t s, Split& out) {
  const int64_t tiles = (steps + kTile - 1) / kTile;
  const SplitLayout l(groups, tiles, channels);
  char* p = static_cast<char*>(ws);
  out = {reinterpret_cast<uint32_t*>(p), reinterpret_cast<uint32_t*>(p + l.marks), reinterpret_cast<uint64_t*>(p + l.maps),
         reinterpret_cast<uint32_t*>(p + l.ends), tiles, (uint32_t)groups};
  const int64_t words = (int64_t)(l.maps / sizeof(uint32_t));
  split_clear_kernel<<<dim3((unsigned)(words / 1024 < 256 ? words / 1024 + 1 : 256)), dim3(256), 0, s>>>(out.counter, words);
  return hipGetLastError();
}
template <typename A, typename F>
hipError_t launch(const A& a, hipStream_t s, F kernel) {
  return with_type(a.type, a.mode, a.n, [&](auto t, auto v, auto m) {
    constexpr int V = decltype(v)::value;
    const int64_t groups = groups_of(a.batch, a.n, V);
    const int waves = waves_of(a.steps);
    if (splits(groups, a.steps)) {
      Split split;
      const hipError_t e = split_of(groups, a.steps, 64 * V, a.ws, s, split);
      if (e != hipSuccess) return e;
      kernel(t, v, m, std::true_type())<<<dim3((unsigned)(groups * split.tiles)), dim3(64 * waves), 0, s>>>(a, split);
    } else {
      kernel(t, v, m, std::false_type())<<<dim3((unsigned)groups), dim3(64 * waves), 0, s>>>(a, Split());
    }
    return hipGetLastError();
  });
}
// (batch entries may count as channels of one entry in the launch, so the larger need of either)
size_t workspace(int64_t steps, int64_t batch, int64_t n) {
  size_t most = 0;
  for (int V : {1, 2})
    for (int flat = 0; flat < 2; ++flat) {
      const int64_t groups = flat ? groups_of(1, batch * n, V) : groups_of(batch, n, V);
      if (!splits(groups, steps)) continue;
      const size_t need = SplitLayout(groups, (steps + kTile - 1) / kTile, 64 * V).bytes;
      most = need > most ? need : most;
    }
  return most;
}

}  // namespace

size_t recurrence_workspace(int64_t steps, int64_t batch, int64_t n, int) { return workspace(steps, batch, n); }
size_t recurrence_grad_workspace(int64_t steps, int64_t batch, int64_t n, int) { return workspace(steps, batch, n); }

hipError_t launch_recurrence(const RecurrenceArgs& a, hipStream_t s) {
  return launch(a, s, [](auto t, auto v, auto m, auto split) {
    return recurrence_kernel<decltype(t), decltype(m)::value, decltype(v)::value, decltype(split)::value>;
  });
}

hipError_t launch_recurrence_grad(const RecurrenceGradArgs& a, hipStream_t s) {
  return launch(a, s, [](auto t, auto v, auto m, auto split) {
    return recurrence_grad_kernel<decltype(t), decltype(m)::value, decltype(v)::value, decltype(split)::value>;
  });
}

}  // namespace amq
