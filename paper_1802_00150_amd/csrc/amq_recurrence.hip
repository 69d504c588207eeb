// Linear recurrences over whole sequences, forward and backward: every channel has a state of its own,
//
//   blend   f = sigmoid(g), i = 1 - f:  h_t = f h_{t-1} + i x_t
//   decay   h_t = a_t h_{t-1} + x_t, the factor a given
//   back    e_t = dh_t + f_{t+1} e_{t+1} (from dh_last):  dx = i e,  dg = e (h_{t-1} - x) f i;  decay: dx = e, da = e h_{t-1}
//
// 28 vector instructions per entry forward and 46 backward, against 6 and 10 bytes (16-bit types): bound by memory once enough is under way
// (backward with 16-bit types by instructions as much), by latency for few entries.  A step is an affine map of the
// state, so time is split: the 8 steps of a wave are read at once, turned into one map (factor A, offset B) from a zero state, the waves
// of a workgroup exchange those through LDS, every wave folds the ones before it onto the state and replays its steps, which are still
// in registers, from the state they really start in.  So inputs are read once, and the results' error is that of steps one after the
// other but for the folds'.  A tile is up to 16 waves of 8 steps = 128 steps of 64 channels (128 where a lane has two).
//
// With channels enough for the card a workgroup walks over the tiles of its channels.  Otherwise every tile (of 256 steps forward) has a
// workgroup: it leaves its map in memory, looks back for the nearest tile whose end state is there, folds the maps between and leaves its
// own end state ("Tiles of one sequence" below): a single-pass scan with decoupled look-back, as Merrill and Garland published it in 2016.
//
// Measured (steps x channels; a large copy 5.1 TB/s): 2000 x 16384 float 78 us, 5.05 TB/s; 1000 x 32768 bfloat16 39.5 to 41.5 us, 4.9; 35 x 262144
// backward 20.2, 4.7; 1000 x 16384 backward 40, 4.1; with the chain 32768 x 1024 bfloat16 54, 3.7; 16384 x 1024 float 47, 4.3; 4001 x 2100 float
// 28, 3.6, backward 50, 3.4; 2000 x 8192 float backward 71, 4.6.  (The second figure is TB/s.)
//
// The backward pass takes h_{t-1} in full precision from the states that the forward pass leaves in front of every 128th
// step (4 / 128 bytes per entry instead of the 2 of reading rounded states): each tile replays the recurrence from there.
//
// States, products of factors and gradients along time are binary32; sigmoids are within (2 |g| + 8) 2^-24 of their value.  For g >= 0 a
// step is h + i x - i h, a rounding of the sum and one of the fused rest, and a map keeps A - i A: 1 - i is not rounded by itself, which would be
// off by up to 2^-25 the same way in every step of a gate that stays.  (Roundings of states that move by little are alike too: over 20000 steps
// of gates near 10 the error is half of that of a rounded f with maps of 16 steps, about 0.7 with 8.)  For g < 0 the step is f h + i x.
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
constexpr int kLongSpan = 16, kLongTile = kLongSpan * kTileWaves;  // of tiles with workgroups of their own, forward
static_assert(kLongTile % AMQ_STATE_STEPS == 0 && AMQ_STATE_STEPS % kLongSpan == 0, "states are left behind a wave's steps");
static_assert(kTile == AMQ_STATE_STEPS, "a backward tile begins where a state was left");

__device__ __forceinline__ bool is_finite(float v) { return fabsf(v) < __builtin_inff(); }  // (false for NaN)

// What a step does to the state.  BACK: in the backward pass, which needs i and x apart.
template <int MODE, bool BACK>
struct Step {
  float p;  // blend: f where g < 0, -i where g >= 0 (its sign bit says which: a mask per step would not fit the scalar registers);  decay: the factor
  float v;  // i x;  BACK: x
  float i;  // (BACK)
  __device__ __forceinline__ void set(float g, float x) {
    if constexpr (MODE == AMQ_RECURRENCE_BLEND) {
      const float e = __expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.0f + e), small = e * r;  // sigmoid(|g|), sigmoid(-|g|)
      const bool pos = g >= 0.0f;
      p = pos ? -small : small;
      i = pos ? small : r;
      v = BACK ? x : i * x;
    } else {
      p = g;
      i = 1.0f;
      v = x;
    }
  }
  __device__ __forceinline__ void hold() {
    p = 1.0f;  // (times the state, which may be infinite)
    i = v = 0.0f;
  }
  __device__ __forceinline__ float held(float h) const { return __float_as_int(p) < 0 ? h : 0.0f; }
  __device__ __forceinline__ float keep(float h) const { return MODE == AMQ_RECURRENCE_BLEND ? fmaf(p, h, held(h)) : p * h; }
  __device__ __forceinline__ float next(float h) const {
    if constexpr (MODE == AMQ_RECURRENCE_BLEND) return fmaf(p, h, BACK ? fmaf(i, v, held(h)) : v + held(h));
    return fmaf(p, h, v);
  }
  // next() and keep() where they leave the finite numbers: f h by itself, since h - i h of an infinite state is NaN and h + i x may pass the
  // range that f h + i x is in.
  __device__ __forceinline__ float next_exact(float h) const {
    const float n = next(h);
    return MODE == AMQ_RECURRENCE_BLEND && !is_finite(n) && __float_as_int(p) < 0 ? fmaf(1.0f + p, h, BACK ? i * v : v) : n;
  }
  __device__ __forceinline__ float keep_exact(float h) const {
    const float n = keep(h);
    return MODE == AMQ_RECURRENCE_BLEND && !is_finite(n) && __float_as_int(p) < 0 ? (1.0f + p) * h : n;
  }
  __device__ __forceinline__ float dx(float e) const { return MODE == AMQ_RECURRENCE_BLEND ? i * e : e; }
  __device__ __forceinline__ float dgate(float e, float h) const {
    if constexpr (MODE == AMQ_RECURRENCE_BLEND) {
      const float small = fabsf(p);
      return e * (h - v) * fmaf(-small, small, small);
    }
    return e * h;
  }
  // (a comparison made again takes one operation, one kept from the maps to the results two scalar registers)
  __device__ __forceinline__ void again() {
    if constexpr (MODE == AMQ_RECURRENCE_BLEND) asm volatile("" : "+v"(p));
  }
};

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
  // The same in the block it is called in, so that the compiler sees 32 bits beside a scalar address there.
  __device__ __forceinline__ Lane here() const {
    Lane l = *this;
    asm volatile("" : "+v"(l.first));
    return l;
  }
  template <typename T>
  __device__ __forceinline__ Elements<T, V> get(const T* row) const {
    return *reinterpret_cast<const Elements<T, V>*>(reinterpret_cast<const char*>(row) + first * (uint32_t)sizeof(T));
  }
  template <typename T>
  __device__ __forceinline__ void put(T* row, const float (&v)[V]) const {
    store_whole<T, V>(reinterpret_cast<T*>(reinterpret_cast<char*>(row) + first * (uint32_t)sizeof(T)), v);
  }
  // those of them that are `wanted`
  template <typename T>
  __device__ __forceinline__ void put(T* row, const float (&v)[V], const bool (&wanted)[V]) const {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (any && wanted[j]) row[first + j] = (T)v[j];
  }
};

// ---- Tiles of one sequence in workgroups of their own.
//
// Tiles are taken in the order of counters, those that others wait for first, so that a workgroup waits only
// for ones that have begun (and those for earlier ones): every wait ends, whatever part of the grid has room at a time.  A tile leaves
// {A, B} of every channel, raises its mark to 1, and once it knows the state that it starts in leaves the one it ends in and raises it
// to 2.  The one it starts in is that of the nearest earlier tile with mark 2 folded through the maps between: the same operations in
// the same order wherever that one is, so results do not depend on the order of execution.  Up to 64 tiles back are looked at.
// Values go past the caches of the chip's dies as relaxed atomics of device scope; a mark is written when its values have arrived.
struct Chain {
  uint32_t* marks;  // [tiles]
  uint64_t* maps;   // [tiles][64]
  uint32_t* ends;   // [tiles][64]
};
constexpr unsigned kPollLimit = 1u << 22;  // (seconds; a workgroup that gave up would leave NaN)

__device__ __forceinline__ void leave(uint32_t* p, uint32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void leave(uint64_t* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t look(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t look(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ void leave_map(const Chain& c, int64_t tile, float A, float B) {
  leave(c.maps + tile * 64 + lane_id(), (uint64_t)__float_as_uint(B) << 32 | __float_as_uint(A));
  arrived();
  if (lane_id() == 0) leave(c.marks + tile, 1u);
}
__device__ __forceinline__ void leave_end(const Chain& c, int64_t tile, float h) {
  leave(c.ends + tile * 64 + lane_id(), __float_as_uint(h));
}
// (mark 2; what it was where the end is not known after all)
__device__ __forceinline__ void mark_end(const Chain& c, int64_t tile, bool known) {
  arrived();
  const uint32_t mark = known ? 2u : tile > 0 ? 1u : 0u;
  if (lane_id() == 0) leave(c.marks + tile, mark);
}
// The state that tile > 0 starts in, for one wave: it polls the marks, all waves of the workgroup bring the maps between to LDS, and it
// folds them.  (One wave that read up to 63 maps by itself was most of the time of a long sequence.)
constexpr int kWindow = 64;
__device__ __forceinline__ void look_back(const Chain& c, int64_t tile, uint64_t (*stage)[64], int& found, int w, bool mine, float& h) {
  const int l = lane_id();
  if (mine) {
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
    if (l == 0) found = back;
  }
  lds_barrier();  // (and what the stage held has been read)
  const int back = __builtin_amdgcn_readfirstlane(found);
  if (mine) h = back < 0 ? __builtin_nanf("") : __uint_as_float(look(c.ends + (tile - 1 - (back < 0 ? 0 : back)) * 64 + l));
#pragma unroll
  for (int i = 0; i < kWindow / kTileWaves; ++i) {
    const int u = w + i * kTileWaves;
    if (u < back) stage[u][l] = look(c.maps + (tile - back + u) * 64 + l);
  }
  lds_barrier();
  if (mine)
#pragma unroll 8
    for (int u = 0; u < back; ++u) {
      const uint64_t m = stage[u][l];
      h = fmaf(__uint_as_float((uint32_t)m), h, __uint_as_float((uint32_t)(m >> 32)));
    }
}
// One wave: the state behind a tile, once it is there.
__device__ __forceinline__ float end_of(const Chain& c, int64_t tile) {
  bool there = false;
  for (unsigned polls = 0; polls < kPollLimit && !there; ++polls) {
    there = __ballot(look(c.marks + tile) == 2u) != 0;
    if (!there) __builtin_amdgcn_s_sleep(8);
  }
  float h = there ? __uint_as_float(look(c.ends + tile * 64 + lane_id())) : __builtin_nanf("");
  asm volatile("" : "+v"(h));  // (waited for here, not where branches with and without it meet)
  return h;
}
// What a launch with workgroups of their own keeps in the workspace: the counters, then the marks (both cleared first), maps and ends.
constexpr uint32_t kCounters = 4, kCounterWords = 32;  // a cache line each
struct SplitLayout {
  int64_t groups, tiles;
  size_t marks, maps, ends, bytes;
  SplitLayout(int64_t g, int64_t t) : groups(g), tiles(t) {
    constexpr int channels = 64;
    marks = sizeof(uint32_t) * kCounters * kCounterWords;
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
  uint32_t groups, kinds;
};
__device__ __forceinline__ Chain chain_of(const Split& s, int64_t group) {
  return {s.marks + group * s.tiles, s.maps + group * s.tiles * 64, s.ends + group * s.tiles * 64};
}
// A tile that nobody has begun, by its order in the chain of its group, the same in all threads; false if there is none.  Every
// `kinds`th group shares a counter: four of them (with one for all 1000 x 8192 bfloat16 takes 1.23 times as long, 4001 x 2100 float 1.10
// times, backward 1000 x 4096 bfloat16 1.25 times; with eight, whose groups each keep to one die, 32768 x 1024 1.10 times), but one where a row of
// tiles fills the card (3000 x 16500 with four 1.07 times).
__device__ __forceinline__ bool take_tile(const Split& s, uint32_t& shared, uint32_t& order, uint32_t& group) {
  const uint32_t kinds = s.kinds, kind = blockIdx.x % kinds;
  if (threadIdx.x == 0) shared = __hip_atomic_fetch_add(s.counter + kind * kCounterWords, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const uint32_t now = __builtin_amdgcn_readfirstlane(shared), of_kind = (s.groups - kind + kinds - 1) / kinds;
  order = now / of_kind;
  group = (now - order * of_kind) * kinds + kind;
  return order < (uint32_t)s.tiles;
}
__global__ __launch_bounds__(256) void split_clear_kernel(uint32_t* p, int64_t words) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// ---- forward

// k < left, decided by itself (the compiler would join the steps of a tile that ends early, and index what is in registers).
__device__ __forceinline__ bool within(int k, int left) {
  asm volatile("" : "+s"(left));
  return k < left;
}

// Ends a branch: the compiler would take the same last operations out of both branches, and wait there for what has just been asked for.
__device__ __forceinline__ void branch_end() { asm volatile(""); }

// Where a group of 64 V channels lies, and the steps of its batch entry that count.
template <int V, typename A>
struct Group {
  int64_t b, state;   // batch entry; of the group's first channel in [B][n]
  int steps, length;  // all; the entry's
  uint32_t c;         // first channel
  Lane<V> ch;
  __device__ __forceinline__ Group(const A& a, uint32_t group) : ch(0, V) {
    const uint32_t pieces = ((uint32_t)a.n + 64 * V - 1) / (64 * V), entry = group / pieces;
    b = entry;
    c = (group - entry * pieces) * 64 * V;
    state = b * a.n + c;
    ch = Lane<V>((int)c, a.n);
    length = steps = (int)a.steps;
    if (a.lengths) {
      const int64_t l = a.lengths[b];
      length = l < 0 ? 0 : l < steps ? (int)l : steps;
    }
  }
  template <typename T>
  __device__ __forceinline__ T* row(T* p, int64_t t, int64_t step, int64_t entry) const { return p + t * step + b * entry + c; }
};

template <typename T, int V, int K = kSpan>
struct Inputs {
  Elements<T, V> g[K], x[K];
  // asks for the steps from t0 on
  template <typename A>
  __device__ __forceinline__ void ask(const A& a, const Group<V, A>& at, int t0) {
    const int left = at.length - t0;
    const T *pg = at.row((const T*)a.gate, t0, a.gate_step, a.gate_batch), *px = at.row((const T*)a.x, t0, a.x_step, a.x_batch);
    if (K >= kSpan && left >= K) {
      const Lane<V> ch = at.ch.here();
#pragma unroll
      for (int k = 0; k < K; ++k, pg += a.gate_step, px += a.x_step) {
        g[k] = ch.get(pg);
        x[k] = ch.get(px);
      }
      branch_end();
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k, pg += a.gate_step, px += a.x_step)
        if (within(k, left)) {
          g[k] = at.ch.get(pg);
          x[k] = at.ch.get(px);
        }
    }
  }
};
template <typename T, int MODE, int V, bool BACK, int K = kSpan>
struct Steps {
  Step<MODE, BACK> s[K][V];
  // `left`: of the entry's steps
  __device__ __forceinline__ void set(const Inputs<T, V, K>& in, int left) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) s[k][j].set((float)in.g[k].v[j], (float)in.x[k].v[j]);
    if (left < K)
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (!within(k, left))
#pragma unroll
          for (int j = 0; j < V; ++j) s[k][j].hold();
  }
  __device__ __forceinline__ void again() {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) s[k][j].again();
  }
  // The map of all: A the product of what is kept, B continued from what it holds.
  __device__ __forceinline__ void map(float (&A)[V], float (&B)[V]) const {
#pragma unroll
    for (int j = 0; j < V; ++j) A[j] = 1.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        A[j] = s[k][j].keep(A[j]);
        B[j] = s[k][j].next(B[j]);
      }
  }
  // From the state in front of them to the one behind, with everything that is written on the way.
  __device__ __forceinline__ void replay(const RecurrenceArgs& a, const Group<V, RecurrenceArgs>& at, int t0, float (&h)[V]) {
    if (t0 >= at.steps || !at.ch.any) return;
    again();
    const int left = at.length - t0, end = t0 + K;
    T* py = at.row((T*)a.hs, t0, a.hs_step, a.hs_batch);
    if (left >= K) {
      const Lane<V> ch = at.ch.here();
#pragma unroll
      for (int k = 0; k < K; ++k, py += a.hs_step) {
#pragma unroll
        for (int j = 0; j < V; ++j) h[j] = s[k][j].next(h[j]);
        ch.put(py, h);
      }
      branch_end();
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k, py += a.hs_step) {
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          h[j] = s[k][j].next(h[j]);
          out[j] = within(k, left) ? h[j] : 0.0f;
        }
        if (t0 + k < at.steps) at.ch.put(py, out);
      }
    }
    if (a.h_last && end >= at.steps) at.ch.put(a.h_last + at.state, h);
    if (a.states && end % AMQ_STATE_STEPS == 0 && end < at.steps)
      at.ch.put(a.states + (end / AMQ_STATE_STEPS - 1) * (int64_t)a.batch * a.n + at.state, h);
  }
};
// Rows behind the end of a batch entry: zeros, every `by`-th from t on.
template <typename T, int V, typename A>
__device__ __forceinline__ void clear_rows(const A& a, const Group<V, A>& at, T* p, int64_t t, int64_t end, int by, int64_t step, int64_t entry) {
  float zero[V];
#pragma unroll
  for (int j = 0; j < V; ++j) zero[j] = 0.0f;
  if (at.ch.any)
    for (T* row = at.row(p, t, step, entry); t < end; t += by, row += by * step) at.ch.put(row, zero);
}
template <int V, typename A>
__device__ __forceinline__ void given(const float* p, const Group<V, A>& at, float (&h)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) h[j] = 0.0f;
  if (p) {
    const Elements<float, V> e = at.ch.get(p + at.state);
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = e.v[j];
  }
}

// ---- Steps one after the other, where a map or a fold has left the finite numbers.
//
// An infinite state, and a product of factors or an offset that passes binary32 although the states do not (factors above 1 of a state that is 0),
// make inf - inf or 0 inf in a map or a fold.  What comes of that is infinite or NaN and stays so up to the end of the wave's steps and,
// through the folds, of the tile and the sequence.  So a look at the end of a wave's replay is enough: a channel that is not finite there is
// formed again from the state that the wave began in, or where that is not finite from the one in front of the tile, in order, with its inputs
// read again (few steps at a time: this lies beside what the kernels keep in registers); no other channel and nothing finite changes.  A NaN in
// front of the tile is one behind it either way.
constexpr int kMend = 4;
// A kernel's first argument, AGAIN: read once more, so that what is rare keeps nothing in scalar registers for itself.  (Inside a loop, which needs the
// argument afterwards, that takes more of them.)
template <bool AGAIN, typename A>
__device__ __forceinline__ A argument(const A& a) {
  if constexpr (AGAIN) {
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const A*)p;
  }
  return a;
}

// Whether some lane's value is not finite, which is rare.
template <int V>
__device__ __forceinline__ bool leaves(const float (&h)[V]) {
  bool all = true;
#pragma unroll
  for (int j = 0; j < V; ++j) all = all && is_finite(h[j]);
  return __builtin_expect(__ballot(!all) != 0, 0);
}
// Which channels are to be formed again, by their state in front and behind; whether a lane of the wave has any.
template <int V>
__device__ __forceinline__ bool spoiled(const float (&begin)[V], const float (&end)[V], bool (&which)[V]) {
  bool any = false;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    which[j] = !is_finite(end[j]) && begin[j] == begin[j];
    any = any || which[j];
  }
  return __ballot(any) != 0;
}
// h from in front of step t to in front of `end`, or to behind the entry's steps (`end` some steps of kMend on).
template <typename T, int MODE, int V, bool BACK, typename A>
__device__ __forceinline__ void advance(const A& a, const Group<V, A>& at, int t, int end, float (&h)[V]) {
  for (t = __builtin_amdgcn_readfirstlane(t); t < end && t < at.length; t = __builtin_amdgcn_readfirstlane(t + kMend)) {
    Inputs<T, V, kMend> in;
    in.ask(a, at, t);
    Steps<T, MODE, V, BACK, kMend> steps;
    steps.set(in, at.length - t);
#pragma unroll
    for (int k = 0; k < kMend; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = steps.s[k][j].next_exact(h[j]);
  }
}
// Takes `start` where it is finite.
template <int V>
__device__ __forceinline__ void finite_or(const float (&start)[V], float (&h)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) h[j] = is_finite(start[j]) ? start[j] : h[j];
}
// A wave's steps from t0 to `end` again, from `start`, or from the state h in front of step t.
template <typename T, int MODE, int V>
__device__ __forceinline__ void replay_again(const RecurrenceArgs& a, const Group<V, RecurrenceArgs>& at, int t, int t0, int end, const float (&start)[V],
                                             float (&h)[V], const bool (&which)[V]) {
  advance<T, MODE, V, false>(a, at, t, t0, h);
  finite_or<V>(start, h);
  for (t = __builtin_amdgcn_readfirstlane(t0); t < end; t = __builtin_amdgcn_readfirstlane(t + kMend)) {
    Inputs<T, V, kMend> in;
    in.ask(a, at, t);
    Steps<T, MODE, V, false, kMend> steps;
    steps.set(in, at.length - t);
#pragma unroll
    for (int k = 0; k < kMend; ++k) {
      const int behind = t + k + 1;
      float out[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[j] = steps.s[k][j].next_exact(h[j]);
        out[j] = within(k, at.length - t) ? h[j] : 0.0f;
      }
      if (!within(k, at.steps - t)) break;
      at.ch.put(at.row((T*)a.hs, t + k, a.hs_step, a.hs_batch), out, which);
      if (a.h_last && behind == at.steps) at.ch.put(a.h_last + at.state, h, which);
      if (a.states && behind % AMQ_STATE_STEPS == 0 && behind < at.steps)
        at.ch.put(a.states + (behind / AMQ_STATE_STEPS - 1) * (int64_t)a.batch * a.n + at.state, h, which);
    }
  }
}

// A workgroup per group of channels, tile after tile; ONE: there is one.
template <typename T, int MODE, int V, bool ONE>
__global__ __launch_bounds__(64 * kTileWaves, ONE ? 8 : 4) void recurrence_kernel(RecurrenceArgs a) {
  __shared__ float maps[ONE ? 1 : 2][kTileWaves][2][64 * V];
  const int w = __builtin_amdgcn_readfirstlane(wave_id()), waves = blockDim.x / 64, lane = lane_id();
  const Group<V, RecurrenceArgs> at(a, blockIdx.x);
  Inputs<T, V> in;
  Steps<T, MODE, V, false> steps;
  float carry[V];  // (wave 0 alone has it, and reads h0: h_last, written behind a barrier, may lie there)
#pragma unroll
  for (int j = 0; j < V; ++j) carry[j] = 0.0f;
  if (w == 0) given<V>(a.h0, at, carry);
  int turn = 0;
  in.ask(a, at, w * kSpan);
  int first = 0;
  for (; first < at.length; first += waves * kSpan, turn ^= 1) {
    const int t0 = first + w * kSpan;
    steps.set(in, at.length - t0);
    if constexpr (!ONE) in.ask(a, at, t0 + waves * kSpan);
    float h[V];
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = carry[j];
    if (waves > 1) {
      // the wave's map; wave 0 knows the state it starts in, and leaves the one that it ends in
      float A[V], B[V];
#pragma unroll
      for (int j = 0; j < V; ++j) B[j] = carry[j];
      steps.map(A, B);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        maps[turn][w][0][lane * V + j] = w == 0 ? carry[j] : A[j];  // (nobody folds wave 0's factor)
        maps[turn][w][1][lane * V + j] = B[j];
      }
      lds_barrier();
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = w == 0 ? B[j] : maps[turn][0][1][lane * V + j];
      const int before = w > 0 ? w : ONE ? 0 : waves;
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
    float start[V];
#pragma unroll
    for (int j = 0; j < V; ++j) start[j] = h[j];
    steps.replay(a, at, t0, h);
    if (leaves(h) || (!ONE && w == 0 && leaves(carry))) {
      float begin[V], next[V];
      bool which[V];
#pragma unroll
      for (int j = 0; j < V; ++j) begin[j] = next[j] = waves > 1 ? maps[turn][0][0][lane * V + j] : carry[j];
      const RecurrenceArgs b = argument<ONE>(a);
      const Group<V, RecurrenceArgs> here = ONE ? Group<V, RecurrenceArgs>(b, blockIdx.x) : at;
      if (spoiled(begin, h, which)) replay_again<T, MODE, V>(b, here, first, t0, t0 + kSpan, start, begin, which);
      if (!ONE && w == 0 && spoiled(next, carry, which)) {
        advance<T, MODE, V, false>(b, here, first, first + waves * kSpan, next);
#pragma unroll
        for (int j = 0; j < V; ++j) carry[j] = which[j] ? next[j] : carry[j];
      }
    }
    if constexpr (ONE) return;
  }
  if (first >= at.steps) return;
  clear_rows(a, at, (T*)a.hs, first + w, a.steps, waves, a.hs_step, a.hs_batch);
  if (w == 0 && a.h_last && at.ch.any) at.ch.put(a.h_last + at.state, carry);
}

// A workgroup per tile, of 16 steps of 16 waves of one channel a lane: a longer tile waits less for others than a wider one
// (8 steps of two channels and 12 of one take 1.07 times as long at 32768 x 1024 bfloat16, 1.02 and 0.98 times at 16384 x 1024 float), and needs no even
// number of channels.
template <typename T, int MODE>
__global__ __launch_bounds__(64 * kTileWaves, 8) void recurrence_tiles_kernel(RecurrenceArgs a, Split split) {
  constexpr int V = 1, K = kLongSpan;
  __shared__ uint64_t stage[kWindow][64];
  __shared__ float begin[64];
  __shared__ uint32_t number;
  __shared__ int found;
  auto maps = reinterpret_cast<float(*)[2][64]>(stage);  // [kTileWaves]
  const int w = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id();
  uint32_t tile, group;
  if (!take_tile(split, number, tile, group)) return;
  const Group<V, RecurrenceArgs> at(a, group);
  const int t0 = (int)tile * kLongTile + w * K;
  const Chain chain = chain_of(split, group);
  if ((int)tile * kLongTile >= at.length) {  // behind the entry's end
    clear_rows(a, at, (T*)a.hs, t0, t0 + K < at.steps ? t0 + K : at.steps, 1, a.hs_step, a.hs_batch);
    if (w == 0 && a.h_last && tile == split.tiles - 1) {
      float h[V];
      if (at.length == 0) given<V>(a.h0, at, h);
      else h[0] = end_of(chain, (at.length - 1) / kLongTile);
      if (at.ch.any) at.ch.put(a.h_last + at.state, h);
    }
    return;
  }
  Steps<T, MODE, V, false, K> steps;
  {
    Inputs<T, V, K> in;
    in.ask(a, at, t0);
    steps.set(in, at.length - t0);
  }
  float A[V], B[V] = {0.0f}, h[V];
  steps.map(A, B);
  maps[w][0][lane] = A[0];
  maps[w][1][lane] = B[0];
  lds_barrier();
  // the maps of the waves before it as one; wave 0 takes those of all
  float fa = 1.0f, fb = 0.0f;
  const int before = w == 0 ? kTileWaves : w;
#pragma unroll 4
  for (int u = 0; u < before; ++u) {
    const float one = maps[u][0][lane];
    fa *= one;
    fb = fmaf(one, fb, maps[u][1][lane]);
  }
  if (tile > 0) {
    if (w == 0) leave_map(chain, tile, fa, fb);
    look_back(chain, tile, stage, found, w, w == 0, h[0]);
  } else if (w == 0) {
    given<V>(a.h0, at, h);
  }
  bool late = false;  // wave 0: the end is not known
  if (w == 0) {
    begin[lane] = h[0];
    const float end[V] = {fmaf(fa, h[0], fb)};
    leave_end(chain, tile, end[0]);
    late = leaves(end);  // (also where h does)
    lds_barrier();
    mark_end(chain, tile, !late);
  } else {
    lds_barrier();
    h[0] = begin[lane];
  }
  if (leaves(h)) {  // (the same in all waves) the maps between may have made that: the state that the tile before ends in, by itself
    if (w == 0) maps[0][0][lane] = tile > 0 ? end_of(chain, tile - 1) : h[0];
    lds_barrier();
    begin[lane] = h[0] = maps[0][0][lane];
  }
  if (w > 0) h[0] = fmaf(fa, h[0], fb);
  const float start[V] = {h[0]};
  steps.replay(a, at, t0, h);
  bool which[V];
  if (late) {
    const float from[V] = {begin[lane]};
    float end[V] = {fmaf(fa, from[0], fb)};
    if (spoiled(from, end, which)) {
      float again[V] = {from[0]};
      const RecurrenceArgs b = argument<true>(a);
      advance<T, MODE, V, false>(b, Group<V, RecurrenceArgs>(b, group), t0, t0 + kLongTile, again);
      end[0] = which[0] ? again[0] : end[0];
    }
    leave_end(chain, tile, end[0]);
    mark_end(chain, tile, true);
  }
  if (leaves(h)) {
    float from[V] = {begin[lane]};
    const RecurrenceArgs b = argument<true>(a);
    if (spoiled(from, h, which)) replay_again<T, MODE, V>(b, Group<V, RecurrenceArgs>(b, group), (int)tile * kLongTile, t0, t0 + K, start, from, which);
  }
}

// ---- backward

template <typename T, int V, int K = kSpan>
struct GradInputs {
  Inputs<T, V, K> in;
  Elements<T, V> d[K];
  Elements<float, V> h;  // the state in front of the tile
  bool some;             // (there is one)
  __device__ __forceinline__ void ask(const RecurrenceGradArgs& a, const Group<V, RecurrenceGradArgs>& at, int tile, int t0) {
    const int left = at.length - t0;
    in.ask(a, at, t0);
    const T* pd = at.row((const T*)a.dhs, t0, a.dhs_step, a.dhs_batch);
    if (K >= kSpan && left >= K) {
      const Lane<V> ch = at.ch.here();
#pragma unroll
      for (int k = 0; k < K; ++k, pd += a.dhs_step) d[k] = ch.get(pd);
      branch_end();
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k, pd += a.dhs_step)
        if (within(k, left)) d[k] = at.ch.get(pd);
    }
    const float* from = tile == 0 ? a.h0 : a.states + (tile - 1) * (int64_t)a.batch * a.n;
    some = from != nullptr;
    if (some) h = at.ch.get(from + at.state);
  }
  __device__ __forceinline__ void clear_behind(int left) {
    if (left < K)
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (!within(k, left))
#pragma unroll
          for (int j = 0; j < V; ++j) d[k].v[j] = (T)0.0f;
  }
};
// The map of a wave's gradient against time, from nothing behind it.
template <typename T, int MODE, int V>
__device__ __forceinline__ void map_back(const Steps<T, MODE, V, true>& steps, const Elements<T, V> (&d)[kSpan], float (&R)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) R[j] = 0.0f;
#pragma unroll
  for (int k = kSpan - 1; k >= 0; --k)
#pragma unroll
    for (int j = 0; j < V; ++j) R[j] = steps.s[k][j].keep(R[j] + (float)d[k].v[j]);
}
// From the state h in front of a wave's steps and the gradient r that reaches the last of them from behind, to the one that leaves the first.
template <typename T, int MODE, int V>
__device__ __forceinline__ void replay_back(const RecurrenceGradArgs& a, const Group<V, RecurrenceGradArgs>& at, Steps<T, MODE, V, true>& steps,
                                            const GradInputs<T, V>& in, int t0, float (&h)[V], float (&r)[V]) {
  if (t0 >= at.steps || !at.ch.any) return;
  steps.again();
  const int left = at.length - t0;
  T *qg = at.row((T*)a.dgate, t0, a.dgate_step, a.dgate_batch), *qx = at.row((T*)a.dx, t0, a.dx_step, a.dx_batch);
  float before[kSpan][V];
#pragma unroll
  for (int k = 0; k < kSpan; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      before[k][j] = h[j];
      h[j] = steps.s[k][j].next(h[j]);
    }
  auto step = [&](int k, float (&og)[V], float (&ox)[V]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float e = r[j] + (float)in.d[k].v[j];
      og[j] = steps.s[k][j].dgate(e, before[k][j]);
      ox[j] = steps.s[k][j].dx(e);
      r[j] = steps.s[k][j].keep(e);
    }
  };
  qg += (kSpan - 1) * a.dgate_step;
  qx += (kSpan - 1) * a.dx_step;
  if (left >= kSpan) {
    const Lane<V> ch = at.ch.here();
#pragma unroll
    for (int k = kSpan - 1; k >= 0; --k, qg -= a.dgate_step, qx -= a.dx_step) {
      float og[V], ox[V];
      step(k, og, ox);
      ch.put(qg, og);
      ch.put(qx, ox);
    }
    branch_end();
  } else {
#pragma unroll
    for (int k = kSpan - 1; k >= 0; --k, qg -= a.dgate_step, qx -= a.dx_step) {
      float og[V], ox[V];
      step(k, og, ox);
      if (!within(k, left))
#pragma unroll
        for (int j = 0; j < V; ++j) og[j] = ox[j] = 0.0f;
      if (t0 + k < at.steps) {
        at.ch.put(qg, og);
        at.ch.put(qx, ox);
      }
    }
  }
  if (t0 == 0 && a.dh0) at.ch.put(a.dh0 + at.state, r);
}

// Steps one after the other again: the gradient r that reaches the last of the steps [t, end) from behind, to the one that leaves step t.  WRITE: with
// the gradients of these steps, from `first`, the state in front of step t; `which` as above.
template <typename T, int MODE, int V, bool WRITE>
__device__ __forceinline__ void retreat(const RecurrenceGradArgs& a, const Group<V, RecurrenceGradArgs>& at, int tile, int t, int end, const float (&first)[V],
                                        float (&r)[V], const bool (&which)[V]) {
  const int steps_end = ((WRITE ? at.steps : at.length) + kMend - 1) / kMend * kMend;
  int u = __builtin_amdgcn_readfirstlane((end < steps_end ? end : steps_end) - kMend);
  for (; u >= t; u = __builtin_amdgcn_readfirstlane(u - kMend)) {
    float before[kMend][V], h[V];
    if constexpr (WRITE) {
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] = first[j];
      advance<T, MODE, V, true>(a, at, t, u, h);
    }
    GradInputs<T, V, kMend> in;
    in.ask(a, at, tile, u);
    Steps<T, MODE, V, true, kMend> steps;
    steps.set(in.in, at.length - u);
    in.clear_behind(at.length - u);
    if constexpr (WRITE)
#pragma unroll
      for (int k = 0; k < kMend; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          before[k][j] = h[j];
          h[j] = steps.s[k][j].next_exact(h[j]);
        }
#pragma unroll
    for (int k = kMend - 1; k >= 0; --k) {
      float og[V], ox[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float e = r[j] + (float)in.d[k].v[j];
        if constexpr (WRITE) {
          const bool here = within(k, at.length - u);
          og[j] = here ? steps.s[k][j].dgate(e, before[k][j]) : 0.0f;
          ox[j] = here ? steps.s[k][j].dx(e) : 0.0f;
        }
        r[j] = steps.s[k][j].keep_exact(e);
      }
      if constexpr (WRITE)
        if (within(k, at.steps - u)) {
          at.ch.put(at.row((T*)a.dgate, u + k, a.dgate_step, a.dgate_batch), og, which);
          at.ch.put(at.row((T*)a.dx, u + k, a.dx_step, a.dx_batch), ox, which);
        }
    }
  }
  if constexpr (WRITE)
    if (t == 0 && a.dh0) at.ch.put(a.dh0 + at.state, r, which);
}
// Behind a wave's replay that began in the state h0 and with the gradient r0, and ended in h and r: what is to be formed again is.  `behind`: the
// gradient that reaches the tile from behind.
template <typename T, int MODE, int V>
__device__ __forceinline__ void mend_back(const RecurrenceGradArgs& a, const Group<V, RecurrenceGradArgs>& at, int tile, int t0, const float (&behind)[V],
                                          const float (&h0)[V], const float (&r0)[V], const float (&h)[V], float (&r)[V]) {
  float from[V], again[V];
  bool which[V], of_r[V];
  given<V>(tile == 0 ? a.h0 : a.states + (tile - 1) * (int64_t)a.batch * a.n, at, from);
  const bool some_h = spoiled(from, h, which), some_r = spoiled(behind, r, of_r);
  if (!some_h && !some_r) return;
  advance<T, MODE, V, true>(a, at, tile * kTile, t0, from);
  finite_or<V>(h0, from);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    again[j] = behind[j];
    which[j] = which[j] || of_r[j];
  }
  retreat<T, MODE, V, false>(a, at, tile, t0 + kSpan, (tile + 1) * kTile, from, again, which);
  finite_or<V>(r0, again);
  retreat<T, MODE, V, true>(a, at, tile, t0, t0 + kSpan, from, again, which);
#pragma unroll
  for (int j = 0; j < V; ++j) r[j] = of_r[j] ? again[j] : r[j];
}

template <typename T, int MODE, bool ONE>
__global__ __launch_bounds__(64 * kTileWaves, ONE ? 8 : 4) void recurrence_grad_kernel(RecurrenceGradArgs a) {
  constexpr int V = 1;
  __shared__ float maps[ONE ? 1 : 2][kTileWaves][3][64];
  const int w = __builtin_amdgcn_readfirstlane(wave_id()), waves = blockDim.x / 64, lane = lane_id();
  const Group<V, RecurrenceGradArgs> at(a, blockIdx.x);
  __shared__ float behind[ONE ? 1 : 2][64];
  float back[V];  // wave 0: the gradient that reaches a tile's last state from the steps behind it
  if (w == 0) given<V>(a.dh_last, at, back);
  int turn = 0;
  const int end = at.length == 0 ? 0 : ONE ? kTile : ((at.length - 1) / kTile + 1) * kTile;  // of its last tile
  if (end < at.steps) {
    clear_rows(a, at, (T*)a.dgate, end + w, a.steps, waves, a.dgate_step, a.dgate_batch);
    clear_rows(a, at, (T*)a.dx, end + w, a.steps, waves, a.dx_step, a.dx_batch);
  }
  if (end == 0) {
    if (w == 0 && a.dh0 && at.ch.any) at.ch.put(a.dh0 + at.state, back);
    return;
  }
  int tile = ONE ? 0 : end / kTile - 1;
  GradInputs<T, V> ahead;
  ahead.ask(a, at, tile, tile * kTile + w * kSpan);
  for (; tile >= 0; --tile, turn ^= 1) {
    const int t0 = tile * kTile + w * kSpan;
    GradInputs<T, V> in = ahead;
    Steps<T, MODE, V, true> steps;
    steps.set(in.in, at.length - t0);
    if constexpr (!ONE)
      if (tile > 0) ahead.ask(a, at, tile - 1, t0 - kTile);
    in.clear_behind(at.length - t0);
    // the wave's maps: of the state along time, and of the gradient against it (the same factor)
    float A[V], B[V] = {0.0f}, R[V], h[V], r[V];
    steps.map(A, B);
    map_back(steps, in.d, R);
    maps[turn][w][0][lane] = A[0];
    maps[turn][w][1][lane] = B[0];
    maps[turn][w][2][lane] = R[0];
    if (w == 0) behind[turn][lane] = back[0];
    h[0] = in.some ? in.h.v[0] : 0.0f;
    lds_barrier();
#pragma unroll 4
    for (int u = 0; u < w; ++u) h[0] = fmaf(maps[turn][u][0][lane], h[0], maps[turn][u][1][lane]);
    r[0] = behind[turn][lane];
#pragma unroll 4
    for (int u = waves - 1; u > w; --u) r[0] = fmaf(maps[turn][u][0][lane], r[0], maps[turn][u][2][lane]);
    if (!ONE && w == 0) back[0] = fmaf(A[0], r[0], R[0]);
    const float h_start[V] = {h[0]}, r_start[V] = {r[0]};
    replay_back(a, at, steps, in, t0, h, r);
    if (leaves<2>({h[0], r[0]})) {
      const float from[V] = {behind[turn][lane]};
      const RecurrenceGradArgs b = argument<ONE>(a);
      mend_back<T, MODE, V>(b, ONE ? Group<V, RecurrenceGradArgs>(b, blockIdx.x) : at, tile, t0, from, h_start, r_start, h, r);
    }
    if constexpr (ONE) return;
    if (w == 0 && !is_finite(back[0])) back[0] = r[0];  // (that of the map may be infinite by the map alone)
  }
}

template <typename T, int MODE>
__global__ __launch_bounds__(64 * kTileWaves, 8) void recurrence_grad_tiles_kernel(RecurrenceGradArgs a, Split split) {
  constexpr int V = 1;
  __shared__ uint64_t stage[kWindow][64];
  __shared__ float begin[64];
  __shared__ uint32_t number;
  __shared__ int found;
  auto maps = reinterpret_cast<float(*)[3][64]>(stage);  // [kTileWaves]
  const int w = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id();
  const bool mine = w == kTileWaves - 1;
  uint32_t turn, group;
  if (!take_tile(split, number, turn, group)) return;
  const int tile = (int)(split.tiles - 1 - turn), t0 = tile * kTile + w * kSpan;
  const Group<V, RecurrenceGradArgs> at(a, group);
  if (tile * kTile >= at.length) {  // behind the entry's end
    const int end = t0 + kSpan < at.steps ? t0 + kSpan : at.steps;
    clear_rows(a, at, (T*)a.dgate, t0, end, 1, a.dgate_step, a.dgate_batch);
    clear_rows(a, at, (T*)a.dx, t0, end, 1, a.dx_step, a.dx_batch);
    if (t0 == 0 && a.dh0 && at.ch.any) {
      float r[V];
      given<V>(a.dh_last, at, r);
      at.ch.put(a.dh0 + at.state, r);
    }
    return;
  }
  const int order = (at.length - 1) / kTile - tile;  // in the chain, which begins at the entry's end
  GradInputs<T, V> in;
  in.ask(a, at, tile, t0);
  Steps<T, MODE, V, true> steps;
  steps.set(in.in, at.length - t0);
  in.clear_behind(at.length - t0);
  float A[V], B[V] = {0.0f}, R[V], h[V], r[V];
  steps.map(A, B);
  map_back(steps, in.d, R);
  maps[w][0][lane] = A[0];
  maps[w][1][lane] = B[0];
  maps[w][2][lane] = R[0];
  h[0] = in.some ? in.h.v[0] : 0.0f;
  lds_barrier();
#pragma unroll 4
  for (int u = 0; u < w; ++u) h[0] = fmaf(maps[u][0][lane], h[0], maps[u][1][lane]);
  // the maps of the waves behind it as one; the last wave takes those of all
  float fa = 1.0f, fr = 0.0f;
  const int until = mine ? 0 : w + 1;
#pragma unroll 4
  for (int u = kTileWaves - 1; u >= until; --u) {
    const float one = maps[u][0][lane];
    fa *= one;
    fr = fmaf(one, fr, maps[u][2][lane]);
  }
  const Chain chain = chain_of(split, group);
  if (order > 0) {
    if (mine) leave_map(chain, order, fa, fr);
    look_back(chain, order, stage, found, w, mine, r[0]);
  } else if (mine) {
    given<V>(a.dh_last, at, r);
  }
  bool late = false;  // as forward
  if (mine) {
    begin[lane] = r[0];
    const float end[V] = {fmaf(fa, r[0], fr)};
    leave_end(chain, order, end[0]);
    late = leaves(end);
    lds_barrier();
    mark_end(chain, order, !late);
  } else {
    lds_barrier();
    r[0] = begin[lane];
  }
  if (leaves(r)) {
    if (mine) maps[0][0][lane] = order > 0 ? end_of(chain, order - 1) : r[0];
    lds_barrier();
    begin[lane] = r[0] = maps[0][0][lane];
  }
  if (!mine) r[0] = fmaf(fa, r[0], fr);
  const float h_start[V] = {h[0]}, r_start[V] = {r[0]};
  replay_back(a, at, steps, in, t0, h, r);
  if (late) {
    bool which[V];
    const float from[V] = {begin[lane]};
    float end[V] = {fmaf(fa, from[0], fr)};
    if (spoiled(from, end, which)) {
      float again[V] = {from[0]};
      const RecurrenceGradArgs b = argument<true>(a);
      retreat<T, MODE, V, false>(b, Group<V, RecurrenceGradArgs>(b, group), tile, tile * kTile, (tile + 1) * kTile, again, again, which);
      end[0] = which[0] ? again[0] : end[0];
    }
    leave_end(chain, order, end[0]);
    mark_end(chain, order, true);
  }
  if (leaves<2>({h[0], r[0]})) {
    const float from[V] = {begin[lane]};
    const RecurrenceGradArgs b = argument<true>(a);
    mend_back<T, MODE, V>(b, Group<V, RecurrenceGradArgs>(b, group), tile, t0, from, h_start, r_start, h, r);
  }
}

// ---- launches

template <typename F>
hipError_t with_type(int type, int mode, F f) {
  auto modes = [&](auto t) {
    return mode == AMQ_RECURRENCE_BLEND ? f(t, std::integral_constant<int, AMQ_RECURRENCE_BLEND>())
                                        : f(t, std::integral_constant<int, AMQ_RECURRENCE_DECAY>());
  };
  return type == AMQ_F32 ? modes(float()) : type == AMQ_BF16 ? modes(bf16()) : modes(f16());
}

// Waves of a tile: 16 where a tile begins where a state was left, else as many as share the steps evenly.
int waves_of(int64_t steps, bool even) {
  const int64_t spans = (steps + kSpan - 1) / kSpan, tiles = (spans + kTileWaves - 1) / kTileWaves;
  return (int)(tiles == 1 ? spans : even ? (spans + tiles - 1) / tiles : kTileWaves);
}
int64_t groups_of(int64_t batch, int64_t n, int V) { return batch * ((n + 64 * V - 1) / (64 * V)); }
int64_t tiles_of(int64_t steps, int tile) { return (steps + tile - 1) / tile; }

// Channels of a lane: two of 16 bits where a workgroup walks over tiles forward and groups of 64 channels are more than the card holds at
// once (300 x 17408 13.9 us, with one 16.8; 1000 x 32768 41 and 48; but 2000 x 16384 62 and 46); one otherwise (35 x 262144 backward
// takes 1.12 times as long with two).
bool two_channels(int64_t batch, int64_t n) { return n % 2 == 0 && groups_of(batch, n, 1) > 256; }

// The form with the least time, by measurement.  Per 128 steps a workgroup per group takes c0 us and 256 of them, one on every compute unit,
// c0 + c1; a workgroup per tile e for 256 groups, and 7.5 us more for clearing the marks, the second launch and the chain.  Steps x
// channels, a workgroup per group and one per tile: 16-bit types 300 x 1024 8.4 and 10.0, 1000 x 1024 18.7 and 11.0, 1000 x 8192 20.3 and
// 16.4, 1000 x 12288 21.1 and 21.4, 3000 x 12288 62 and 55, 3000 x 16384 67 and 69, 1000 x 24576 35 and 42; float 1000 x 4096 17.8 and
// 15.4, 1000 x 12288 30.2 and 33.7; backward 200 x 1024 8.9 and 11.1, 1000 x 1024 28 and 11, 1000 x 16384 39 and 50, 3000 x 12288 109 and
// 98, float 3000 x 8192 113 and 103, 1000 x 24576 107 and 102.  The constants are those of up to 256 groups; for more they are only what
// the choice goes by: 3000 x 16500 bfloat16 takes 91 us in tiles, by them 68, backward 162 and 126.  Beyond four rounds of the card the last
// one's share is small, and the workspace would grow with the channels (64 of them to a tile, used or not).
bool splits(int64_t batch, int64_t n, int64_t steps, bool wide, bool backward) {
  const bool pairs = !wide && !backward && two_channels(batch, n);
  const double c0 = pairs ? 2.6 : wide ? backward ? 2.7 : 1.75 : backward ? 3.25 : 2.1;
  const double c1 = pairs ? 2.27 : wide ? backward ? 5.5 : 2.7 : backward ? 1.6 : 0.75;
  const double e = wide ? backward ? 7.85 : 4.5 : backward ? 5.0 : 2.55;
  const int64_t groups = groups_of(batch, n, 1), g = groups_of(batch, n, pairs ? 2 : 1), last = g % 256;
  if (steps <= kTile || groups > 4 * 256) return false;
  const double one = (double)(g / 256) * (c0 + c1) + (last ? c0 + c1 * (double)last / 256 : 0.0);
  return (double)steps / kTile * (one - e * (double)groups / 256) > 7.5;
}

hipError_t split_of(int64_t groups, int64_t tiles, void* ws, hipStream_t s, Split& out) {
  const SplitLayout l(groups, tiles);
  char* p = static_cast<char*>(ws);
  out = {reinterpret_cast<uint32_t*>(p), reinterpret_cast<uint32_t*>(p + l.marks), reinterpret_cast<uint64_t*>(p + l.maps),
         reinterpret_cast<uint32_t*>(p + l.ends), tiles, (uint32_t)groups, groups >= 256 ? 1u : groups < kCounters ? (uint32_t)groups : kCounters};
  const int64_t words = (int64_t)(l.maps / sizeof(uint32_t));
  split_clear_kernel<<<dim3((unsigned)(words / 1024 < 256 ? words / 1024 + 1 : 256)), dim3(256), 0, s>>>(out.counter, words);
  return hipGetLastError();
}
// A grid has less than 2^32 threads, which batches of millions of entries and millions of steps of a thousand pass: those take several launches.
int64_t most_blocks(int waves) { return 0xffffffffLL / (64 * waves); }
// The batch from entry b on.  (`batch` stays what it is: the states in front of two tiles are that many entries apart.)
RecurrenceArgs from_entry(RecurrenceArgs a, int64_t b) {
  const int64_t size = a.type == AMQ_F32 ? 4 : 2;
  a.gate = (const char*)a.gate + b * a.gate_batch * size;
  a.x = (const char*)a.x + b * a.x_batch * size;
  a.hs = (char*)a.hs + b * a.hs_batch * size;
  if (a.lengths) a.lengths += b;
  if (a.h0) a.h0 += b * a.n;
  if (a.h_last) a.h_last += b * a.n;
  if (a.states) a.states += b * a.n;
  return a;
}
RecurrenceGradArgs from_entry(RecurrenceGradArgs a, int64_t b) {
  const int64_t size = a.type == AMQ_F32 ? 4 : 2;
  a.dhs = (const char*)a.dhs + b * a.dhs_batch * size;
  a.gate = (const char*)a.gate + b * a.gate_batch * size;
  a.x = (const char*)a.x + b * a.x_batch * size;
  a.dgate = (char*)a.dgate + b * a.dgate_batch * size;
  a.dx = (char*)a.dx + b * a.dx_batch * size;
  if (a.lengths) a.lengths += b;
  if (a.h0) a.h0 += b * a.n;
  if (a.states) a.states += b * a.n;
  if (a.dh_last) a.dh_last += b * a.n;
  if (a.dh0) a.dh0 += b * a.n;
  return a;
}
template <typename A, typename F>
hipError_t launch_tiles(const A& a, int tile, hipStream_t s, F kernel) {
  const int64_t groups = groups_of(a.batch, a.n, 1);
  Split split;
  const hipError_t e = split_of(groups, tiles_of(a.steps, tile), a.ws, s, split);
  if (e != hipSuccess) return e;
  // as many workgroups for every counter as the one with the most tiles needs; the counters run on from launch to launch
  int64_t blocks = (groups + split.kinds - 1) / split.kinds * split.tiles * split.kinds;
  for (const int64_t most = most_blocks(kTileWaves) / split.kinds * split.kinds; blocks > 0; blocks -= most) {
    kernel<<<dim3((unsigned)(blocks < most ? blocks : most)), dim3(64 * kTileWaves), 0, s>>>(a, split);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename A, typename F>
hipError_t launch_groups(const A& a, int channels, bool even, hipStream_t s, F kernel) {
  const int waves = waves_of(a.steps, even);
  const int64_t pieces = groups_of(1, a.n, channels), most = most_blocks(waves) / pieces;  // of an entry; entries of a launch
  for (int64_t b = 0; b < a.batch; b += most) {
    const int64_t entries = a.batch - b < most ? a.batch - b : most;
    kernel<<<dim3((unsigned)(entries * pieces)), dim3(64 * waves), 0, s>>>(from_entry(a, b));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// (batch entries may count as channels of one entry in the launch, so the larger need of either)
size_t workspace(int64_t steps, int64_t batch, int64_t n, int type, bool backward) {
  size_t most = 0;
  for (int flat = 0; flat < 2; ++flat) {
    const int64_t b = flat ? 1 : batch, c = flat ? batch * n : n;
    if (!splits(b, c, steps, type == AMQ_F32, backward)) continue;
    const size_t need = SplitLayout(groups_of(b, c, 1), tiles_of(steps, backward ? kTile : kLongTile)).bytes;
    most = need > most ? need : most;
  }
  return most;
}

}  // namespace

bool recurrence_entries_join(int64_t steps, int64_t channels, int type, bool backward) {
  if (splits(1, channels, steps, type == AMQ_F32, backward)) return true;
  const bool pairs = type != AMQ_F32 && !backward && steps > kTile && two_channels(1, channels);
  return groups_of(1, channels, pairs ? 2 : 1) <= most_blocks(waves_of(steps, !backward));
}

size_t recurrence_workspace(int64_t steps, int64_t batch, int64_t n, int type) { return workspace(steps, batch, n, type, false); }
size_t recurrence_grad_workspace(int64_t steps, int64_t batch, int64_t n, int type) { return workspace(steps, batch, n, type, true); }

hipError_t launch_recurrence(const RecurrenceArgs& a, hipStream_t s) {
  return with_type(a.type, a.mode, [&](auto t, auto m) {
    using T = decltype(t);
    constexpr int M = decltype(m)::value;
    constexpr bool wide = sizeof(T) == 4;
    if (splits(a.batch, a.n, a.steps, wide, false)) return launch_tiles(a, kLongTile, s, recurrence_tiles_kernel<T, M>);
    if (a.steps <= kTile) return launch_groups(a, 1, true, s, recurrence_kernel<T, M, 1, true>);
    if constexpr (!wide)
      if (two_channels(a.batch, a.n)) return launch_groups(a, 2, true, s, recurrence_kernel<T, M, 2, false>);
    return launch_groups(a, 1, true, s, recurrence_kernel<T, M, 1, false>);
  });
}

hipError_t launch_recurrence_grad(const RecurrenceGradArgs& a, hipStream_t s) {
  return with_type(a.type, a.mode, [&](auto t, auto m) {
    using T = decltype(t);
    constexpr int M = decltype(m)::value;
    constexpr bool wide = sizeof(T) == 4;
    if (splits(a.batch, a.n, a.steps, wide, true)) return launch_tiles(a, kTile, s, recurrence_grad_tiles_kernel<T, M>);
    if (a.steps <= kTile) return launch_groups(a, 1, false, s, recurrence_grad_kernel<T, M, true>);
    return launch_groups(a, 1, false, s, recurrence_grad_kernel<T, M, false>);
  });
}

}  // namespace amq
