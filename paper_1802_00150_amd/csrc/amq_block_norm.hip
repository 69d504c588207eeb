// The join of a block with the residual stream, forward and backward: the norm behind the block, its gate and scale, the
// residual, and the norm in front of the next block, in one pass.
//
//   z = (x - mu) r,  u = z w + b,  y = residual + s act(gate) u,  zy = (y - mu') r',  normed = zy w' + b'
//   G = dy + r' (g' - mean g' - zy mean(g' zy)),  g' = dnormed w';     dresidual = G,  dgate = G s u act'(gate)
//   g = G s act w:  dx = r (g - mean g - z mean(g z));   dw = s S1, db = s S0, ds = w S1 + b S0,  S1 = sum G act z,  S0 = sum G act
//   dw' = sum dnormed zy,  db' = sum dnormed  (sums over rows)
//
// About 30 operations per entry forward and 60 backward, against 10 and 16 bytes (16-bit types): bound by memory, or by latency
// for few rows.  So every entry is read once and kept in registers between the four sums of a row and the results; a row belongs to one
// wave (its sums need no barrier) or to a workgroup of 4, 8 or 16, a short one to 16 or 32 lanes of a wave.  Workgroups walk over rows, with
// the parameters and, in the backward pass, four sums per column in registers (in LDS where a lane has two pieces of a row); those leave one
// partial row per workgroup, added up by a second launch in a fixed order.  normed is formed from y before its rounding; statistics and
// sums are binary32.
//
// Measured (a large copy 5.1 TB/s): 8960 x 1024 half 17.6 us, 5.2 TB/s (part of it stays in the memory-side cache); backward 8960 x 1500
// bfloat16 with a float residual 59 us, 5.0, and 5 for the second launch; 8960 x 1024 bfloat16 backward 43, 3.4, with vector
// instructions (87 per entry, some to read spilled scalars back) and latency in the way; 2000 x 8192 bfloat16 backward 100, 2.6: one workgroup per
// compute unit that has no row ahead; forward 41, 4.0.  Rows above 8192 entries do not fit the registers of 16 waves (82 to 168 are spilled forward,
// 150 to 217 backward): 2000 x 16384 bfloat16 177 us and 452, float 221 and 786.
#include "../../include/amq.h"

#include <type_traits>

#include "amq_device.h"
#include "amq_train.h"
#include "amq_typed.h"

namespace amq {
namespace {

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// v + its value 16 or 32 lanes away (the swap of two copies leaves one half's values twice in either).
__device__ __forceinline__ float add_16_away(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_32_away(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
// Sums over the even lanes and over the odd lanes of a value; every lane ends with that of its kind.
__device__ __forceinline__ float sums_by_parity(float v) {
  v += dpp<0x4E>(v);   // quad_perm [2,3,0,1]
  v += dpp<0x124>(v);  // row_ror 4
  v += dpp<0x128>(v);  // row_ror 8
  return add_32_away(add_16_away(v));
}

// Sums of two values over the `waves` waves, up to 16, that share a row, beginning with wave `first`: a in even lanes and b in odd ones
// take one reduction together.  One barrier, of all that meet in the workgroup: the slots of consecutive calls alternate.
__device__ __forceinline__ void row_sum2(float& a, float& b, float (*slots)[2], int& turn, int first, int waves) {
  const bool odd = lane_id() & 1;
  float v = (odd ? b : a) + dpp<0xB1>(odd ? a : b);  // quad_perm [1,0,3,2]
  v = sums_by_parity(v);
  if (waves > 1) {
    float(*s)[2] = slots + turn * 16;
    turn ^= 1;
    if (lane_id() < 2) s[wave_id()][lane_id()] = v;
    lds_barrier();
    v = lane_id() < 2 * waves ? s[first + (lane_id() >> 1)][lane_id() & 1] : 0.0f;
    v = sums_by_parity(v);
  }
  a = lane_of(v, 0);
  b = lane_of(v, 1);
}
// Sum over 16 or 32 lanes that share a row.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  static_assert(L == 16 || L == 32, "lanes of a row");
  v = v + dpp<0xB1>(v);  // quad_perm [1,0,3,2]
  v += dpp<0x4E>(v);     // quad_perm [2,3,0,1]
  v += dpp<0x124>(v);    // row_ror 4
  v += dpp<0x128>(v);    // row_ror 8
  return L == 32 ? add_16_away(v) : v;
}
template <int L>
__device__ __forceinline__ float row_sum(float a, float (*slots)[2], int& turn, int first, int waves) {
  if constexpr (L < 64) return lanes_sum<L>(a);
  float b = 0.0f;
  row_sum2(a, b, slots, turn, first, waves);
  return a;
}

// Piece j of a row's pieces of V entries for thread `tid` of `threads`.  The last one ends with the row and overlaps the one before
// it (its first `repeated` entries count there); threads past the end hold it once more with nothing that counts, and store
// nothing.  (n >= V.)  Rows are the same in all lanes of a wave: an address is theirs and 32 bits of a lane.
template <int V>
struct Piece {
  uint32_t start;
  int repeated;
  bool even;  // the row is a number of whole pieces (the same in all lanes)
  __device__ __forceinline__ Piece(int j, int tid, int n, int threads) {
    const int c = (j * threads + tid) * V, s = c < n - V ? c : n - V;
    start = (uint32_t)s;
    repeated = c - s < V ? c - s : V;
    even = n % V == 0;
  }
  __device__ __forceinline__ bool counts(int i) const { return i >= repeated; }
  __device__ __forceinline__ bool any() const { return repeated < V; }
  // (A new value at every use: the compiler made 64-bit addresses of lanes that it kept over all rows, most of the registers.)
  template <typename T>
  __device__ __forceinline__ uint32_t offset() const {
    uint32_t bytes = start * (uint32_t)sizeof(T);
    asm volatile("" : "+v"(bytes));
    return bytes;
  }
  template <typename T>
  __device__ __forceinline__ Elements<T, V> get(const T* row) const {
    return *reinterpret_cast<const Elements<T, V>*>(reinterpret_cast<const char*>(row) + offset<T>());
  }
  // parameters, absent ones (null) as `absent`
  template <typename P>
  __device__ __forceinline__ void get(const void* p, float absent, float (&out)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = absent;
    if (!p) return;
    const Elements<P, V> e = get((const P*)p);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = (float)e.v[i];
  }
  // A result; entries that the piece before has are stored there (they may lie where an operand did).  (The values of the row's end are
  // made new ones, so that the compiler does not join both ways of storing into one of single entries.)
  template <typename T>
  __device__ __forceinline__ void put(T* row, const float (&v)[V]) const {
    T* p = reinterpret_cast<T*>(reinterpret_cast<char*>(row) + offset<T>());
    if (repeated == 0) {
      store_whole<T, V>(p, v);
    } else if (!even && any()) {
#pragma unroll
      for (int i = 1; i < V; ++i) {
        float e = v[i];
        asm volatile("" : "+v"(e));
        if (i >= repeated) p[i] = (T)e;
      }
    }
  }
};

// act(z) and its slope for V entries.
template <typename T, int V>
__device__ __forceinline__ void gates_of(int act, const Elements<T, V>& z, float (&value)[V], float (&slope)[V]) {
  if (act == AMQ_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      value[i] = (float)z.v[i];
      slope[i] = 1.0f;
    }
    return;
  }
  float p[V], q[V];  // sigmoid(z), 1 - sigmoid(z)
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float v = (float)z.v[i], e = __expf(-fabsf(v)), r = __builtin_amdgcn_rcpf(1.0f + e), small = e * r;
    p[i] = v >= 0.0f ? r : small;
    q[i] = v >= 0.0f ? small : r;
  }
  if (act == AMQ_ACT_SIGMOID) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      value[i] = p[i];
      slope[i] = p[i] * q[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float v = (float)z.v[i];
      value[i] = v * p[i];
      slope[i] = p[i] * fmaf(v, q[i], 1.0f);
    }
  }
}

template <typename T, int V, int NV, typename F>
__device__ __forceinline__ void ask(Elements<T, V> (&r)[NV], const void* base, int64_t offset, F piece) {
#pragma unroll
  for (int j = 0; j < NV; ++j) r[j] = piece(j).get((const T*)base + offset);
}

// Makes the compiler take what was read as new values, so that it does not keep what was formed from them.
template <typename T, int V>
__device__ __forceinline__ void again(Elements<T, V>& e) {
  if constexpr (sizeof(e) % 4 == 0) {
    typedef uint32_t Words __attribute__((ext_vector_type(sizeof(e) / 4)));
    Words w = __builtin_bit_cast(Words, e);
#pragma unroll
    for (int i = 0; i < (int)sizeof(e) / 4; ++i) {
      uint32_t v = w[i];
      asm volatile("" : "+v"(v));
      w[i] = v;
    }
    e = __builtin_bit_cast(Elements<T, V>, w);
  }
}

// T: x, gate and normed; R: residual and y; P: parameters.  W waves per row (or L lanes of one wave, short rows sharing it), NV pieces of V
// entries per lane.
template <typename T, typename R, typename P, int V, int W, int NV, int L>
__global__ __launch_bounds__(W > 4 ? W * 64 : 256) void block_norm_kernel(BlockNormArgs a) {
  constexpr int kLanes = L < 64 ? L : W * 64, kRows = (W > 4 ? W * 64 : 256) / kLanes;
  __shared__ float slots[2 * 16][2];
  int turn = 0;
  const int wave = L < 64 ? 0 : __builtin_amdgcn_readfirstlane(wave_id() / W * W);  // the row's first
  const int group = L < 64 ? (int)threadIdx.x / L : wave / W, tid = (int)threadIdx.x - group * kLanes;
  auto piece = [&](int j) __attribute__((always_inline)) { return Piece<V>(j, tid, a.n, kLanes); };
  const float inv_n = 1.0f / (float)a.n;
  Elements<T, V> rx[NV], rg[NV];
  Elements<R, V> rr[NV];
  auto fetch_row = [&](int64_t row) __attribute__((always_inline)) {
    if (row >= a.rows) return;
    ask(rx, a.x, row * a.ld_x, piece);
    ask(rr, a.residual, row * a.ld_r, piece);
    if (a.gate) ask(rg, a.gate, row * a.ld_g, piece);
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t first = (int64_t)blockIdx.x * kRows;  // of the workgroup's rows: its groups meet at barriers, so they leave together
  fetch_row(first + group);
  // the scale is folded into the first norm's parameters
  float w[NV][V], b[NV][V], w2[NV][V], b2[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float s[V];
    piece(j).template get<P>(a.weight, 1.0f, w[j]);
    piece(j).template get<P>(a.bias, 0.0f, b[j]);
    piece(j).template get<P>(a.scale, 1.0f, s);
    piece(j).template get<P>(a.next_weight, 1.0f, w2[j]);
    piece(j).template get<P>(a.next_bias, 0.0f, b2[j]);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      w[j][i] *= s[i];
      b[j][i] *= s[i];
    }
  }
  for (; first < a.rows; first += step) {
    const int64_t row = first + group;
    const bool here = row < a.rows;
    float x[NV][V], y[NV][V], act[NV][V], s = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[j][i] = here ? (float)rx[j].v[i] : 0.0f;
        y[j][i] = here ? (float)rr[j].v[i] : 0.0f;
        act[j][i] = 1.0f;
        s += piece(j).counts(i) ? x[j][i] : 0.0f;
      }
      if (a.gate && here) {
        float slope[V];
        gates_of(a.act, rg[j], act[j], slope);
      }
    }
    fetch_row(row + step);
    const float mean = row_sum<L>(s, slots, turn, wave, W) * inv_n;
    s = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[j][i] -= mean;
        s = fmaf(piece(j).counts(i) ? x[j][i] : 0.0f, x[j][i], s);
      }
    const float rstd = 1.0f / sqrtf(row_sum<L>(s, slots, turn, wave, W) * inv_n + a.eps);
    s = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        y[j][i] = fmaf(fmaf(x[j][i] * rstd, w[j][i], b[j][i]), act[j][i], y[j][i]);
        s += piece(j).counts(i) ? y[j][i] : 0.0f;
      }
      if (here) piece(j).put((R*)a.y + row * a.ld_y, y[j]);
    }
    float mean_y = 0.0f, rstd_y = 0.0f;
    if (a.normed) {
      mean_y = row_sum<L>(s, slots, turn, wave, W) * inv_n;
      s = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          y[j][i] -= mean_y;
          s = fmaf(piece(j).counts(i) ? y[j][i] : 0.0f, y[j][i], s);
        }
      rstd_y = 1.0f / sqrtf(row_sum<L>(s, slots, turn, wave, W) * inv_n + a.eps);
      if (here)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
          for (int i = 0; i < V; ++i) y[j][i] = fmaf(y[j][i] * rstd_y, w2[j][i], b2[j][i]);
          piece(j).put((T*)a.normed + row * a.ld_n, y[j]);
        }
    }
    if (tid == 0 && here && a.stats) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = rstd;
      if (a.normed) {
        a.stats[2 * a.rows + row] = mean_y;
        a.stats[3 * a.rows + row] = rstd_y;
      }
    }
  }
}

// `waves` waves per row (or L lanes of one wave), as many rows in a workgroup as 16 waves have room for.
template <typename T, typename R, typename P, int V, int NV, int L>
__global__ __launch_bounds__(1024) void block_norm_grad_kernel(BlockNormGradArgs a, int waves) {
  __shared__ float slots[2 * 16][2];
  // [group][sum][j][i][thread]: consecutive lanes on consecutive banks
  constexpr bool kInLds = NV == 2;  // the sums themselves lie there (one row per workgroup), for want of registers
  __shared__ float shared_sums[(kInLds ? 4 : NV == 1 ? 2 : 1) * (NV > 2 ? 1 : 1024 * NV * V)];
  int turn = 0;
  const int threads = L < 64 ? L : waves * 64, groups = blockDim.x / threads, entries = threads * NV * V;
  const int group = L < 64 ? (int)threadIdx.x / L : __builtin_amdgcn_readfirstlane(wave_id() / waves), tid = (int)threadIdx.x - group * threads;
  auto row_sums = [&](float& u, float& v) __attribute__((always_inline)) {
    if constexpr (L < 64) {
      u = lanes_sum<L>(u);
      v = lanes_sum<L>(v);
    } else {
      row_sum2(u, v, slots, turn, group * waves, waves);
    }
  };
  auto piece = [&](int j) __attribute__((always_inline)) { return Piece<V>(j, tid, a.n, threads); };
  // scale x weight, scale x bias, next_weight; 0 where an entry does not count, so that sums along the row leave it out.  With one piece a lane
  // has room for them and for a row ahead; with more it reads them again for every row (from L2).
  constexpr bool kRoom = NV == 1;
  float sw[NV][V], sb[NV][V], w2[NV][V];
  auto first_parameters = [&](int j) __attribute__((always_inline)) {
    const Piece<V> p = piece(j);
    float sc[V];
    p.template get<P>(a.scale, 1.0f, sc);
    p.template get<P>(a.weight, 1.0f, sw[j]);
    p.template get<P>(a.bias, 0.0f, sb[j]);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sw[j][i] = p.counts(i) ? sw[j][i] * sc[i] : 0.0f;
      sb[j][i] *= sc[i];
    }
  };
  auto next_parameters = [&](int j) __attribute__((always_inline)) {
    const Piece<V> p = piece(j);
    p.template get<P>(a.next_weight, 1.0f, w2[j]);
#pragma unroll
    for (int i = 0; i < V; ++i) w2[j][i] = p.counts(i) ? w2[j][i] : 0.0f;
  };
  // sums over the rows of G act z, G act, dnormed zy, dnormed
  float sums[4][NV][V];
  auto in_lds = [&](int k, int j, int i) __attribute__((always_inline)) -> float& {
    return shared_sums[((k * NV + j) * V + i) * 1024 + threadIdx.x];
  };
  auto sum_up = [&](int k, int j, int i, float u, float v) __attribute__((always_inline)) {
    if constexpr (kInLds) in_lds(k, j, i) = fmaf(u, v, in_lds(k, j, i));
    else sums[k][j][i] = fmaf(u, v, sums[k][j][i]);
  };
  const float inv_n = 1.0f / (float)a.n;
  struct Row {
    Elements<T, V> x[NV], g[NV], n[NV];
    Elements<R, V> y[NV], d[NV];
    float mean, rstd, mean_y, rstd_y;
  };
  auto ask_first = [&](Row& r, int64_t row) __attribute__((always_inline)) {
    if (row >= a.rows) return;
    if (a.dnormed) {
      ask(r.n, a.dnormed, row * a.ld_dn, piece);
      ask(r.y, a.y, row * a.ld_y, piece);
      r.mean_y = a.stats[2 * a.rows + row];
      r.rstd_y = a.stats[3 * a.rows + row];
    }
    if (a.dy) ask(r.d, a.dy, row * a.ld_dy, piece);
  };
  auto ask_second = [&](Row& r, int64_t row) __attribute__((always_inline)) {
    if (row >= a.rows) return;
    ask(r.x, a.x, row * a.ld_x, piece);
    if (a.gate) ask(r.g, a.gate, row * a.ld_g, piece);
    r.mean = a.stats[row];
    r.rstd = a.stats[a.rows + row];
  };
  auto apart = [] __attribute__((always_inline)) {
    if constexpr (!kRoom) __builtin_amdgcn_sched_barrier(0);
  };
  const int64_t step = (int64_t)gridDim.x * groups;
  Row ahead;
  if constexpr (kRoom) {
    ask_first(ahead, (int64_t)blockIdx.x * groups + group);
    ask_second(ahead, (int64_t)blockIdx.x * groups + group);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (kRoom) {
      first_parameters(j);
      next_parameters(j);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if constexpr (kInLds) in_lds(k, j, i) = 0.0f;
        else sums[k][j][i] = 0.0f;
      }
  }
  for (int64_t first = (int64_t)blockIdx.x * groups; first < a.rows; first += step) {
    const int64_t row = first + group;
    const bool here = row < a.rows;
    Row now;
    if constexpr (kRoom) {
      now = ahead;
      ask_first(ahead, row + step);
      ask_second(ahead, row + step);
    } else {
      ask_first(now, row);
    }
    float G[NV][V], s = 0.0f, q = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) G[j][i] = a.dy ? (float)now.d[j].v[i] : 0.0f;
    if (a.dnormed) {
      float zy[NV][V], g[NV][V];
      const float shift = -now.mean_y * now.rstd_y;
      if (here)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          apart();
          if constexpr (!kRoom) next_parameters(j);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float d = (float)now.n[j].v[i];
            zy[j][i] = fmaf((float)now.y[j].v[i], now.rstd_y, shift);
            sum_up(2, j, i, d, zy[j][i]);
            sum_up(3, j, i, d, 1.0f);
            g[j][i] = d * w2[j][i];
            s += g[j][i];
            q = fmaf(g[j][i], zy[j][i], q);
          }
        }
      apart();
      if constexpr (!kRoom)
#pragma unroll
        for (int j = 0; j < NV; ++j) again(now.y[j]), again(now.n[j]);
      row_sums(s, q);
      s *= inv_n;
      q *= inv_n;
      if (here)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            if constexpr (!kRoom) {  // (formed again: what was read takes less room)
              if (i == 0) next_parameters(j);
              zy[j][i] = fmaf((float)now.y[j].v[i], now.rstd_y, shift);
              g[j][i] = (float)now.n[j].v[i] * w2[j][i];
            }
            G[j][i] = fmaf(now.rstd_y, fmaf(-zy[j][i], q, g[j][i] - s), G[j][i]);
          }
    }
    s = q = 0.0f;
    apart();
    if constexpr (!kRoom) ask_second(now, row);
    float g[NV][V], z[NV][V];
    const float shift = -now.mean * now.rstd;
    if (here) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        apart();
        if constexpr (!kRoom) first_parameters(j);
        if (a.dresidual) piece(j).put((R*)a.dresidual + row * a.ld_dr, G[j]);
#pragma unroll
        for (int i = 0; i < V; ++i) z[j][i] = fmaf((float)now.x[j].v[i], now.rstd, shift);
        if (a.gate) {
          float act[V], slope[V];
          gates_of(a.act, now.g[j], act, slope);
          if (a.dgate) {
            float dg[V];
#pragma unroll
            for (int i = 0; i < V; ++i) dg[i] = G[j][i] * fmaf(z[j][i], sw[j][i], sb[j][i]) * slope[i];
            piece(j).put((T*)a.dgate + row * a.ld_dg, dg);
          }
#pragma unroll
          for (int i = 0; i < V; ++i) G[j][i] *= act[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sum_up(0, j, i, G[j][i], z[j][i]);
          sum_up(1, j, i, G[j][i], 1.0f);
          g[j][i] = G[j][i] * sw[j][i];
          s += g[j][i];
          q = fmaf(g[j][i], z[j][i], q);
        }
      }
    }
    if constexpr (!kRoom)
#pragma unroll
      for (int j = 0; j < NV; ++j) again(now.x[j]);
    row_sums(s, q);
    s *= inv_n;
    q *= inv_n;
    if (here)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          if constexpr (!kRoom) z[j][i] = fmaf((float)now.x[j].v[i], now.rstd, shift);
          o[i] = now.rstd * fmaf(-z[j][i], q, g[j][i] - s);
        }
        piece(j).put((T*)a.dx + row * a.ld_dx, o);
      }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 4 * a.n;
  if (NV == 1 && groups > 1) {
    for (int half = 0; half < 2; ++half) {
      if (half) __syncthreads();
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) shared_sums[((group * 2 + k) * V + i) * threads + tid] = half ? sums[2 + k][0][i] : sums[k][0][i];
      __syncthreads();
      for (int at = threadIdx.x; at < 2 * entries; at += groups * threads) {
        const int k = at >= entries, of = at - k * entries, i = of / threads;
        float sum = 0.0f;
        for (int r = 0; r < groups; ++r) sum += shared_sums[r * 2 * entries + at];
        const Piece<V> p(0, of - i * threads, a.n, threads);
        if (p.counts(i)) part[(int64_t)(half * 2 + k) * a.n + p.start + i] = sum;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (piece(j).counts(i)) part[(int64_t)k * a.n + piece(j).start + i] = kInLds ? in_lds(k, j, i) : sums[k][j][i];
  }
}

// Adds up the partial rows and forms the parameters' gradients: 16 columns per workgroup, 64 groups of partial rows side by side.
template <typename P>
__global__ __launch_bounds__(1024) void block_norm_sum_kernel(BlockNormGradArgs a, int parts) {
  __shared__ float sums[4][64][17];
  const int lane = threadIdx.x & 15, group = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
  float s[4] = {};
  if (c < a.n)
#pragma unroll 4
    for (int p = group; p < parts; p += 64)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += a.part[((int64_t)p * 4 + k) * a.n + c];
#pragma unroll
  for (int k = 0; k < 4; ++k) sums[k][group][lane] = s[k];
  __syncthreads();
  if (group < 4) {  // one wave: 16 groups each, then the four of them
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s[k] = 0.0f;
#pragma unroll
      for (int g = 0; g < 16; ++g) s[k] += sums[k][group * 16 + g][lane];
      s[k] += __shfl_xor(s[k], 16, 64);
      s[k] += __shfl_xor(s[k], 32, 64);
    }
    if (group == 0 && c < a.n) {
      const float w = a.weight ? (float)((const P*)a.weight)[c] : 1.0f, b = a.bias ? (float)((const P*)a.bias)[c] : 0.0f;
      const float sc = a.scale ? (float)((const P*)a.scale)[c] : 1.0f;
      if (a.dweight) ((P*)a.dweight)[c] = (P)(sc * s[0]);
      if (a.dbias) ((P*)a.dbias)[c] = (P)(sc * s[1]);
      if (a.dscale) ((P*)a.dscale)[c] = (P)fmaf(w, s[0], b * s[1]);
      if (a.dnext_weight) ((P*)a.dnext_weight)[c] = (P)s[2];
      if (a.dnext_bias) ((P*)a.dnext_bias)[c] = (P)s[3];
    }
  }
}

// Forward: waves per row, pieces per lane, and lanes per row.  16 entries per lane at most (one wave up to 1024).  Few rows go to four waves each
// from 512 entries on, where the row's latency counts; short ones share a wave (35000 x 64 bfloat16 29 us with a wave each, backward 30).
struct Shape {
  int waves, pieces, lanes;
};
constexpr int kPerLane = 16;
template <int V>
Shape shape_of(int64_t rows, int n) {
  if (n <= 16 * V) return {1, 1, 16};
  if (n <= 32 * V) return {1, 1, 32};
  for (int p = 1; p * V <= kPerLane; p *= 2)
    if (n <= 64 * p * V && (rows > 512 || n <= 512)) return {1, p, 64};
  for (int p = 1; p * V <= kPerLane; p *= 2)
    if (n <= 256 * p * V) return {4, p, 64};
  return {n <= 512 * kPerLane ? 8 : 16, kPerLane / V, 64};
}

template <typename F>
hipError_t with_types(int type, int residual, int param, F f) {
  auto params = [&](auto t, auto r) { return param == AMQ_F32 ? f(t, r, float()) : f(t, r, t); };
  if (type == AMQ_F32) return f(float(), float(), float());
  if (type == AMQ_BF16) return residual == AMQ_F32 ? params(bf16(), float()) : params(bf16(), bf16());
  return residual == AMQ_F32 ? params(f16(), float()) : params(f16(), f16());
}
template <int V, typename F>
hipError_t with_shape(Shape h, F f) {
#define AMQ_SHAPE(W, NV, L)                                     \
  if (h.waves == W && h.pieces == NV && h.lanes == L)           \
  return f(std::integral_constant<int, V>(), std::integral_constant<int, W>(), std::integral_constant<int, NV>(), std::integral_constant<int, L>())
  AMQ_SHAPE(1, 1, 16);
  if constexpr (V > 1) {  // (rows of less than 16 bytes have pieces of one entry, and 16 lanes)
    constexpr int most = kPerLane / V;
    AMQ_SHAPE(1, 1, 32);
    AMQ_SHAPE(1, 1, 64);
    AMQ_SHAPE(1, 2, 64);
    if constexpr (most >= 4) AMQ_SHAPE(1, 4, 64);
    AMQ_SHAPE(4, 1, 64);
    AMQ_SHAPE(4, 2, 64);
    if constexpr (most >= 4) AMQ_SHAPE(4, 4, 64);
    AMQ_SHAPE(8, most, 64);
    AMQ_SHAPE(16, most, 64);
  }
#undef AMQ_SHAPE
  return hipErrorInvalidValue;
}

// Backward: pieces of 4 entries, one per lane where 16 waves have room for the row, else 2 or 4.  Four parameters, four sums and what is read take
// 27 registers per entry: with 8 entries a lane, as 16-byte loads would have, a compute unit had room for 8 waves.
constexpr int kGradPiece = 4;
template <typename F>
hipError_t with_grad_pieces(int n, F f) {
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, kGradPiece> v;
  const std::integral_constant<int, 16> short_row;
  const std::integral_constant<int, 32> half;
  const std::integral_constant<int, 64> whole;
  if (n < kGradPiece) return f(one, one, short_row);
  if (n <= 16 * kGradPiece) return f(v, one, short_row);
  if (n <= 32 * kGradPiece) return f(v, one, half);
  if (n <= 1024 * kGradPiece) return f(v, one, whole);
  if (n <= 2048 * kGradPiece) return f(v, std::integral_constant<int, 2>(), whole);
  return f(v, std::integral_constant<int, 4>(), whole);
}

// Rows that a grid of at most `most` workgroups takes at a time, spread evenly over its rounds.
int64_t even_blocks(int64_t tasks, int64_t most) {
  const int64_t rounds = (tasks + most - 1) / most;
  return (tasks + rounds - 1) / rounds;
}

constexpr int64_t kMostParts = 256;  // one workgroup per compute unit: more partial rows cost more than they hide


}  // namespace

int block_norm_grad_parts(int64_t rows, int) { return (int)(rows < kMostParts ? rows : kMostParts); }

hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
  return with_types(a.type, a.residual_type, a.param_type, [&](auto t, auto r, auto p) {
    using T = decltype(t);
    auto f = [&](auto v, auto w, auto nv, auto l) {
      constexpr int W = decltype(w)::value, L = decltype(l)::value, kThreads = W > 4 ? W * 64 : 256, kRows = kThreads / (L < 64 ? L : W * 64);
      const int64_t tasks = (a.rows + kRows - 1) / kRows;
      block_norm_kernel<T, decltype(r), decltype(p), decltype(v)::value, W, decltype(nv)::value, L>
          <<<dim3((unsigned)even_blocks(tasks, W >= 8 ? 512 : 1024)), dim3(kThreads), 0, s>>>(a);
      return hipGetLastError();
    };
    constexpr int V = kPer16<T>;
    return a.n < V ? with_shape<1>({1, 1, 16}, f) : with_shape<V>(shape_of<V>(a.rows, a.n), f);
  });
}

hipError_t launch_block_norm_grad(const BlockNormGradArgs& a0, hipStream_t s) {
  BlockNormGradArgs a = a0;
  const bool sums = a.dweight || a.dbias || a.dscale || a.dnext_weight || a.dnext_bias;
  if (!sums) a.part = nullptr;
  return with_types(a.type, a.residual_type, a.param_type, [&](auto t, auto r, auto p) {
    using T = decltype(t);
    using P = decltype(p);
    int64_t parts = 0;
    const hipError_t e = with_grad_pieces(a.n, [&](auto v, auto nv, auto l) {
      constexpr int V = decltype(v)::value, NV = decltype(nv)::value, L = decltype(l)::value, kPerWave = 64 / L;
      const int waves = (a.n + 64 * V * NV - 1) / (64 * V * NV);
      // few rows: one each (or a wave's) for as many compute units as there are
      const int64_t share = (a.rows + kMostParts * kPerWave - 1) / (kMostParts * kPerWave);
      const int groups = (share < 16 / waves ? (int)share : 16 / waves) * kPerWave;
      parts = even_blocks((a.rows + groups - 1) / groups, kMostParts);
      block_norm_grad_kernel<T, decltype(r), P, V, NV, L><<<dim3((unsigned)parts), dim3(L < 64 ? groups * L : groups * waves * 64), 0, s>>>(a, waves);
      return hipGetLastError();
    });
    if (e != hipSuccess || !sums) return e;
    block_norm_sum_kernel<P><<<dim3((unsigned)((a.n + 15) / 16)), dim3(1024), 0, s>>>(a, (int)parts);
    return hipGetLastError();
  });
}

}  // namespace amq
