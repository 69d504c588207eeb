// Matrix products on the 16-bit matrix cores for the training operators: result[m][n] = sum_k R[m][k] C[n][k], both
// operands with k running along their rows, fp32 accumulation, and an epilogue object that takes the finished values.
//
// An operand is bfloat16 or half values, or numbers of 22 bits as a high and a low half value: then
// high*high + high*low + low*high is summed, and what is left out is 2^-22 of a product at most.  k runs along an operand's rows
// in memory or down its columns.  Rows begin on 16 bytes and hold a multiple of 8 values or are padded with zeros to one; numbers of two halves lie in blocks of
// 32 high and 32 low parts, padded with zeros to a multiple of 64 numbers.  64 steps of k (of numbers of two halves 32) are one
// stage of the contraction; steps past the end are read as zeros, rows past the operand's end as its last ones, and
// their results dropped.
//
// A product may take two passes over k (TWO), the second over the low parts of one operand, which lie apart from its high ones; the
// other operand's values are read again.  That makes an operand of two parts times one of one, in half the rate.  (Known only at run time, the
// number of passes cost the products of one 2.5 to 3.5 %.)
//
// A workgroup of WR x WC waves owns BM x BN of the result and walks over the stages.  A stage goes from memory to LDS without
// passing registers (global_load_lds, 16 bytes a lane), into a ring of PLACES stages: up to that many are under way while one is
// multiplied.  The copy writes consecutive 16-byte pieces of LDS per lane, so the order that keeps
// the operand reads free of bank conflicts is made on the reading side of memory: piece p of row r holds piece p ^ f(r).
//
// Bounds and figures.  Large products: bfloat16 16384 x 4096 over 4096 with tiles of 256 432 us = 1270 TFLOP/s, where a library's product of 16384^3
// reaches 1560; numbers of two halves, tiles of 128 with two groups of waves, 1443 us = 1140 TFLOP/s of half products. Counters: the matrix
// cores are busy for 58 and 51 % of the cycles, at 2.1 GHz; the rest are waits for copies at the barriers, starts and epilogues. LDS has conflicts of 256 to 1024 cycles per tile
// (of symmetric results 1700) whatever its number of stages, 1 to 5 % of its use: those are the epilogue's, operand reads have none.  At the matrix cores' full rate tiles of 128 would
// take 64 bytes of operands per cycle, all that the cache above the L2 gives: 2048^3 24.6 us = 700 TFLOP/s.  Small products are bound by
// latency: a launch, a first load, the ring's start, the epilogue, 4 to 5 us together; so what has few tiles gets small ones, and groups of
// waves that share a tile's stages (64 x 1024 x 1024 5.3 us).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "amq_typed.h"

namespace amq {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct MatmulOperand {
  const void* p;
  int64_t ld, batch;  // strides in 16-bit values: rows of memory, batch entries
  int rows;           // of the operand
  int64_t second;     // of a product in two passes: how far from the first pass's values the second's lie (0: the same ones)
};
// Where value k of a row of numbers of two halves has its high part; the low part follows 32 values on.
__host__ __device__ inline int64_t high_part(int64_t k) { return (k >> 5) * 64 + (k & 31); }
struct MatmulArgs {
  MatmulOperand r, c;
  int M, N;              // of the result
  int k;                 // of the contraction
  int pass_k, tiles_k;   // stages of a pass, and in all
  int nbm, nbn;          // tiles of the result
  int tiles_per_split;   // stages for each of gridDim.y
  int lower;             // symmetric result (r = c): only tiles with bm >= bn
};

// 16 x 16 values, 32 steps of k.  (This form takes 8 KB from and to the registers for 16384 multiplications, 32 x 32 x 16 takes 10 KB.)
template <typename E>
struct MatmulElement;
template <>
struct MatmulElement<bf16> {
  typedef bf16 v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct MatmulElement<f16> {
  typedef f16 v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

__device__ const uint4 kZeros = {0, 0, 0, 0};

// Tile of the result for workgroup `id` of `count`.  Workgroups are dealt to the 8 dies in turn: each die gets a run of
// consecutive tiles, in groups of 8 tile rows, so that what its L2 holds of both operands is used again.
__device__ __forceinline__ void tile_of(int id, int count, const MatmulArgs& g, int& bm, int& bn) {
  const int per = count >> 3, rest = count & 7, die = id & 7;
  id = die * per + (die < rest ? die : rest) + (id >> 3);
  if (g.lower) {
    int row = (int)((sqrtf(8.0f * (float)id + 1.0f) - 1.0f) * 0.5f);
    while ((row + 1) * (row + 2) / 2 <= id) ++row;
    while (row * (row + 1) / 2 > id) --row;
    bm = row;
    bn = id - row * (row + 1) / 2;
    return;
  }
  constexpr int kGroup = 8;
  const int in_group = kGroup * g.nbn, first = id / in_group * kGroup;
  const int rows = g.nbm - first < kGroup ? g.nbm - first : kGroup;
  const int at = id % in_group;
  bm = first + at % rows;
  bn = at / rows;
}

// An epilogue takes four values along n at a time, in three parts, so that what it reads is under way before it is needed:
//   Column column(z, n)             what goes with columns n .. n + 3, once per wave (a lane keeps its columns)
//   Extra fetch(z, m, n)            what goes with the values, for several rows ahead
//   put(z, m, n, v, column, extra)  the values
// With kTransposed it gets the transpose of tiles off the diagonal too, by fetch and put with m and n exchanged.
//
// Hands over a subtile of 32 x KW values.  They lie in LDS, rows KW + 4 apart, as the sum of KG parts `apart` values apart; KG
// waves share the subtile, this one is number `share`.
template <int KW>
__device__ __forceinline__ int column_of(int lane) {
  return lane % (KW / 4) * 4;
}
template <int KW, int KG, typename Epi>
__device__ __forceinline__ void finish_subtile(const float* t, int apart, int share, const Epi& epi, const typename Epi::Column& column, int z, int m0,
                                               int n0, bool mirror, int lane) {
  constexpr int kStride = KW + 4, kPerRow = KW / 4, kRows = 64 / kPerRow, kAll = (32 + kRows - 1) / kRows;  // calls of a whole wave
  constexpr bool kWhole = 64 % kPerRow == 0;  // else the last lanes are left out, and rows past the last
  constexpr int kCalls = kAll > KG ? kAll / KG : 1, kAhead = kCalls < 4 ? kCalls : 4;
  static_assert(kWhole ? kAll % KG == 0 || KG % kAll == 0 : KG == 1, "whole calls");
  const int col = column_of<KW>(lane), line = lane / kPerRow;
  auto row_of = [&](int call) __attribute__((always_inline)) { return call * kRows + line; };
  auto counts = [&](int row) __attribute__((always_inline)) { return kWhole || (line < kRows && row < 32); };
#pragma unroll 1
  for (int c = 0; c < kCalls && (KG <= kAll || share < kAll); c += kAhead) {
    typename Epi::Extra extra[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) extra[u] = epi.fetch(z, m0 + row_of((c + u) * KG + share), n0 + col);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int row = row_of((c + u) * KG + share);
      if (!counts(row)) continue;
      const float* q = t + row * kStride + col;
      f32x4 v = *reinterpret_cast<const f32x4*>(q);
#pragma unroll
      for (int g = 1; g < KG; ++g) v += *reinterpret_cast<const f32x4*>(q + g * apart);
      epi.put(z, m0 + row, n0 + col, v, column, extra[u]);
    }
  }
  if constexpr (Epi::kTransposed) {
    if (!mirror) return;
    constexpr int kTurned = 8 * KW / 64;  // pieces of 64 lanes
    for (int c = share; c < kTurned; c += KG) {
      const int n = (c * 64 + lane) >> 3, m = ((c * 64 + lane) & 7) * 4;
      const typename Epi::Extra extra = epi.fetch(z, n0 + n, m0 + m);
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int g = 0; g < KG; ++g) {
        const float* q = t + g * apart + m * kStride + n;
        v += f32x4{q[0], q[kStride], q[2 * kStride], q[3 * kStride]};
      }
      epi.put(z, n0 + n, m0 + m, v, typename Epi::Column{}, extra);
    }
  }
}

// Copies 16 bytes per lane from `base` + the lane's offset to LDS, lane by lane from `to` on, which all lanes share.  Written
// out, since behind the builtin the compiler lets every read of LDS wait for all copies under way, the other buffer's
// too.  The instruction has no result in registers; who reads LDS waits by vmcnt and a barrier.  (m0
// is the compiler's to reserve, and nothing else in these kernels needs it.)
__device__ __forceinline__ void copy_to_lds(const char* base, uint32_t offset, uint16_t* to) {
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)to;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(base));
}
// The same from an address per lane.
__device__ __forceinline__ void copy_to_lds(const char* from, uint16_t* to) {
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)to;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from));
}

// One operand of a workgroup's tile: its copies to LDS, and its fragments for the matrix cores (16 rows, 32 steps of k: eight
// values per lane, row lane % 16, steps (lane / 16) * 8 on).
//
// Rows (k runs along the rows of memory): LDS holds B rows of 128 bytes, one stage of each.
// Columns (k runs down the columns of memory): LDS holds one stage's rows of memory, B operand rows wide.  A fragment is
// gathered by two transposing reads: 16 lanes read 4 steps of k of 16 operand rows, and get them turned.  Its 32 lanes a cycle
// cover 8 steps of k; those are given 8 different 32-byte parts of the 64 banks.
template <typename E, int NP, bool TWO, int B, int kWaves, bool COLUMNS>
struct Side {
  using v8 = typename MatmulElement<E>::v8;
  typedef short v4s __attribute__((ext_vector_type(4)));
  static constexpr int kCopies = B / 8 / kWaves;         // of 1 KB that a wave makes per stage
  static constexpr int kLine = COLUMNS ? B * NP * 2 : 128;  // bytes of a row in LDS
  static constexpr int kLanes = kLine / 16;              // lanes per row of a copy
  static constexpr int kSteps = NP == 1 ? 64 : 32;       // of k in a stage
  static_assert(kCopies * 8 * kWaves == B, "copies");

  // Rows of memory that the copies of a wave are apart.  Down columns every 16 rows have the same offsets within their rows, so
  // that one offset serves several copies (rows may end inside a tile and need one each).
  static constexpr int kApart = kWaves * 64 / kLanes;
  static constexpr bool kWhole = 64 % kLanes == 0;  // a copy has whole rows
  static constexpr int kOffsets = COLUMNS && kWhole ? (kApart >= 16 ? 1 : 16 / kApart) : kCopies;
  static_assert(!kWhole || kApart >= 16 || 16 % kApart == 0, "copies and the order of pieces");
  static_assert(kWhole || kLine % 256 == 128, "order of pieces");

  const char* base;    // of the tile, uniform
  int64_t stage;       // bytes from one stage to the next
  int64_t line;        // bytes from one row of memory to the next
  int64_t second;      // bytes from the first pass's values to the second's
  uint32_t off[kOffsets];
  int k, pass_k, lane, wave;

  static __device__ __forceinline__ int swizzle(int row) {  // of 16-byte pieces
    if (!COLUMNS) return (row >> 1) & 7;
    if (kLine == 64) return ((row >> 3) & 1) << 1;
    // (rows an odd multiple of 128 bytes apart: every other one begins in the other half of the banks)
    if (kLine % 256 == 128) return (((row >> 1) & 1) | ((row >> 2) & 2)) << 1;
    return ((row & 3) | ((row >> 1) & 4)) << 1;
  }
  __device__ __forceinline__ Side(const MatmulOperand& o, const MatmulArgs& g, int z, int first_row, int lane_, int wave_)
      : k(g.k), pass_k(g.pass_k), lane(lane_), wave(wave_) {
    const uint16_t* p = (const uint16_t*)o.p + z * o.batch;
    line = o.ld * 2;
    second = o.second * 2;
    if constexpr (COLUMNS) {
      base = (const char*)(p + (int64_t)first_row * NP);
      stage = o.ld * kSteps * 2;
    } else {
      base = (const char*)(p + first_row * o.ld);
      stage = 128;
    }
#pragma unroll
    for (int j = 0; j < kOffsets; ++j) {
      const int row = row_of(j), piece = piece_of(j) ^ swizzle(row);
      if constexpr (COLUMNS) {
        // past the operand's last rows those again (their number is a multiple of 8)
        const int left = (o.rows - first_row) * NP - 8, at = piece * 8;
        off[j] = (uint32_t)(row * o.ld + (at < left ? at : left)) * 2u;
      } else {
        const int left = o.rows - 1 - first_row;
        off[j] = (uint32_t)((row < left ? row : left) * o.ld + piece * 8) * 2u;
      }
    }
  }
  // The lane's row of copy j in LDS, and its place there.
  __device__ __forceinline__ int row_of(int j) const {
    return kWhole ? (wave + j * kWaves) * (64 / kLanes) + lane / kLanes : ((wave + j * kWaves) * 64 + lane) / kLanes;
  }
  __device__ __forceinline__ int piece_of(int j) const { return kWhole ? lane % kLanes : ((wave + j * kWaves) * 64 + lane) % kLanes; }
  // Copy j of stage t.  Steps of k past the end are zeros (along rows: to the next multiple of 8 what lies there).
  __device__ __forceinline__ void copy(uint16_t* s, int t, int j) const {
    const char* start = base;
    if (TWO && t >= pass_k) {
      t -= pass_k;
      start += second;
    }
    const char* from = start + t * stage + (COLUMNS ? j / kOffsets * (kOffsets * kApart) * line : 0);
    const uint32_t at = off[j % kOffsets];
    uint16_t* to = s + (wave + j * kWaves) * 512;
    if ((t + 1) * kSteps > k) {
      const int piece = piece_of(j) ^ swizzle(row_of(j));
      const int step = t * kSteps + (COLUMNS ? row_of(j) : (NP == 1 ? piece : piece & 3) * 8);
      copy_to_lds(step < k ? from + at : (const char*)&kZeros, to);
    } else {
      copy_to_lds(from, at, to);
    }
  }
  // Fragment of 16 rows from row0 + 16 i on (row0: of the wave): half `half` of the stage, or of its numbers.
  __device__ __forceinline__ v8 read(const uint16_t* s, int row0, int i, int half) const {
    if constexpr (!COLUMNS) {
      return *reinterpret_cast<const v8*>(s + (row0 + i * 16 + (lane & 15)) * 64 + ((half * 4 + (lane >> 4)) ^ swizzle(lane & 15)) * 8);
    } else {
      // The 32-byte part within a row: row0 takes the high bits, the fragment's number the low ones.  (The number comes in last, so
      // that an address is one operation on the place's and not a register held for each fragment.)
      const int step = (lane >> 4) * 8 + ((lane & 15) >> 2);
      const int part = NP == 1 ? i : (i >> 1) * 4 + half * 2 + (i & 1);
      const uint32_t place = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint16_t*)s;
      uint32_t at;
      if constexpr (kWhole) {
        at = (place + (uint32_t)(step * kLine + ((row0 * NP / 8) ^ swizzle(step)) * 16 + (lane & 3) * 8)) ^ (uint32_t)(part * 32);
      } else {  // row0 is a multiple of 16 only: the order goes by 128 bytes
        static_assert(NP == 1, "tiles of numbers of two halves are powers of two");
        const int bytes = (row0 + i * 16) * 2;
        at = ((place + (uint32_t)(step * kLine + swizzle(step) * 16 + (lane & 3) * 8)) ^ (uint32_t)(bytes & 127)) + (uint32_t)(bytes & ~127);
      }
      const auto* q = (__attribute__((address_space(3))) const char*)(uintptr_t)at + (NP == 1 ? half * 32 * kLine : 0);
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)q);
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(q + 4 * kLine));
      return __builtin_bit_cast(v8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// KG groups of WR x WC waves, each with its share of the stages and a ring of its own; their results are added up at the end.
// `id` of `count`: the tile; `split`: the part of the stages; `z`: the batch entry.
template <int BM, int BN, int KG, int PLACES>
constexpr int kTileLds = KG * PLACES * (BM + BN) * 64;  // 16-bit values
template <typename E, int NP, bool TWO, bool RC, bool CC, int BM, int BN, int WR, int WC, int KG, int PLACES, typename Epi>
__device__ __forceinline__ void matmul_tile(uint16_t* all_lds, const MatmulArgs& g, const Epi& epi, int id, int count, int split, int z) {
  constexpr int kWaves = WR * WC, TM = BM / WR / 16, TN = BN / WC / 16;
  constexpr int kStage = (BM + BN) * 64;  // 16-bit values
  constexpr int KW = TN * 16, kStride = KW + 4;
  static_assert(TM % 2 == 0 && kWaves * 32 * kStride * 4 <= PLACES * kStage * 2, "the result's subtiles take the place of the operands");
  using Element = MatmulElement<E>;
  using v8 = typename Element::v8;
  using R = Side<E, NP, TWO, BM, kWaves, RC>;
  using C = Side<E, NP, TWO, BN, kWaves, CC>;

  const int lane = threadIdx.x & 63;
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kWaves;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - group * kWaves;
  uint16_t* lds = all_lds + group * (PLACES * kStage);
  const int wr = wave / WC, wc = wave % WC;
  int bm, bn;
  tile_of(id, count, g, bm, bn);
  // (the groups take as many stages each, so that they meet at every barrier; what lies past the end counts as zeros)
  int first = split * g.tiles_per_split;
  int last = (first + g.tiles_per_split < g.tiles_k ? first + g.tiles_per_split : g.tiles_k) - 1;
  if constexpr (KG > 1) {
    const int each = (last - first + KG) / KG;
    first += group * each;
    last = first + each - 1;
  }
  const R r(g.r, g, z, bm * BM, lane, wave);
  const C c(g.c, g, z, bn * BN, lane, wave);
  // copy j of stage t of the contraction to its place in the ring; past the end the last stage again, so that as many copies
  // are under way at every wait
  auto copy = [&](int t, int j) __attribute__((always_inline)) {
    uint16_t* s = lds + (unsigned)(t - first) % PLACES * kStage;
    const int at = t < last ? t : last;
    if (j < R::kCopies) r.copy(s, at, j);
    else c.copy(s + BM * 64, at, j - R::kCopies);
  };
  constexpr int kCopies = R::kCopies + C::kCopies, kTiles = TM * TN;
  // This wave's reads have returned; of the copies that it issued all but the newest `LEFT` stages' have landed.  After the
  // barrier that holds for the other waves too.
  auto together = [](auto left) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0), so that the compiler knows of it
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(decltype(left)::value * kCopies) : "memory");
  };
  auto fence = [] __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // Operands of 32 steps of k: one half of a stage (of numbers of two halves, its high or its low parts).
  struct Fragments {
    v8 r[TM], c[TN];
  };
  auto read_r = [&](int t, int half, int i) __attribute__((always_inline)) {
    return r.read(lds + (unsigned)(t - first) % PLACES * kStage, wr * (BM / WR), i, half);
  };
  auto read_c = [&](int t, int half, int j) __attribute__((always_inline)) {
    return c.read(lds + (unsigned)(t - first) % PLACES * kStage + BM * 64, wc * KW, j, half);
  };
  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // One stage is multiplied in two steps: `a` of its first half and `b` of its second; of numbers of two halves, high by high
  // and the two mixed products.  Both are read from LDS during the second step of the stage before, rows each behind their
  // last products, so that a place of the ring is in use for one step and its next stage under way for the other 2 PLACES - 1.  A wave issues in order, and the matrix cores are busy for
  // 16 cycles with each product: what is asked for between products costs them nothing.
  Fragments a, b;
  constexpr int kMeet = kTiles / 4 > 0 ? kTiles / 4 - 1 : 0;  // the product behind which the reads of the stage have returned
  auto first_step = [&](int t) __attribute__((always_inline)) {
    int copied = 0;
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      const int i = x / TN, j = x % TN;
      // (the first operand's rows become the result's registers: four along n to a lane)
      acc[i][j] = Element::mfma(a.c[j], a.r[i], acc[i][j]);
      if (x == kMeet) {
        __builtin_amdgcn_sched_barrier(0);
        together(std::integral_constant<int, PLACES - 1>());  // (for the reads: every wave has those of stage t)
      }
      if (x >= kMeet && copied < kCopies) {
#pragma unroll
        for (; copied < kCopies && copied * (kTiles - kMeet) < (x - kMeet + 1) * kCopies; ++copied) copy(t + PLACES, copied);
        fence();
      }
    }
  };
  auto second_step = [&](int t) __attribute__((always_inline)) {
    together(std::integral_constant<int, PLACES - 1>());  // stage t + 1 has landed
    int reads = 0;
    v8 next_c[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        if constexpr (NP == 1) {
          acc[i][j] = Element::mfma(b.c[j], b.r[i], acc[i][j]);
        } else {
          acc[i][j] = Element::mfma(b.c[j], a.r[i], acc[i][j]);
          acc[i][j] = Element::mfma(a.c[j], b.r[i], acc[i][j]);
        }
        __builtin_amdgcn_sched_barrier(0);
        constexpr int kEarly = NP == 1 ? TM + TN : TN;  // (rows of a are free from the start only where they are not used here)
#pragma unroll
        for (; reads < kEarly && reads * (kTiles / 2) < (i * TN + j + 1) * kEarly; ++reads) {
          if (reads < TN) next_c[reads] = read_c(t + 1, 0, reads);
          else a.r[reads - TN] = read_r(t + 1, 0, reads - TN);
        }
        fence();
      }
      if constexpr (NP == 2) a.r[i] = read_r(t + 1, 0, i);
      b.r[i] = read_r(t + 1, 1, i);
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) b.c[j] = read_c(t + 1, 1, j), a.c[j] = next_c[j];
    fence();
  };

#pragma unroll
  for (int t = 0; t < PLACES; ++t)
#pragma unroll
    for (int j = 0; j < kCopies; ++j) copy(first + t, j);
  together(std::integral_constant<int, PLACES - 1>());
#pragma unroll
  for (int i = 0; i < TM; ++i) a.r[i] = read_r(first, 0, i), b.r[i] = read_r(first, 1, i);
#pragma unroll
  for (int j = 0; j < TN; ++j) a.c[j] = read_c(first, 0, j), b.c[j] = read_c(first, 1, j);
  for (int t = first; t <= last; ++t) {
    first_step(t);
    second_step(t);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  // the result, 32 rows at a time, through LDS (each wave its own part): stores of whole row pieces, and one copy of the
  // epilogue's code
  float* mine = reinterpret_cast<float*>(lds) + wave * 32 * kStride;
  const bool mirror = !g.lower || bm != bn;
  const int n0 = bn * BN + wc * KW;
  const typename Epi::Column column = epi.column(z, n0 + column_of<KW>(lane));
#pragma unroll
  for (int i = 0; i < TM; i += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        *reinterpret_cast<f32x4*>(mine + (h * 16 + (lane & 15)) * kStride + j * 16 + (lane >> 4) * 4) = acc[i + h][j];
    if constexpr (KG > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    finish_subtile<KW, KG>(reinterpret_cast<float*>(all_lds) + wave * 32 * kStride, PLACES * kStage / 2, group, epi, column, z,
                           bm * BM + wr * (BM / WR) + i * 16, n0, mirror, lane);
    if constexpr (KG > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
  }
}

template <typename E, int NP, bool TWO, bool RC, bool CC, int BM, int BN, int WR, int WC, int KG, int PLACES, typename Epi>
__global__ __launch_bounds__(KG * WR * WC * 64, KG * WR * WC >= 16 ? 4 : 2) void matmul_kernel(MatmulArgs g, Epi epi) {
  __shared__ __align__(256) uint16_t lds[kTileLds<BM, BN, KG, PLACES>];
  matmul_tile<E, NP, TWO, RC, CC, BM, BN, WR, WC, KG, PLACES>(lds, g, epi, blockIdx.x, gridDim.x, blockIdx.y, blockIdx.z);
}
// Two products that do not depend on each other, d W and d^T x, in one launch: the tiles of the one with the longer contraction come
// first, so that what is left at the end is small. One launch instead of two took the bf16 backward of 700 x 650 by 1300 from 29.5 us
// to 24.8 and of 20 x 100 by 100 from 14.8 to 10.3 (d of one value); plan_pair() leaves the two apart where that is estimated to be faster.
template <typename E, int NP, bool TWO, int BM, int BN, int WR, int WC, int KG, int PLACES, typename Epi>
__global__ __launch_bounds__(KG * WR * WC * 64, KG * WR * WC >= 16 ? 4 : 2) void matmul_pair_kernel(MatmulArgs g, Epi epi, MatmulArgs g2, Epi epi2) {
  __shared__ __align__(256) uint16_t lds[kTileLds<BM, BN, KG, PLACES>];
  const int tiles = g.nbm * g.nbn, tiles2 = g2.nbm * g2.nbn;
  const bool ahead = g.k > g2.k;
  const int id = blockIdx.x, i = ahead ? id : id - tiles2, i2 = ahead ? id - tiles : id;
  if (i2 >= 0 && i2 < tiles2) matmul_tile<E, NP, TWO, true, true, BM, BN, WR, WC, KG, PLACES>(lds, g2, epi2, i2, tiles2, 0, 0);
  else matmul_tile<E, NP, TWO, false, true, BM, BN, WR, WC, KG, PLACES>(lds, g, epi, i, tiles, 0, 0);
}

// ---- contractions split over k: partial results, added up in the order of the splits
struct PartialStore {
  static constexpr bool kTransposed = false;
  float* part;        // [batch][splits][M][ld]
  int64_t ld;         // a multiple of 4
  int M;
  struct Column {};
  struct Extra {};
  __device__ __forceinline__ Column column(int, int) const { return {}; }
  __device__ __forceinline__ Extra fetch(int, int, int) const { return {}; }
  __device__ __forceinline__ void put(int z, int m, int n, f32x4 v, const Column&, const Extra&) const {
    if (m < M && n < ld)
      *reinterpret_cast<f32x4*>(part + (((int64_t)z * gridDim.y + blockIdx.y) * M + m) * ld + n) = v;
  }
};

// One wave per 32 x 32 values, up to the next multiple of 64 in both directions (operands of further products want zeros
// there).  `lower`: only the values of tiles of `tile` x `tile` with bm >= bn exist.
template <typename Epi>
__global__ __launch_bounds__(256) void matmul_sum_kernel(const float* part, int splits, int M, int64_t ld, int tile, int lower, Epi epi) {
  __shared__ __align__(16) float t[4][32 * 36];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = blockIdx.z;
  const int m0 = blockIdx.y * 32, n0 = (blockIdx.x * 4 + wave) * 32;
  if (n0 >= ((ld + 63) & ~int64_t(63))) return;
  if (lower && m0 / tile < n0 / tile) return;
  float* mine = t[wave];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + (lane >> 3), col = (lane & 7) * 4, m = m0 + row, n = n0 + col;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (m < M && n < ld) {
      const float* p = part + ((int64_t)z * splits * M + m) * ld + n;
#pragma unroll 4
      for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(p + (int64_t)s * M * ld);
    }
    *reinterpret_cast<f32x4*>(mine + row * 36 + col) = v;
  }
  __builtin_amdgcn_wave_barrier();
  finish_subtile<32, 1>(mine, 0, 0, epi, epi.column(z, n0 + column_of<32>(lane)), z, m0, n0, !lower || m0 / tile != n0 / tile, lane);
}

// ---- host side
inline int64_t pad64(int64_t n) { return (n + 63) & ~int64_t(63); }
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int stage_of(int planes) { return planes == 1 ? 64 : 32; }  // values of k

struct ProductPlan {
  int tile;             // of the result: tile x tile values per workgroup
  int groups;           // of waves that share a workgroup's stages
  int splits, tiles_per_split;
  size_t part_bytes;    // of partial results (splits > 1)
  double us;            // estimated time
};
// Stages of g's contraction, all passes.
inline void set_stages(MatmulArgs& g, int planes, bool two) {
  g.pass_k = (int)div_up(g.k, stage_of(planes));
  g.tiles_k = two ? 2 * g.pass_k : g.pass_k;
}

ProductPlan plan_product(int64_t M, int64_t N, int64_t k, int planes, int64_t batch, bool lower, int passes = 1);
// The best form for two products in one launch (M x N over k, M2 x N2 over k2).
ProductPlan plan_pair(int64_t M, int64_t N, int64_t k, int64_t M2, int64_t N2, int64_t k2, int planes, int passes);

template <typename E, int NP, bool TWO, bool RC, bool CC, int BM, int BN, int WR, int WC, int KG, int PLACES, typename Epi>
hipError_t launch_tiles(MatmulArgs g, const ProductPlan& p, int batch, const Epi& epi, hipStream_t s) {
  set_stages(g, NP, TWO);
  g.tiles_per_split = p.tiles_per_split;
  g.nbm = (int)div_up(g.M, BM);
  g.nbn = (int)div_up(g.N, BN);
  const int64_t tiles = g.lower ? (int64_t)g.nbm * (g.nbm + 1) / 2 : (int64_t)g.nbm * g.nbn;
  matmul_kernel<E, NP, TWO, RC, CC, BM, BN, WR, WC, KG, PLACES, Epi><<<dim3((unsigned)tiles, (unsigned)p.splits, (unsigned)batch), dim3(KG * WR * WC * 64), 0, s>>>(g, epi);
  return hipGetLastError();
}

// The product of g with the tiles of `p`; RC, CC: whether k runs down the columns of the operand; TWO: in two passes.
template <typename E, int NP, bool RC, bool CC, bool TWO = false, typename Epi>
hipError_t launch_product(const MatmulArgs& g, const ProductPlan& p, int batch, const Epi& epi, float* part, hipStream_t s) {
  auto run = [&](const auto& store) {
    if constexpr (NP == 1)
      if (p.tile == 256) return launch_tiles<E, NP, TWO, RC, CC, 256, 256, 2, 4, 1, 2>(g, p, batch, store, s);
    // (8 waves: 253 tiles over 16384 287 us; with 4 that hold twice the values each 416, with 12 or a ring of three places the same)
    if constexpr (NP == 1)
      if (p.tile == 192) return launch_tiles<E, NP, TWO, RC, CC, 192, 192, 2, 4, 1, 2>(g, p, batch, store, s);
    if (p.tile == 128 && p.groups == 2) return launch_tiles<E, NP, TWO, RC, CC, 128, 128, 2, 2, 2, 2>(g, p, batch, store, s);
    if (p.tile == 128) return launch_tiles<E, NP, TWO, RC, CC, 128, 128, 2, 2, 1, 2>(g, p, batch, store, s);
    if (p.tile == 32) return launch_tiles<E, NP, TWO, RC, CC, 32, 32, 1, 1, 8, 2>(g, p, batch, store, s);
    if (p.groups == 4) return launch_tiles<E, NP, TWO, RC, CC, 64, 64, 2, 2, 4, 2>(g, p, batch, store, s);
    return launch_tiles<E, NP, TWO, RC, CC, 64, 64, 2, 2, 1, 3>(g, p, batch, store, s);
  };
  if (p.splits == 1) return run(epi);
  const PartialStore store{part, (g.N + 3) & ~3, g.M};
  const hipError_t e = run(store);
  if (e != hipSuccess) return e;
  matmul_sum_kernel<Epi><<<dim3((unsigned)div_up(pad64(g.N), 128), (unsigned)(pad64(g.M) / 32), (unsigned)batch), dim3(256), 0, s>>>(
      part, p.splits, g.M, store.ld, p.tile, g.lower, epi);
  return hipGetLastError();
}

template <typename E, int NP, bool TWO, int BM, int BN, int WR, int WC, int KG, int PLACES, typename Epi>
hipError_t launch_pair_tiles(MatmulArgs g, const Epi& epi, MatmulArgs g2, const Epi& epi2, hipStream_t s) {
  int64_t tiles[2];
  MatmulArgs* both[2] = {&g, &g2};
  for (int i = 0; i < 2; ++i) {
    MatmulArgs& a = *both[i];
    set_stages(a, NP, TWO);
    a.tiles_per_split = a.tiles_k;
    a.nbm = (int)div_up(a.M, BM);
    a.nbn = (int)div_up(a.N, BN);
    tiles[i] = (int64_t)a.nbm * a.nbn;
  }
  matmul_pair_kernel<E, NP, TWO, BM, BN, WR, WC, KG, PLACES, Epi>
      <<<dim3((unsigned)(tiles[0] + tiles[1])), dim3(KG * WR * WC * 64), 0, s>>>(g, epi, g2, epi2);
  return hipGetLastError();
}
template <typename E, int NP, bool TWO, typename Epi>
hipError_t launch_pair(const MatmulArgs& g, const Epi& epi, const MatmulArgs& g2, const Epi& epi2, const ProductPlan& p, hipStream_t s) {
  if (p.tile == 128 && p.groups == 2) return launch_pair_tiles<E, NP, TWO, 128, 128, 2, 2, 2, 2>(g, epi, g2, epi2, s);
  if (p.tile == 128) return launch_pair_tiles<E, NP, TWO, 128, 128, 2, 2, 1, 2>(g, epi, g2, epi2, s);
  if (p.tile == 32) return launch_pair_tiles<E, NP, TWO, 32, 32, 1, 1, 8, 2>(g, epi, g2, epi2, s);
  if (p.groups == 4) return launch_pair_tiles<E, NP, TWO, 64, 64, 2, 2, 4, 2>(g, epi, g2, epi2, s);
  return launch_pair_tiles<E, NP, TWO, 64, 64, 2, 2, 1, 3>(g, epi, g2, epi2, s);
}

}  // namespace amq
