// Matrix products on the 16-bit matrix cores for the training operators: result[m][n] = sum_k R[m][k] C[n][k], both
// operands with k running along their rows, fp32 accumulation, and an epilogue object that takes the finished values.
//
// An operand is one plane of bfloat16 or half values, or numbers of 22 bits as a high and a low half value: then
// high*high + high*low + low*high is summed, and what is left out is 2^-22 of a product at most.  Rows are padded with zeros
// to a multiple of 64 values and begin on 16 bytes; numbers of two halves lie in blocks of 32 high and 32 low parts.  So 128
// bytes of a row are one stage of the contraction in either case (64 or 32 values), there is no remainder, and every
// copy to LDS is 16 bytes per lane; rows past the operand's end are read as its last row and their results dropped.
//
// A workgroup of WR x WC waves owns BM x BN of the result and walks over the stages.  A stage goes from memory to LDS without
// passing registers (global_load_lds, 16 bytes a lane), into a ring of PLACES stages: up to that many are under way while one is
// multiplied.  The copy writes consecutive 16-byte pieces of LDS per lane, so the order that keeps
// the operand reads free of bank conflicts is made on the reading side of memory: piece p of row r holds piece p ^ f(r).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "amq_typed.h"

namespace amq {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct MatmulOperand {
  const void* p;
  int64_t ld, batch;  // strides in 16-bit values: rows, batch entries
  int rows;
};
// Where value k of a row of numbers of two halves has its high part; the low part follows 32 values on.
__host__ __device__ inline int64_t high_part(int64_t k) { return (k >> 5) * 64 + (k & 31); }
struct MatmulArgs {
  MatmulOperand r, c;
  int M, N;              // of the result
  int tiles_k;           // stages
  int nbm, nbn;          // tiles of the result
  int tiles_per_split;   // stages for each of gridDim.y
  int lower;             // symmetric result (r = c): only tiles with bm >= bn
};

// 16 x 16 values, 32 steps of k.  (The card's power limits large products: this form takes 8 KB from and to the registers for
// 16384 multiplications, 32 x 32 x 16 takes 10 KB.)
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

// Position, among the eight 16-byte pieces of a row in LDS, of piece `piece`.  The 64 banks serve 256 bytes a cycle, 16 lanes
// of an operand read: 16 rows in a row put the same piece on 16 different positions of 256 bytes, two rows to that many.
__device__ __forceinline__ int piece_at(int row, int piece) { return piece ^ ((row >> 1) & 7); }

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

// Hands a subtile of 32 x KW values (LDS, rows KW + 4 apart) to the epilogue, by one wave: four values along n per
// call, consecutive lanes along n; then, where the epilogue wants the transpose too, four values along m per call.
template <int KW, typename Epi>
__device__ __forceinline__ void finish_subtile(const float* t, const Epi& epi, int z, int m0, int n0, bool mirror, int lane) {
  constexpr int kStride = KW + 4, kPerRow = KW / 4;
#pragma unroll 1
  for (int i = 0; i < 32 * kPerRow; i += 64) {
    const int row = (i + lane) / kPerRow, col = (i + lane) % kPerRow * 4;
    epi.along_n(z, m0 + row, n0 + col, *reinterpret_cast<const f32x4*>(t + row * kStride + col));
  }
  if constexpr (Epi::kTransposed) {
    if (!mirror) return;
#pragma unroll 1
    for (int i = 0; i < 8 * KW; i += 64) {
      const int col = (i + lane) >> 3, row = ((i + lane) & 7) * 4;
      const float* q = t + row * kStride + col;
      epi.along_m(z, m0 + row, n0 + col, f32x4{q[0], q[kStride], q[2 * kStride], q[3 * kStride]});
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

template <typename E, int NP, int BM, int BN, int WR, int WC, int PLACES, typename Epi>
__global__ __launch_bounds__(WR * WC * 64, 2) void matmul_kernel(MatmulArgs g, Epi epi) {
  constexpr int kWaves = WR * WC, TM = BM / WR / 16, TN = BN / WC / 16;
  constexpr int JR = BM / 8 / kWaves, JC = BN / 8 / kWaves;  // copies of 8 rows that a wave makes per stage
  constexpr int kStage = (BM + BN) * 64;                     // 16-bit values
  constexpr int KW = TN * 16, kStride = KW + 4;
  static_assert(JR >= 1 && JC >= 1 && JR * 8 * kWaves == BM && JC * 8 * kWaves == BN, "copies");
  static_assert(TM % 2 == 0 && kWaves * 32 * kStride * 4 <= PLACES * kStage * 2, "the result's subtiles take the place of the operands");
  using Element = MatmulElement<E>;
  using v8 = typename Element::v8;
  __shared__ __align__(16) uint16_t lds[PLACES * kStage];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / WC, wc = wave % WC;
  int bm, bn;
  tile_of(blockIdx.x, gridDim.x, g, bm, bn);
  const int z = blockIdx.z;
  const int first = blockIdx.y * g.tiles_per_split;
  const int last = (first + g.tiles_per_split < g.tiles_k ? first + g.tiles_per_split : g.tiles_k) - 1;

  const uint16_t* pr = (const uint16_t*)g.r.p + z * g.r.batch + (int64_t)bm * BM * g.r.ld;
  const uint16_t* pc = (const uint16_t*)g.c.p + z * g.c.batch + (int64_t)bn * BN * g.c.ld;
  uint32_t off_r[JR], off_c[JC];  // bytes from the tile's first row
#pragma unroll
  for (int j = 0; j < JR; ++j) {
    const int row = (wave + j * kWaves) * 8 + (lane >> 3), left = g.r.rows - 1 - bm * BM;
    off_r[j] = (uint32_t)((row < left ? row : left) * g.r.ld + piece_at(row, lane & 7) * 8) * 2u;
  }
#pragma unroll
  for (int j = 0; j < JC; ++j) {
    const int row = (wave + j * kWaves) * 8 + (lane >> 3), left = g.c.rows - 1 - bn * BN;
    off_c[j] = (uint32_t)((row < left ? row : left) * g.c.ld + piece_at(row, lane & 7) * 8) * 2u;
  }
  // copy j of stage t of the contraction to its place in the ring; past the end the last stage again, so that as many copies
  // are under way at every wait
  auto copy = [&](int t, int j) __attribute__((always_inline)) {
    uint16_t* s = lds + (unsigned)(t - first) % PLACES * kStage;
    const int64_t at = (t < last ? t : last) * 64;
    if (j < JR) copy_to_lds((const char*)(pr + at), off_r[j], s + (wave + j * kWaves) * 512);
    else copy_to_lds((const char*)(pc + at), off_c[j - JR], s + BM * 64 + (wave + (j - JR) * kWaves) * 512);
  };
  constexpr int kCopies = JR + JC, kTiles = TM * TN;
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
    const uint16_t* s = lds + (unsigned)(t - first) % PLACES * kStage + (wr * (BM / WR) + i * 16) * 64;
    return *reinterpret_cast<const v8*>(s + (lane & 15) * 64 + piece_at(lane & 15, half * 4 + (lane >> 4)) * 8);
  };
  auto read_c = [&](int t, int half, int j) __attribute__((always_inline)) {
    const uint16_t* s = lds + (unsigned)(t - first) % PLACES * kStage + (BM + wc * KW + j * 16) * 64;
    return *reinterpret_cast<const v8*>(s + (lane & 15) * 64 + piece_at(lane & 15, half * 4 + (lane >> 4)) * 8);
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
#pragma unroll
  for (int i = 0; i < TM; i += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        *reinterpret_cast<f32x4*>(mine + (h * 16 + (lane & 15)) * kStride + j * 16 + (lane >> 4) * 4) = acc[i + h][j];
    __builtin_amdgcn_wave_barrier();
    finish_subtile<KW>(mine, epi, z, bm * BM + wr * (BM / WR) + i * 16, bn * BN + wc * KW, mirror, lane);
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- contractions split over k: partial results, added up in the order of the splits
struct PartialStore {
  static constexpr bool kTransposed = false;
  float* part;        // [batch][splits][M][ld]
  int64_t ld;         // a multiple of 4
  int M;
  __device__ __forceinline__ void along_n(int z, int m, int n, f32x4 v) const {
    if (m < M && n < ld)
      *reinterpret_cast<f32x4*>(part + (((int64_t)z * gridDim.y + blockIdx.y) * M + m) * ld + n) = v;
  }
  __device__ __forceinline__ void along_m(int, int, int, f32x4) const {}
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
  finish_subtile<32>(mine, epi, z, m0, n0, !lower || m0 / tile != n0 / tile, lane);
}

// ---- host side
inline int64_t pad64(int64_t n) { return (n + 63) & ~int64_t(63); }
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int stage_of(int planes) { return planes == 1 ? 64 : 32; }  // values of k

struct ProductPlan {
  int tile;             // of the result: tile x tile values per workgroup
  int splits, tiles_per_split;
  size_t part_bytes;    // of partial results (splits > 1)
};
ProductPlan plan_product(int64_t M, int64_t N, int64_t k, int planes, int64_t batch, bool lower);

template <typename E, int NP, int BM, int BN, int WR, int WC, int PLACES, typename Epi>
hipError_t launch_tiles(MatmulArgs g, const ProductPlan& p, int batch, const Epi& epi, hipStream_t s) {
  g.tiles_k /= stage_of(NP);  // (comes as k)
  g.tiles_per_split = p.tiles_per_split;
  g.nbm = (int)div_up(g.M, BM);
  g.nbn = (int)div_up(g.N, BN);
  const int64_t tiles = g.lower ? (int64_t)g.nbm * (g.nbm + 1) / 2 : (int64_t)g.nbm * g.nbn;
  matmul_kernel<E, NP, BM, BN, WR, WC, PLACES, Epi><<<dim3((unsigned)tiles, (unsigned)p.splits, (unsigned)batch), dim3(WR * WC * 64), 0, s>>>(g, epi);
  return hipGetLastError();
}

// The product of g (g.tiles_k holds k, a multiple of 64) with the tiles of `p`.
template <typename E, int NP, typename Epi>
hipError_t launch_product(const MatmulArgs& g, const ProductPlan& p, int batch, const Epi& epi, float* part, hipStream_t s) {
  if (p.splits > 1) {
    PartialStore store{part, (g.N + 3) & ~3, g.M};
    const hipError_t e = p.tile == 128 ? launch_tiles<E, NP, 128, 128, 2, 2, 2>(g, p, batch, store, s)
                                       : launch_tiles<E, NP, 64, 64, 2, 2, 3>(g, p, batch, store, s);
    if (e != hipSuccess) return e;
    matmul_sum_kernel<Epi><<<dim3((unsigned)div_up(pad64(g.N), 128), (unsigned)(pad64(g.M) / 32), (unsigned)batch), dim3(256), 0, s>>>(
        part, p.splits, g.M, store.ld, p.tile, g.lower, epi);
    return hipGetLastError();
  }
  if constexpr (NP == 1) {
    if (p.tile == 256) return launch_tiles<E, NP, 256, 256, 2, 4, 2>(g, p, batch, epi, s);
  }
  if (p.tile == 128) return launch_tiles<E, NP, 128, 128, 2, 2, 2>(g, p, batch, epi, s);
  return launch_tiles<E, NP, 64, 64, 2, 2, 3>(g, p, batch, epi, s);
}

}  // namespace amq
