// Matrix products on the 16-bit matrix cores for the training operators: result[m][n] = sum_k R[m][k] C[n][k], both
// operands with k running along their rows, fp32 accumulation, and an epilogue object that takes the finished values.
//
// An operand is one plane of bfloat16 or half values, or two planes of half values (high and low part of numbers of 22
// bits): then high*high + high*low + low*high is summed, and what is left out is 2^-22 of a product at most.  Rows are
// padded with zeros to a multiple of 64 values and begin on 16 bytes, so the contraction has no remainder and every copy to
// LDS is 16 bytes per lane; rows past the operand's end are read as its last row and their results dropped.
//
// A workgroup of WR x WC waves owns BM x BN of the result and walks over k in tiles of BK.  A tile goes from memory to LDS
// without passing registers (global_load_lds, 16 bytes a lane), the next one while the present one is multiplied (two
// buffers, one barrier per tile).  The copy writes consecutive 16-byte pieces of LDS per lane, so the order that keeps
// the operand reads free of bank conflicts is made on the reading side of memory: piece p of row r holds piece p ^ f(r).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "amq_typed.h"

namespace amq {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct MatmulOperand {
  const void* p;
  int64_t ld, plane, batch;  // strides in elements: rows, planes, batch entries
  int rows;
};
struct MatmulArgs {
  MatmulOperand r, c;
  int M, N;              // of the result
  int tiles_k;           // k / BK
  int nbm, nbn;          // tiles of the result
  int tiles_per_split;   // tiles of k for blockIdx.y
  int lower;             // symmetric result (r = c): only tiles with bm >= bn
};

template <typename E>
struct MatmulElement;
template <>
struct MatmulElement<bf16> {
  typedef bf16 v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ v16f mfma(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct MatmulElement<f16> {
  typedef f16 v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ v16f mfma(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// Position, among the 16-byte pieces of a row in LDS, of piece `chunk`.  Rows of 128 bytes (BK 64): eight rows in a row
// put the same piece on eight different positions; rows of 64 bytes (BK 32): two rows share 128 bytes.
template <int BK>
__device__ __forceinline__ int piece_at(int row, int chunk) {
  return BK == 64 ? chunk ^ (row & 7) : chunk ^ ((row >> 1) & 3);
}

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

template <typename E, int NP, int BM, int BN, int WR, int WC, typename Epi>
__global__ __launch_bounds__(WR * WC * 64) void matmul_kernel(MatmulArgs g, Epi epi) {
  constexpr int BK = NP == 1 ? 64 : 32;
  constexpr int kWaves = WR * WC, TM = BM / WR / 32, TN = BN / WC / 32;
  constexpr int kRowsPerCopy = 512 / BK;                           // rows that one wave copies at a time
  constexpr int JR = BM / kRowsPerCopy / kWaves, JC = BN / kRowsPerCopy / kWaves;
  constexpr int kBuffer = NP * (BM + BN) * BK;
  static_assert(JR >= 1 && JC >= 1 && JR * kRowsPerCopy * kWaves == BM && JC * kRowsPerCopy * kWaves == BN, "copies");
  static_assert(kWaves * 32 * (TN * 32 + 4) * 4 <= 2 * kBuffer * 2, "the result's subtiles take the place of the operands");
  using Element = MatmulElement<E>;
  using v8 = typename Element::v8;
  __shared__ __align__(16) uint16_t s0[kBuffer];
  __shared__ __align__(16) uint16_t s1[kBuffer];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / WC, wc = wave % WC;
  int bm, bn;
  tile_of(blockIdx.x, gridDim.x, g, bm, bn);
  const int z = blockIdx.z;
  const int first = blockIdx.y * g.tiles_per_split;
  const int last = first + g.tiles_per_split < g.tiles_k ? first + g.tiles_per_split : g.tiles_k;

  const uint16_t* pr = (const uint16_t*)g.r.p + z * g.r.batch + (int64_t)bm * BM * g.r.ld;
  const uint16_t* pc = (const uint16_t*)g.c.p + z * g.c.batch + (int64_t)bn * BN * g.c.ld;
  uint32_t off_r[JR], off_c[JC];  // bytes from the tile's first row; at most 256 rows of 2^31 / 256 bytes
  {
    const int in_copy = lane / (BK / 8), piece = lane % (BK / 8);
#pragma unroll
    for (int j = 0; j < JR; ++j) {
      const int row = (wave + j * kWaves) * kRowsPerCopy + in_copy;
      const int left = g.r.rows - 1 - bm * BM;
      off_r[j] = (uint32_t)((row < left ? row : left) * g.r.ld + piece_at<BK>(row, piece) * 8) * 2u;
    }
#pragma unroll
    for (int j = 0; j < JC; ++j) {
      const int row = (wave + j * kWaves) * kRowsPerCopy + in_copy;
      const int left = g.c.rows - 1 - bn * BN;
      off_c[j] = (uint32_t)((row < left ? row : left) * g.c.ld + piece_at<BK>(row, piece) * 8) * 2u;
    }
  }
  auto copy = [&](uint16_t* s, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const char* br = (const char*)(pr + p * g.r.plane + (int64_t)t * BK);
      const char* bc = (const char*)(pc + p * g.c.plane + (int64_t)t * BK);
#pragma unroll
      for (int j = 0; j < JR; ++j) copy_to_lds(br, off_r[j], s + p * (BM + BN) * BK + (wave + j * kWaves) * 512);
#pragma unroll
      for (int j = 0; j < JC; ++j) copy_to_lds(bc, off_c[j], s + (p * (BM + BN) + BM) * BK + (wave + j * kWaves) * 512);
    }
  };

  v16f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  auto multiply = [&](const uint16_t* s) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < BK / 16; ++ks) {
      const int at = (lane & 31) * BK + piece_at<BK>(lane & 31, ks * 2 + (lane >> 5)) * 8;
      v8 r[NP][TM], c[NP][TN];
#pragma unroll
      for (int p = 0; p < NP; ++p) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
          r[p][i] = *reinterpret_cast<const v8*>(s + (p * (BM + BN) + wr * (BM / WR) + i * 32) * BK + at);
#pragma unroll
        for (int j = 0; j < TN; ++j)
          c[p][j] = *reinterpret_cast<const v8*>(s + (p * (BM + BN) + BM + wc * (BN / WC) + j * 32) * BK + at);
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          // (the first operand's rows become the result's registers: four along n to a lane)
          if constexpr (NP == 2) {
            acc[i][j] = Element::mfma(c[1][j], r[0][i], acc[i][j]);
            acc[i][j] = Element::mfma(c[0][j], r[1][i], acc[i][j]);
          }
          acc[i][j] = Element::mfma(c[0][j], r[0][i], acc[i][j]);
        }
    }
  };
  // the copies that this wave issued have landed, and so have the other waves' after the barrier; nobody reads the other
  // buffer any more
  auto landed = [] __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  copy(s0, first);
  for (int t = first; t < last; t += 2) {
    landed();
    if (t + 1 < last) copy(s1, t + 1);
    multiply(s0);
    if (t + 1 < last) {
      landed();
      if (t + 2 < last) copy(s0, t + 2);
      multiply(s1);
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

  // the result, 32 rows at a time, through LDS (each wave its own part): stores of whole row pieces, and one copy of the
  // epilogue's code
  constexpr int KW = TN * 32, kStride = KW + 4;
  constexpr int kHalf = kWaves * 32 * kStride * 4 <= kBuffer * 2 ? kWaves : kWaves / 2;  // waves whose part lies in s0
  float* mine = wave < kHalf ? reinterpret_cast<float*>(s0) + wave * 32 * kStride : reinterpret_cast<float*>(s1) + (wave - kHalf) * 32 * kStride;
  const bool mirror = !g.lower || bm != bn;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(mine + (lane & 31) * kStride + j * 32 + q * 8 + (lane >> 5) * 4) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __builtin_amdgcn_wave_barrier();
    finish_subtile<KW>(mine, epi, z, bm * BM + wr * (BM / WR) + i * 32, bn * BN + wc * KW, mirror, lane);
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

struct ProductPlan {
  int tile;             // of the result: tile x tile values per workgroup
  int splits, tiles_per_split;
  size_t part_bytes;    // of partial results (splits > 1)
};
ProductPlan plan_product(int64_t M, int64_t N, int64_t k, int planes, int64_t batch, bool lower);

template <typename E, int NP, int BM, int BN, int WR, int WC, typename Epi>
hipError_t launch_tiles(MatmulArgs g, const ProductPlan& p, int batch, const Epi& epi, hipStream_t s) {
  constexpr int BK = NP == 1 ? 64 : 32;
  g.tiles_k = (int)(g.tiles_k / BK);  // (comes as k)
  g.tiles_per_split = p.tiles_per_split;
  g.nbm = (int)div_up(g.M, BM);
  g.nbn = (int)div_up(g.N, BN);
  const int64_t tiles = g.lower ? (int64_t)g.nbm * (g.nbm + 1) / 2 : (int64_t)g.nbm * g.nbn;
  matmul_kernel<E, NP, BM, BN, WR, WC, Epi><<<dim3((unsigned)tiles, (unsigned)p.splits, (unsigned)batch), dim3(WR * WC * 64), 0, s>>>(g, epi);
  return hipGetLastError();
}

// The product of g (g.tiles_k holds k, a multiple of 64) with the tiles of `p`.
template <typename E, int NP, typename Epi>
hipError_t launch_product(const MatmulArgs& g, const ProductPlan& p, int batch, const Epi& epi, float* part, hipStream_t s) {
  if (p.splits > 1) {
    PartialStore store{part, (g.N + 3) & ~3, g.M};
    const hipError_t e = p.tile == 128 ? launch_tiles<E, NP, 128, 128, 2, 2>(g, p, batch, store, s)
                                       : launch_tiles<E, NP, 64, 64, 2, 2>(g, p, batch, store, s);
    if (e != hipSuccess) return e;
    matmul_sum_kernel<Epi><<<dim3((unsigned)div_up(pad64(g.N), 128), (unsigned)(pad64(g.M) / 32), (unsigned)batch), dim3(256), 0, s>>>(
        part, p.splits, g.M, store.ld, p.tile, g.lower, epi);
    return hipGetLastError();
  }
  if (p.tile == 256) return launch_tiles<E, NP, 256, 256, 2, 4>(g, p, batch, epi, s);
  if (p.tile == 128) return launch_tiles<E, NP, 128, 128, 2, 2>(g, p, batch, epi, s);
  return launch_tiles<E, NP, 64, 64, 2, 2>(g, p, batch, epi, s);
}

}  // namespace amq
