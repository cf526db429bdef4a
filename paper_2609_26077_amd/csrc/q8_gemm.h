// The matrix-core product of the 8-bit linear layer: C = A B^T over rows that
// are contiguous along the contracted axis, int8 (int32 sums) or bfloat16
// (fp32 sums).
//
// Both element types share one data path.  A step is 128 bytes of every row of
// the tile (128 int8 or 64 bfloat16 positions) in LDS, two slots, filled by
// global_load_lds one step ahead; a matrix instruction takes 16 bytes a lane
// of 32 rows of each side (v_mfma_i32_32x32x32_i8, v_mfma_f32_32x32x16_bf16),
// so a step is four instructions per 32 x 32 tile.  Which positions a lane's
// 16 bytes are does not matter as long as both sides agree: instruction t of a
// step takes chunk 2 t + h of the row in lane half h.
//
// LDS rows are 128 bytes; 16-byte chunk c of row r sits at chunk
// c ^ (r & 7) ^ ((r >> 3) & 1), so that the lanes of a fragment read fall on
// distinct banks.  A transfer moves eight rows (lane l: row l / 8, chunk
// position l % 8), the swizzle being applied to the address that the lane
// reads from, so each row's 128 bytes are one full line of HBM or L2.
//
// The instruction's first operand is B and its second is A: a lane then holds
// one row of C and, per four accumulators, four consecutive columns of it.
#pragma once

#include <hip/hip_runtime.h>

#include "lds_dma.h"
#include "q8.h"
#include "q8_types.h"

namespace fmm {
namespace q8 {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int kStep = 128;   // bytes of a row per step

struct Int8 {
  typedef v4i frag;
  typedef v16i acc;
  static __device__ __forceinline__ acc mma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
  }
};
struct Bf16 {
  typedef v8bf frag;
  typedef v16f acc;
  static __device__ __forceinline__ acc mma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

// Tile of TM x TN outputs, WM x WN waves.
template <int TM_, int TN_, int WM_, int WN_>
struct Tile {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int MI = TM / WM / 32, NI = TN / WN / 32;   // 32 x 32 tiles of a wave
  static constexpr int kSlot = (TM + TN) * kStep;
  static constexpr int JA = TM / 8 / kWaves, JB = TN / 8 / kWaves;   // transfers of a wave per step and side
  static_assert(MI * 32 * WM == TM && NI * 32 * WN == TN && JA * 8 * kWaves == TM && JB * 8 * kWaves == TN, "tile");
};
typedef Tile<256, 256, 2, 4> Tile256;
typedef Tile<128, 128, 2, 2> Tile128;
typedef Tile<64, 64, 2, 2> Tile64;

__device__ __forceinline__ int swz128(int row) { return (row & 7) ^ ((row >> 3) & 1); }

// Which tile and split item `id` of a problem is.  Workgroups are dispatched
// round-robin over the eight XCDs, each with an L2 of its own: the ids of one
// XCD get a contiguous range of items, and tiles run in groups of GM tile rows,
// so that the workgroups that share an L2 share rows of A and B.
template <int GM>
__device__ __forceinline__ void item_of(int id, int items, int tiles_m, int tiles_n, int &tm, int &tn, int &split) {
  if (items >= 8) {
    // XCD x takes items base(x) .. : the first `extra` XCDs one more than the others
    const int per = items / 8, extra = items - 8 * per, x = id & 7;
    id = x * per + min(x, extra) + (id >> 3);
  }
  const int tiles = tiles_m * tiles_n;
  split = id / tiles;
  const int tile = id - split * tiles;
  const int per_group = GM * tiles_n;
  const int group = tile / per_group;
  const int first = group * GM;
  const int gm = min(tiles_m - first, GM);
  const int in = tile - group * per_group;
  tm = first + in % gm;
  tn = in / gm;
}

// Writes (or, for splits, stores raw) a lane's four consecutive columns.
template <int OUT>
__device__ __forceinline__ void finish4(const GemmProblem &g, int m, int n, const float (&acc)[4]) {
  const float sa = g.sa ? g.sa[m] : 1.0f;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = min(n + i, g.N - 1);
    v[i] = acc[i] * sa;
    if (g.sw) v[i] *= g.sw[c];
    if (g.bias) v[i] += g.bias[c];
  }
  store4<OUT>(static_cast<elem_t<OUT> *>(g.C) + (int64_t)m * g.N + n, g.N - n, v);
}

template <class E, class T, int OUT>
__device__ __forceinline__ void gemm_tile(const GemmProblem &g, int id, uint4 *lds_raw) {
  const uint8_t *lds = reinterpret_cast<const uint8_t *>(lds_raw);
  const uint32_t lds_base = dma::lds_addr(lds_raw);
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  const int r32 = lane & 31, h = lane >> 5;
  int tm, tn, split;
  item_of<T::TM == 256 ? 4 : 8>(id, g.tiles_m * g.tiles_n * g.splits, g.tiles_m, g.tiles_n, tm, tn, split);
  const int m0 = tm * T::TM, n0 = tn * T::TN;

  // what this wave transfers: rows 8 (wave J + j) + lane / 8 of each side; rows
  // past the end repeat the last one
  const int lrow = lane >> 3, lpos = lane & 7;
  uint32_t offa[T::JA], offb[T::JB];
#pragma unroll
  for (int j = 0; j < T::JA; ++j) {
    const int row = 8 * (wave * T::JA + j) + lrow;
    offa[j] = (uint32_t)(min(row, g.M - 1 - m0) * g.pitch_a) + 16u * (uint32_t)(lpos ^ swz128(row));
  }
#pragma unroll
  for (int j = 0; j < T::JB; ++j) {
    const int row = 8 * (wave * T::JB + j) + lrow;
    offb[j] = (uint32_t)(min(row, g.N - 1 - n0) * g.pitch_b) + 16u * (uint32_t)(lpos ^ swz128(row));
  }
  const int total = g.steps * g.parts;
  const int s0 = (int)((int64_t)total * split / g.splits), s1 = (int)((int64_t)total * (split + 1) / g.splits);
  const uint8_t *a0 = g.A + (int64_t)m0 * g.pitch_a, *b0 = g.B + (int64_t)n0 * g.pitch_b;
  int part = g.parts == 1 ? 0 : s0 / max(g.steps, 1), k = s0 - part * g.steps;   // of the next step to transfer
  auto issue = [&](int s) {
    const uint32_t dst = lds_base + (uint32_t)(s & 1) * T::kSlot;
    const uint8_t *a = a0 + part * g.part_a + (int64_t)k * kStep, *b = b0 + (int64_t)k * kStep;
#pragma unroll
    for (int j = 0; j < T::JA; ++j) dma::copy16(offa[j], a, dst + (wave * T::JA + j) * 1024);
#pragma unroll
    for (int j = 0; j < T::JB; ++j) dma::copy16(offb[j], b, dst + T::TM * kStep + (wave * T::JB + j) * 1024);
    if (++k == g.steps) {
      k = 0;
      ++part;
    }
  };

  typename E::acc acc[T::MI][T::NI];
#pragma unroll
  for (int i = 0; i < T::MI; ++i)
#pragma unroll
    for (int j = 0; j < T::NI; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

  // byte of chunk 2 t + h of the lane's row in the first 32-row tile of each side
  // (the rows of the others are 32 further on: the same swizzle)
  uint32_t ca[4], cb[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t c = 16u * (uint32_t)((2 * u + h) ^ swz128(r32));
    ca[u] = (uint32_t)(wm * T::MI * 32 + r32) * kStep + c;
    cb[u] = (uint32_t)(T::TM + wn * T::NI * 32 + r32) * kStep + c;
  }

  // Step s: its transfers were issued a step ago; wait for this wave's, barrier
  // (all have landed, and every wave has read step s - 1), start step s + 1 into
  // the slot of step s - 1, multiply step s.
  if (s0 < s1) issue(s0);
  for (int s = s0; s < s1; ++s) {
    dma::wait_vmcnt<0>();
    __syncthreads();
    if (s + 1 < s1) issue(s + 1);
    const uint8_t *slot = lds + (s & 1) * T::kSlot;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      typename E::frag fa[T::MI], fb[T::NI];
#pragma unroll
      for (int j = 0; j < T::NI; ++j) fb[j] = *reinterpret_cast<const typename E::frag *>(slot + cb[u] + j * 32 * kStep);
#pragma unroll
      for (int i = 0; i < T::MI; ++i) fa[i] = *reinterpret_cast<const typename E::frag *>(slot + ca[u] + i * 32 * kStep);
#pragma unroll
      for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int j = 0; j < T::NI; ++j) acc[i][j] = E::mma(fb[j], fa[i], acc[i][j]);
    }
  }

  // lane l, accumulator e of tile (i, j): row 32 i + l % 32 of C, column 32 j + 8 (e / 4) + 4 h + e % 4
#pragma unroll
  for (int i = 0; i < T::MI; ++i) {
    const int m = m0 + (wm * T::MI + i) * 32 + r32;
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < T::NI; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + (wn * T::NI + j) * 32 + 8 * q + 4 * h;
        if (n >= g.N) continue;
        if (g.splits > 1) {
          // raw sums: int32 bits or fp32
          uint32_t *p = static_cast<uint32_t *>(g.partial) + ((int64_t)split * g.M + m) * g.N + n;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < g.N) p[e] = __builtin_bit_cast(uint32_t, acc[i][j][4 * q + e]);
        } else {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (float)acc[i][j][4 * q + e];
          finish4<OUT>(g, m, n, v);
        }
      }
  }
}

// The sums of a split problem's parts (in order; int32 sums are exact in any
// order), four columns a thread.
template <class E, int OUT>
__device__ __forceinline__ void finish_splits(const GemmProblem &g, int64_t e, int64_t n4) {
  const int m = (int)(e / n4), n = 4 * (int)(e - m * n4);
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = (int64_t)m * g.N + min(n + i, g.N - 1);
    decltype(typename E::acc()[0] + 0) s = 0;
    for (int p = 0; p < g.splits; ++p)
      s += static_cast<const decltype(s) *>(g.partial)[(int64_t)p * g.M * g.N + at];
    v[i] = (float)s;
  }
  finish4<OUT>(g, m, n, v);
}

}  // namespace q8
}  // namespace fmm
