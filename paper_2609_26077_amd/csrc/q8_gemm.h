// The matrix-core product of the 8-bit linear layer: C = A B^T over rows that
// are contiguous along the contracted axis, int8 (int32 sums) or bfloat16
// (fp32 sums).
//
// Both element types share one data path.  A step is 128 bytes of every row of
// the tile (128 int8 or 64 bfloat16 positions) in LDS; a matrix instruction takes
// 16 bytes a lane of 32 rows of each side (v_mfma_i32_32x32x32_i8,
// v_mfma_f32_32x32x16_bf16), so a step is four instructions per 32 x 32 tile.
// Which positions a lane's 16 bytes are does not matter as long as both sides
// agree: instruction t of a step takes chunk 2 t + h of the row in lane half h.
//
// A ring of 2 H + 1 half-slots (one side's rows of one step each) is filled by
// global_load_lds: while step s is multiplied, steps s + 1 to s + H - 1 and the A
// side of s + H are on their way, a quarter of a step's transfers started after
// each half of the step's instructions, so that no wave queues behind a burst of
// them.  Fragments are read one instruction ahead of the one that takes
// them, across the barrier too: it stands in the middle of a step's last
// instructions, when the step has been read and the next one has landed.
//
// LDS rows are 128 bytes; 16-byte chunk c of row r sits at chunk
// c ^ (r & 7) ^ ((r >> 3) & 1), so that the lanes of a fragment read fall on
// distinct banks.  A transfer moves eight rows (lane l: row l / 8, chunk
// position l % 8), the swizzle being applied to the address that the lane
// reads from, so each row's 128 bytes are one full line of HBM or L2.
//
// The instruction's first operand is B and its second is A: a lane then holds
// one row of C and, per four accumulators, four consecutive columns of it.
//
// What bounds the 256 x 256 tile is power: at 8192^3 int8 the matrix cores are
// busy 73% of the cycles, at 1.6 to 1.7 GHz; 420 us with operands that the caches
// keep from call to call (2.6 POP/s; the runtime's own int8 product 434 and 71%),
// 450 to 460 with others.  bf16, 8192 x 4096 x 8192: 392 to 400 us, 1.37 to
// 1.40 PFLOP/s.  The smaller tiles reach no unit's rate: at 2048 x 4096 x 4096 (35 us,
// 128 x 128) the matrix cores are busy 41% of the cycles, LDS with reads 22%, and
// 570 MB pass through L2 (16 TB/s, 7 requests a cycle and XCD of 16); at 1000 x 1302 x
// 1472 (9.4 us, 64 x 64) 5%, 6% and 77 MB.  They wait for each step's transfers, at a
// barrier a step, with two workgroups on a CU or one.
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
  static constexpr bool kScaled = true;
  static __device__ __forceinline__ acc mma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
  }
};
struct Bf16 {
  typedef v8bf frag;
  typedef v16f acc;
  static constexpr bool kScaled = false;
  static __device__ __forceinline__ acc mma(frag a, frag b, acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

// Tile of TM x TN outputs, WM x WN waves, H steps ahead.
template <int TM_, int TN_, int WM_, int WN_, int H_>
struct Tile {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, H = H_;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int MI = TM / WM / 32, NI = TN / WN / 32;   // 32 x 32 tiles of a wave
  static constexpr int kHalf = TM * kStep;                     // one side's rows of one step
  static constexpr int kLds = (2 * H + 1) * kHalf;
  static constexpr bool kWhole = MI * NI == 1;   // fragments are read a whole step ahead
  static constexpr int JA = TM / 8 / kWaves, JB = TN / 8 / kWaves;   // transfers of a wave per step and side
  static_assert(TM == TN && JA % 2 == 0, "equal sides, whole transfers in half of one");
  static_assert(MI * 32 * WM == TM && NI * 32 * WN == TN && JA * 8 * kWaves == TM && JB * 8 * kWaves == TN, "tile");
};
typedef Tile<256, 256, 2, 4, 2> Tile256;   // one workgroup a CU
typedef Tile<128, 128, 2, 2, 2> Tile128;   // two
typedef Tile<64, 64, 2, 2, 4> Tile64;      // two
// Where there are no more tiles of 128 than CUs, a CU has one workgroup whatever the
// ring's size: one step further ahead, and eight waves for what four leave waiting.
// The int8 product on such shapes, against Tile128: 16% less time up to 512 positions,
// 11% to 2048, 25% beyond, never more; with more tiles than CUs 4 to 24% more, as only
// one of these fits a CU (four waves as far ahead: 4% more to 24% less; four steps
// ahead: as three).
typedef Tile<128, 128, 2, 4, 3> Tile128Ahead;

__device__ __forceinline__ int swz128(int row) { return (row & 7) ^ ((row >> 3) & 1); }

// Which tile, and which run of steps, item `id` of a problem is.  Workgroups are dispatched
// round-robin over the eight XCDs, each with an L2 of its own: the ids of one
// XCD get a contiguous range of items, and tiles run in groups of GM tile rows,
// so that the workgroups that share an L2 share rows of A and B.
template <int GM>
__device__ __forceinline__ void item_of(int id, int items, int tiles_m, int tiles_n, int &tm, int &tn,
                                        int &split) {
  if (items >= 8) {
    // XCD x takes items base(x) .. : the first `extra` XCDs one more than the others
    const int per = items / 8, extra = items - 8 * per, x = id & 7;
    id = x * per + min(x, extra) + (id >> 3);
  }
  split = id / (tiles_m * tiles_n);
  id -= split * tiles_m * tiles_n;
  const int per_group = GM * tiles_n;
  const int group = id / per_group;
  const int first = group * GM;
  const int gm = min(tiles_m - first, GM);
  const int in = id - group * per_group;
  tm = first + in % gm;
  tn = in / gm;
}

// four consecutive floats of p, of which the first n exist (the others: the last one again)
__device__ __forceinline__ void load4(const float *p, int n, float (&v)[4]) {
  if (n >= 4) {
    const u32x4 w = *reinterpret_cast<const u32x4_a4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = p[min(i, n - 1)];
  }
}

// What leaves a wave: its MI x NI tiles of 32 x 32 sums, scaled, converted and
// stored.  A lane holds four consecutive columns of 32 rows apart, which would
// reach memory as 8-byte pieces of 32 lines at a time (a 256 x 256 tile's start and
// end took 23 us, as much as 14 steps); so the tiles pass through the wave's own
// part of LDS, free once every wave has read the last step, and leave in rows of
// 16 bytes a lane (10 us).  16-byte chunk c of a row sits at chunk c ^ (row mod the row's
// chunks).  FULL: the whole wave tile lies inside C.  STREAM: past the caches.
template <class E, class T, int OUT, bool FULL, bool STREAM = false>
__device__ __forceinline__ void store_tile(const GemmProblem &g, void *C, typename E::acc (&acc)[T::MI][T::NI], int m0,
                                           int n0, uint8_t *lds) {
  constexpr int B = OUT == FMM_F32 ? 4 : 2, EPC = 16 / B;          // bytes of an element, elements of a chunk
  constexpr int CH = T::NI * 32 / EPC;                             // chunks of a row
  constexpr int kRow = CH * 16;
  constexpr int kPasses = T::kWaves * T::MI * 32 * kRow > T::kLds ? 2 : 1;
  constexpr int MP = T::MI / kPasses;                              // tile rows of a pass
  static_assert(MP * kPasses == T::MI && T::kWaves * MP * 32 * kRow <= T::kLds, "the tile passes through LDS");
  const int lane = threadIdx.x & 63, r32 = lane & 31, h = lane >> 5;
  float sa[T::MI];
  if (E::kScaled) {
#pragma unroll
    for (int i = 0; i < T::MI; ++i) sa[i] = g.sa[FULL ? m0 + 32 * i + r32 : min(m0 + 32 * i + r32, g.M - 1)];
  }
#pragma unroll
  for (int pass = 0; pass < kPasses; ++pass) {
#pragma unroll
    for (int j = 0; j < T::NI; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = 32 * j + 8 * q + 4 * h;
        float sw[4] = {}, bias[4] = {};
        if (E::kScaled) {
          const int left = FULL ? 4 : g.N - n0 - n;
          if (left > 0) {
            load4(g.sw + n0 + n, left, sw);
            if (g.bias) load4(g.bias + n0 + n, left, bias);
          }
        }
#pragma unroll
        for (int i = 0; i < MP; ++i) {
          const int row = 32 * i + r32;
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = (float)acc[pass * MP + i][j][4 * q + e];
            if (E::kScaled) v[e] = v[e] * sa[pass * MP + i] * sw[e] + bias[e];
          }
          uint8_t *at = lds + row * kRow + 16 * ((n / EPC) ^ (row & (CH - 1))) + n % EPC * B;
          if constexpr (OUT == FMM_F32) {
            *reinterpret_cast<float4 *>(at) = make_float4(v[0], v[1], v[2], v[3]);
          } else {
            *reinterpret_cast<uint2 *>(at) = make_uint2(pack2<OUT>(v[0], v[1]), pack2<OUT>(v[2], v[3]));
          }
        }
      }
    const int lrow = lane / CH, c = lane % CH;
    const int n = n0 + c * EPC;
    elem_t<OUT> *out = static_cast<elem_t<OUT> *>(C) + (int64_t)(m0 + 32 * pass * MP + lrow) * g.N + n;
    const auto put = [&](u32x4 v) {
      if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_a2 *>(out));
      else *reinterpret_cast<u32x4_a2 *>(out) = v;
    };
#pragma unroll
    for (int e = 0; e < MP * 32 * CH / 64; ++e) {
      const int row = (64 / CH) * e + lrow;
      const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + row * kRow + 16 * (c ^ (row & (CH - 1))));
      if (FULL) {
        put(v);
      } else if (m0 + 32 * pass * MP + row < g.M && n < g.N) {
        if (n + EPC <= g.N) {
          put(v);
        } else {
#pragma unroll
          for (int k = 0; k < EPC; ++k)
            if (n + k < g.N) {
              if constexpr (B == 4) reinterpret_cast<uint32_t *>(out)[k] = v[k];
              else reinterpret_cast<uint16_t *>(out)[k] = (uint16_t)(v[k / 2] >> (16 * (k % 2)));
            }
        }
      }
      out += (int64_t)(64 / CH) * g.N;
    }
  }
}

template <class E, class T, int OUT>
__device__ __forceinline__ void gemm_tile(const GemmProblem &g, int id, uint4 *lds_raw) {
  constexpr int J = T::JA;
  const uint8_t *lds = reinterpret_cast<const uint8_t *>(lds_raw);
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  const int r32 = lane & 31, h = lane >> 5;
  int tm, tn, split;
  item_of<T::TM == 256 ? 4 : 8>(id, g.tiles_m * g.tiles_n * g.splits, g.tiles_m, g.tiles_n, tm, tn, split);
  const int m0 = tm * T::TM, n0 = tn * T::TN;

  // what this wave transfers of each side: rows 8 (wave J + j) + lane / 8, j < J;
  // rows past the end repeat the last one
  const int lrow = lane >> 3, lpos = lane & 7;
  uint32_t offa[J], offb[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int row = 8 * (wave * J + j) + lrow;
    const uint32_t c = 16u * (uint32_t)(lpos ^ swz128(row));
    offa[j] = (uint32_t)(min(row, g.M - 1 - m0) * g.pitch_a) + c;
    offb[j] = (uint32_t)(min(row, g.N - 1 - n0) * g.pitch_b) + c;
  }
  const uint8_t *pa = g.A + (int64_t)m0 * g.pitch_a, *pb = g.B + (int64_t)n0 * g.pitch_b;   // the next step's
  const uint8_t *const pb0 = pb;
  const int64_t next_part = g.part_a - (int64_t)g.steps * kStep;
  // this run of steps, and the place of its first in its plane
  int ns = g.steps * g.parts, ka = 0;
  if (g.splits > 1) {
    const int first = (int)((int64_t)ns * split / g.splits);
    ns = (int)((int64_t)ns * (split + 1) / g.splits) - first;
    const int part = first / g.steps;
    ka = first - part * g.steps;
    pa += part * g.part_a + (int64_t)ka * kStep;
    pb += (int64_t)ka * kStep;
  }
  int kb = ka;
  const uint32_t base = dma::lds_addr(lds_raw) + wave * J * 1024;
  uint32_t wa = 0, wb = T::kHalf, ra = 0, rb = T::kHalf;   // half-slots to fill and to read next, in bytes
  auto turn = [](uint32_t &x) {
    x += 2 * T::kHalf;
    if (x >= T::kLds) x -= T::kLds;
  };
  // half q of the next step's rows of A, of B
  auto start_a = [&](int q) {
#pragma unroll
    for (int j = q * J / 2; j < (q + 1) * J / 2; ++j) dma::copy16(offa[j], pa, base + wa + j * 1024);
    if (q == 1) {
      turn(wa);
      pa += kStep;
      if (++ka == g.steps) {
        ka = 0;
        pa += next_part;
      }
    }
  };
  auto start_b = [&](int q) {
#pragma unroll
    for (int j = q * J / 2; j < (q + 1) * J / 2; ++j) dma::copy16(offb[j], pb, base + wb + j * 1024);
    if (q == 1) {
      turn(wb);
      pb += kStep;
      if (++kb == g.steps) {
        kb = 0;
        pb = pb0;
      }
    }
  };

  typename E::acc acc[T::MI][T::NI];
#pragma unroll
  for (int i = 0; i < T::MI; ++i)
#pragma unroll
    for (int j = 0; j < T::NI; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

  // byte of chunk 2 u + h of the lane's row in the first 32-row tile of each side
  // (the rows of the others are 32 further on: the same swizzle)
  uint32_t ca[4], cb[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t c = 16u * (uint32_t)((2 * u + h) ^ swz128(r32));
    ca[u] = (uint32_t)(wm * T::MI * 32 + r32) * kStep + c;
    cb[u] = (uint32_t)(wn * T::NI * 32 + r32) * kStep + c;
  }
  constexpr int kBufs = T::kWhole ? 8 : 2;
  typename E::frag fa[kBufs][T::MI], fb[kBufs][T::NI];
  auto load = [&](int u, int buf) {
#pragma unroll
    for (int j = 0; j < T::NI; ++j)
      fb[buf][j] = *reinterpret_cast<const typename E::frag *>(lds + rb + cb[u] + j * 32 * kStep);
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
      fa[buf][i] = *reinterpret_cast<const typename E::frag *>(lds + ra + ca[u] + i * 32 * kStep);
    __builtin_amdgcn_sched_barrier(0);   // (left to itself the compiler reads a fragment just before it is used)
  };
  auto multiply = [&](int buf, int i0, int i1) {
#pragma unroll
    for (int i = i0; i < i1; ++i)
#pragma unroll
      for (int j = 0; j < T::NI; ++j) acc[i][j] = E::mma(fb[buf][j], fa[buf][i], acc[i][j]);
  };
  // every wave's transfers of the next step have landed (where `later`, kLater of
  // this wave's may be on their way) and its reads of this one are done
  auto next_step = [&](bool later) {
    constexpr int kLater = 2 * J * (T::H - 2) + J;   // H - 2 whole steps, and A of one more
    if (later) dma::wait_vmcnt<kLater>(); else dma::wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  if (ns > 0) {
#pragma unroll
    for (int s = 0; s < T::H - 1; ++s)
      if (s < ns) {
        start_a(0); start_a(1); start_b(0); start_b(1);
      }
    if (T::H - 1 < ns) {
      start_a(0); start_a(1);
    }
    next_step(T::H - 1 < ns);
    if constexpr (T::kWhole) {
#pragma unroll
      for (int u = 0; u < 4; ++u) load(u, u);
      if (T::H - 1 < ns) {
        start_b(0); start_b(1);
      }
      if (T::H < ns) {
        start_a(0); start_a(1);
      }
    } else {
      if (T::H - 1 < ns) start_b(0);
      load(0, 0);
    }
  }
  // A step; FULL: H + 1 steps or more come after it.  The steps of the loop are
  // FULL ones without a branch: where control flow joins, the compiler waits for
  // every LDS read that is under way, the next step's fragments among them.
  auto step = [&](int s, auto BUF, auto FULL) {
    constexpr bool full = decltype(FULL)::value;
    const bool one = full || s + 1 < ns, more = full || s + T::H - 1 < ns, far = full || s + T::H < ns,
               far1 = full || s + T::H + 1 < ns;
    if constexpr (T::kWhole) {
      // Small tiles: a step's matrix instructions take no longer than reading a
      // fragment does, so all of a step's fragments are read while the step before
      // is multiplied.  B of s + H and A of s + H + 1 go where A and B of s were.
      constexpr int b = decltype(BUF)::value;
      if (one) {
        next_step(far);
        turn(ra);
        turn(rb);
#pragma unroll
        for (int u = 0; u < 4; ++u) load(u, 4 * (1 - b) + u);
        if (far) {
          start_b(0); start_b(1);
        }
        if (far1) {
          start_a(0); start_a(1);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) multiply(4 * b + u, 0, T::MI);
    } else {
      load(1, 1);
      multiply(0, 0, T::MI / 2);
      if (more) start_b(1);
      multiply(0, T::MI / 2, T::MI);
      load(2, 0);
      multiply(1, 0, T::MI / 2);
      if (far) start_a(0);
      multiply(1, T::MI / 2, T::MI);
      load(3, 1);
      multiply(0, 0, T::MI / 2);
      if (far) start_a(1);
      multiply(0, T::MI / 2, T::MI);
      multiply(1, 0, T::MI / 2);
      if (one) {
        // B of s + H may fill A's half-slot of s, and A of s + H + 1 then B's
        next_step(far);
        turn(ra);
        turn(rb);
        load(0, 0);
        if (far) start_b(0);
      }
      multiply(1, T::MI / 2, T::MI);
    }
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  int s = 0;
  if constexpr (T::kWhole) {
    for (; s + 1 + T::H + 1 < ns; s += 2) {
      step(s, even, std::true_type{});
      step(s + 1, odd, std::true_type{});
    }
    for (; s < ns; s += 2) {
      step(s, even, std::false_type{});
      if (s + 1 < ns) step(s + 1, odd, std::false_type{});
    }
  } else {
    for (; s + T::H + 1 < ns; ++s) step(s, even, std::true_type{});
    for (; s < ns; ++s) step(s, even, std::false_type{});
  }

  // lane l, accumulator e of tile (i, j): row 32 i + l % 32 of C, column 32 j + 8 (e / 4) + 4 h + e % 4
  __syncthreads();
  const int mw = m0 + wm * T::MI * 32, nw = n0 + wn * T::NI * 32;
  uint8_t *share = reinterpret_cast<uint8_t *>(lds_raw) + wave * (T::kLds / T::kWaves);
  const bool full = mw + T::MI * 32 <= g.M && nw + T::NI * 32 <= g.N;
  if constexpr (!E::kScaled) {
    if (g.splits > 1) {
      float *sums = g.partial + (int64_t)split * g.M * g.N;
      if (full) store_tile<E, T, FMM_F32, true>(g, sums, acc, mw, nw, share);
      else store_tile<E, T, FMM_F32, false>(g, sums, acc, mw, nw, share);
      return;
    }
  }
  if (full) store_tile<E, T, OUT, true>(g, g.C, acc, mw, nw, share);
  else store_tile<E, T, OUT, false>(g, g.C, acc, mw, nw, share);
}

}  // namespace q8
}  // namespace fmm
