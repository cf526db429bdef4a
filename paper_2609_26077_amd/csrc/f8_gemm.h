// The matrix-core product of the e4m3 layers: C = A B^T over rows that are
// contiguous along the contracted axis, a scale byte for each 128 of them.
//
// Tiles, LDS rows and the ring of half-slots that global_load_lds fills are those of the
// int8 product (q8_gemm.h): a step is 128 bytes of every row of the tile, which here is
// one block, so a row has one scale for it.  A lane takes 32 codes of its row for
// each half step t: the 16-byte chunks 4 t + h and 4 t + 2 + h of the row in lane half h.  Which
// positions they are does not matter as long as both sides agree.
//
// A step of a wave is a chain of slots: slot (t, i) multiplies row tile i of A by the wave's row tiles of
// B, half step t.  A's fragments are read a slot ahead, B's a half step ahead, so that a
// 256 tile's wave holds 48 registers of them beside its 128 sums (a whole half step
// of both ahead would take 96).  The barrier stands before the last slot.
//
// TURNED: B comes as it lies, rows along the contracted axis (dX's weights).  A step is then 128 rows
// of TN bytes in LDS, 16-byte chunk c of row n at c ^ (n / (256 / TN) mod the row's chunks), so that eight rows
// fall on distinct banks, and a lane takes its codes eight at a time by ds_read_b64_tr_b8: of
// sixteen lanes that point at the halves of eight rows' chunks, lane l gets byte l of the eight rows.
//
// Scales stay out of LDS, which the ring of the larger tiles fills: a lane keeps four
// steps' bytes of each of its rows as a word, shifted right by a byte a step.  The
// following words are loaded at the start of the last step of four and waited for at
// its barrier, where few of the ring's transfers are on their way.
//
// What bounds the 256 tile: over a long axis power (8192^3: 432 us, 2.5 PFLOP/s, the matrix cores busy 66% of the
// cycles at 1.7 GHz); over a short one the tiles' ends, which write at HBM's rate (5 us a round of tiles, 7.7 through the
// caches; a start takes 2), and the last, partial round of them (16384
// x 4096 x 4096 of 16 experts, 4.5 rounds of 32 steps: 286 us, busy 48% at 2.0 GHz).  The smaller tiles
// wait for each step's transfers (1000 x 1302 x 1472 fp32: 13 us for 12 steps, busy 8%, LDS reads 5%).  Measured and
// not adopted: one workgroup a CU that walks many tiles, the next one's first steps on their way while a tile
// leaves (grouped products 303 -> 312 us, gradients 360 -> 391: turns fixed beforehand lose what
// dispatching as CUs become free gives); the barrier two slots before the step's end (8192^3 436 -> 455).
#pragma once

#include <hip/hip_runtime.h>

#include "device.h"
#include "f8_types.h"
#include "q8_gemm.h"

namespace fmm {
namespace f8 {

using q8::kStep;
using q8::swz128;
using q8::v16f;
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
using q8::v4i;

// dma::copy16 if `some` > 0 and dma::wait_vmcnt<N> (else <0>), conditions that the compiler does not
// see as control flow: where that joins, it waits for every LDS read that is under way.
__device__ __forceinline__ void copy16_if(int some, uint32_t off, const uint8_t *base, uint32_t m0) {
  asm volatile(
      "s_cmp_le_i32 %3, 0\n\ts_cbranch_scc1 .Lnone%=\n\ts_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1\n.Lnone%=:" ::"v"(off),
      "s"(base), "s"(m0), "s"(some)
      : "memory", "m0", "scc");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt_if(int some) {
  asm volatile("s_cmp_gt_i32 %0, 0\n\ts_cbranch_scc1 .Lsome%=\n\ts_waitcnt vmcnt(0)\n.Lsome%=:\n\ts_waitcnt vmcnt(%1)" ::"s"(some),
               "n"(N)
               : "memory", "scc");
}

// What a workgroup has to do: a tile of C, its rows of A and B, and the steps
// of 128 codes that it contracts.
struct Work {
  const uint8_t *a, *b, *sa, *sb;   // codes and scales of the tile's first rows, from the first step on
  int64_t pitch_a, pitch_b, scale_pitch_a, scale_pitch_b;   // bytes of a row
  int rows_a, rows_b;               // rows that exist (of the tile and past it)
  int steps;
  void *C;                          // the matrix that the tile is of ...
  int m0, n0, M;                    // ... its first output, and the row that ends its expert's
  const float *bias;                // of its first column, or null
};

// fp8 matrix cores (16-bit outputs), or codes converted to bf16 and the bf16
// matrix cores (fp32 outputs): codes and their powers of two are exact in bf16 and
// the sums keep fp32's digits, where the fp8 cores keep 13 bits below the largest
// product of each group of eight: a product of two codes has 8, so the small ones lose some, 1.5e-5 of a sum of normal
// values at any length, a fourteenth of fp16's rounding and a hundredth of bf16's.
struct F8 {
  typedef v16f acc;
  static constexpr bool kScaled = false;      // (the sums leave as they are)
  typedef v8i op;
  static __device__ __forceinline__ op prepare(v8i q, uint32_t) { return q; }
  static __device__ __forceinline__ v16f mma(const op &b, uint32_t sb, const op &a, uint32_t sa, v16f c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, 0, 0, (int)sb, 0, (int)sa);
  }
  static __device__ __forceinline__ v4f mma16(const op &b, uint32_t sb, const op &a, uint32_t sa, v4f c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, 0, (int)sb, 0, (int)sa);
  }
};
struct F8Exact {
  typedef v16f acc;
  static constexpr bool kScaled = false;
  struct op {
    dev::v8bf v[4];
  };
  static __device__ __forceinline__ op prepare(v8i q, uint32_t s) {
    op o;
    const float f = dev::e8m0_at(s, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = dev::dequant8((uint32_t)q[2 * i], (uint32_t)q[2 * i + 1], f);
    return o;
  }
  static __device__ __forceinline__ v16f mma(const op &b, uint32_t, const op &a, uint32_t, v16f c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v[i], a.v[i], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ v4f mma16(const op &b, uint32_t, const op &a, uint32_t, v4f c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[i], a.v[i], c, 0, 0, 0);
    return c;
  }
};

// The work of workgroup `id` (wave-uniform); false: none.  Order as in the int8 product:
// the ids of one XCD get a contiguous range of items, tiles run in groups of GM tile rows.  Where
// the contracted axis is the experts', whose lengths differ, each expert's tiles are spread over the XCDs
// (dW of 16384 x 4096 x 2048 of 16 experts with uneven rows, experts dealt to the XCDs: 270 us).
template <int TM, int TN, bool WEIGHTS, bool TURNED = false>
__device__ __forceinline__ bool work_of(const Product &g, int id, Work &w) {
  constexpr int GM = TM == 256 ? 4 : 8;
  Span s;
  int tm, tn, part;
  if (g.axis) {
    // (whole turns over the XCDs for each expert)
    const int tiles = g.tiles_m * g.tiles_n, turns = (tiles + 7) & ~7, e = id / turns, in = id - e * turns;
    if (in >= tiles || e >= g.experts) return false;
    q8::item_of<GM>(in, tiles, g.tiles_m, g.tiles_n, tm, tn, part);
    Experts x(g.offsets, g.experts, g.rows, kBlock);
    s = x.at(e);
    s.expert = e;
    w.m0 = tm * TM;
    w.M = g.M;
  } else {
    Experts x(g.offsets, g.experts, g.rows, TM);
    if (id >= x.total * g.tiles_n) return false;
    q8::item_of<GM>(id, x.total * g.tiles_n, x.total, g.tiles_n, tm, tn, part);
    s = x.find(tm);
    w.m0 = s.lo + (tm - s.tiles) * TM;
    w.M = s.hi;
  }
  w.n0 = tn * TN;
  const int64_t e = s.expert;
  w.rows_a = w.M - w.m0;
  w.rows_b = g.N - w.n0;
  if (g.axis) {
    // an expert's rows of both operands lie together, as long as its blocks are
    w.steps = (s.hi - s.lo + kBlock - 1) / kBlock;
    w.pitch_a = w.pitch_b = (int64_t)w.steps * kBlock;
    w.scale_pitch_a = w.scale_pitch_b = (w.steps + kScalePad - 1) / kScalePad * kScalePad;
    const int64_t before = (int64_t)s.tiles * kBlock, scales_before = (int64_t)s.wides * kScalePad;
    w.a = g.a.codes + before * g.M + w.m0 * w.pitch_a;
    w.b = g.b.codes + before * g.N + w.n0 * w.pitch_b;
    w.sa = g.a.scales + scales_before * g.M + w.m0 * w.scale_pitch_a;
    w.sb = g.b.scales + scales_before * g.N + w.n0 * w.scale_pitch_b;
    w.C = static_cast<uint8_t *>(g.C) + e * g.M * g.N * g.out_bytes;
  } else {
    w.steps = g.steps;
    w.pitch_a = g.a.pitch;
    w.pitch_b = g.b.pitch;
    w.scale_pitch_a = g.a.scale_pitch;
    w.scale_pitch_b = g.b.scale_pitch;
    w.a = g.a.codes + e * g.a.expert_codes + w.m0 * w.pitch_a;
    w.b = g.b.codes + e * g.b.expert_codes + w.n0 * (TURNED ? 1 : w.pitch_b);
    w.sa = g.a.scales + e * g.a.expert_scales + w.m0 * w.scale_pitch_a;
    w.sb = g.b.scales + e * g.b.expert_scales + (WEIGHTS ? w.n0 / kBlock : w.n0) * w.scale_pitch_b;
    w.C = g.C;
  }
  w.bias = g.bias ? g.bias + e * g.N + w.n0 : nullptr;
  return true;
}

typedef int v2i __attribute__((ext_vector_type(2)));

template <class E, class T, int OUT, bool WEIGHTS, bool TURNED = false>
__device__ __forceinline__ void gemm_tile(const Product &g, const Work &w, uint4 *lds_raw) {
  static_assert(!TURNED || (WEIGHTS && T::NI <= 2), "a row tile's number is one bit of a chunk's");
  constexpr int kChunks = T::TN / 16, kMoved = 64 / kChunks, kApart = 256 / T::TN;   // TURNED: of a row, rows of a transfer, swizzle
  constexpr int J = T::JA, MI = T::MI, NI = T::NI, SB = WEIGHTS ? 1 : NI, Q = 2 * MI;
  static_assert(!WEIGHTS || NI * 32 <= kBlock, "one scale of the weights for a wave's columns");
  const uint8_t *lds = reinterpret_cast<const uint8_t *>(lds_raw);
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  const int r32 = lane & 31, h = lane >> 5;
  const int ns = __builtin_amdgcn_readfirstlane(w.steps);

  // scales of steps 4 i .. 4 i + 3, the first in the low byte
  uint32_t psa[MI], psb[SB];
#pragma unroll
  for (int i = 0; i < MI; ++i) psa[i] = (uint32_t)(min((wm * MI + i) * 32 + r32, w.rows_a - 1) * w.scale_pitch_a);
#pragma unroll
  for (int j = 0; j < SB; ++j) {
    const int row = WEIGHTS ? min(wn * NI * 32, w.rows_b - 1) / kBlock : min((wn * NI + j) * 32 + r32, w.rows_b - 1);
    psb[j] = (uint32_t)(row * w.scale_pitch_b);
  }
  uint32_t sa[MI], sb[SB], na[MI], nb[SB];
  auto load_scales = [&](int step) {
#pragma unroll
    for (int i = 0; i < MI; ++i) na[i] = *reinterpret_cast<const uint32_t *>(w.sa + step + psa[i]);
#pragma unroll
    for (int j = 0; j < SB; ++j) nb[j] = *reinterpret_cast<const uint32_t *>(w.sb + step + psb[j]);
  };
  auto have_scales = [&] {   // (the compiler waits for what load_scales started)
#pragma unroll
    for (int i = 0; i < MI; ++i) asm volatile("" : "+v"(na[i]));
#pragma unroll
    for (int j = 0; j < SB; ++j) asm volatile("" : "+v"(nb[j]));
  };
  auto take_scales = [&] {
#pragma unroll
    for (int i = 0; i < MI; ++i) sa[i] = na[i];
#pragma unroll
    for (int j = 0; j < SB; ++j) sb[j] = nb[j];
  };
  auto shift_scales = [&] {
#pragma unroll
    for (int i = 0; i < MI; ++i) sa[i] >>= 8;
#pragma unroll
    for (int j = 0; j < SB; ++j) sb[j] >>= 8;
  };

  // what this wave transfers of each side: rows 8 (wave J + j) + lane / 8, j < J;
  // rows past the end repeat the last one
  const int lrow = lane >> 3, lpos = lane & 7;
  uint32_t offa[J], offb[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int row = 8 * (wave * J + j) + lrow;
    const uint32_t c = 16u * (uint32_t)(lpos ^ swz128(row));
    offa[j] = (uint32_t)(min(row, w.rows_a - 1) * w.pitch_a) + c;
    // (TURNED: rows kMoved (wave J + j) + lane / kChunks; without the row's own offset, chunks past the row's end repeat its last)
    const int deep = kMoved * (wave * J + j) + lane / kChunks;
    if (TURNED) offb[j] = 16u * (uint32_t)min((lane ^ (deep / kApart)) % kChunks, (int)((w.pitch_b - w.n0) / 16) - 1);
    else offb[j] = (uint32_t)(min(row, w.rows_b - 1) * w.pitch_b) + c;
  }
  const uint32_t rowb = (uint32_t)((kMoved * wave * J + lane / kChunks) * w.pitch_b);
  int leftb = g.turned;   // rows from the next step's first on
  const uint8_t *pa = w.a, *pb = w.b;   // the next step's
  const uint32_t base0 = dma::lds_addr(lds_raw), base = base0 + wave * J * 1024;
  uint32_t wa = 0, wb = T::kHalf, ra = 0, rb = T::kHalf;   // half-slots to fill and to read next, in bytes
  auto turn = [](uint32_t &x) {
    x += 2 * T::kHalf;
    if (x >= T::kLds) x -= T::kLds;
  };
  // half q of the next step's rows of A, of B, if there is such a step
  auto start_a = [&](int q, int some) {
#pragma unroll
    for (int j = q * J / 2; j < (q + 1) * J / 2; ++j) copy16_if(some, offa[j], pa, base + wa + j * 1024);
    if (q == 1) {
      turn(wa);
      pa += kStep;
    }
  };
  auto start_b = [&](int q, int some) {
#pragma unroll
    for (int j = q * J / 2; j < (q + 1) * J / 2; ++j) {
      const uint32_t last = (uint32_t)((min(leftb, kBlock) - 1) * w.pitch_b);
      const uint32_t off = TURNED ? min(rowb + kMoved * j * (uint32_t)w.pitch_b, last) + offb[j] : offb[j];
      copy16_if(some, off, pb, base + wb + j * 1024);
    }
    if (q == 1) {
      turn(wb);
      pb += TURNED ? kStep * w.pitch_b : kStep;
      leftb -= kStep;
    }
  };

  v16f acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = (v16f){};

  // byte of chunk h of the lane's row in the first 32-row tile of each side (chunk 2 u + h: xor 32 u)
  const uint32_t ca = (uint32_t)(wm * MI * 32 + r32) * kStep + 16u * (uint32_t)(h ^ swz128(r32));
  // (TURNED: lane s of sixteen points at half s & 1 of the chunk of its row tile's half, in row s / 2 of eight, sixteen rows on in half h)
  const int deep = lane >> 1 & 7;
  const uint32_t cb = TURNED ? (uint32_t)(deep + 16 * h) * T::TN + 8u * (lane & 1) +
                                   16u * (uint32_t)((2 * wn * NI + (lane >> 4 & 1)) ^ (deep / kApart))
                             : (uint32_t)(wn * NI * 32 + r32) * kStep + 16u * (uint32_t)(h ^ swz128(r32));
  auto read = [&](uint32_t at, int half) {
    const v4i lo = *reinterpret_cast<const v4i *>(lds + (at ^ (64u * half)));
    const v4i hi = *reinterpret_cast<const v4i *>(lds + (at ^ (64u * half + 32u)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  constexpr int kBufs = T::kWhole ? 4 : 2;
  v8i fa[kBufs], fb[kBufs][NI];
  auto load_a = [&](int half, int i, int buf) { fa[buf] = read(ra + ca + i * 32 * kStep, half); };
  auto load_b = [&](int half, int buf) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      if constexpr (TURNED) {
        // chunks 4 half + h and 4 half + 2 + h of sixteen rows, eight rows at a time
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const uint32_t at = ((rb + cb) ^ (32u * j) ^ (128u / kApart * (p & 1))) + (64 * half + 32 * (p >> 1) + 8 * (p & 1)) * T::TN;
          const v2i v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i *)(base0 + at));
          fb[buf][j][2 * p] = v[0];
          fb[buf][j][2 * p + 1] = v[1];
        }
      } else {
        fb[buf][j] = read(rb + cb + j * 32 * kStep, half);
      }
    }
  };
  // every wave's transfers of the next step have landed (where later > 0, kLater of
  // this wave's may be on their way) and its reads of this one are done
  auto next_step = [&](int later) {
    constexpr int kLater = 2 * J * (T::H - 2) + J;   // H - 2 whole steps, and A of one more
    wait_vmcnt_if<kLater>(later);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  if (ns > 0) {
    load_scales(0);
#pragma unroll
    for (int s = 0; s < T::H; ++s) {
      start_a(0, ns - s); start_a(1, ns - s);
      if (s < T::H - 1) {
        start_b(0, ns - s); start_b(1, ns - s);
      }
    }
    next_step(ns - T::H + 1);
    have_scales();
    take_scales();
    if constexpr (T::kWhole) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        load_a(u, 0, u);
        load_b(u, u);
      }
      start_b(0, ns - T::H + 1); start_b(1, ns - T::H + 1);
      start_a(0, ns - T::H); start_a(1, ns - T::H);
    } else {
      start_b(0, ns - T::H + 1);
      load_b(0, 0);
      load_a(0, 0, 0);
    }
  }
  // A step, without control flow: after the last one it reads fragments that nobody
  // uses.  LAST: of four, the following ones' scales are on their way.
  auto step = [&](int s, auto BUF, auto LAST) {
    const int far = ns - s - T::H, more = far + 1, far1 = far - 1;
    if constexpr (T::kWhole) {
      // Small tiles: all of a step's fragments are read while the step before is
      // multiplied.  B of s + H and A of s + H + 1 go where A and B of s were.
      constexpr int b = 2 * decltype(BUF)::value;
      next_step(far);
      if constexpr (decltype(LAST)::value) have_scales();
      turn(ra);
      turn(rb);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        load_a(u, 0, 2 - b + u);
        load_b(u, 2 - b + u);
      }
      __builtin_amdgcn_sched_barrier(0);
      start_b(0, far); start_b(1, far);
      start_a(0, far1); start_a(1, far1);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        acc[0][0] = E::mma(E::prepare(fb[b + u][0], sb[0]), sb[0], E::prepare(fa[b + u], sa[0]), sa[0], acc[0][0]);
    } else {
      typename E::op ob[NI];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int half = q / MI, i = q % MI;
        if (q == Q - 1) {
          // B of s + H may fill A's half-slot of s, and A of s + H + 1 then B's
          next_step(far);
          if constexpr (decltype(LAST)::value) have_scales();
          turn(ra);
          turn(rb);
          load_b(0, 0);
          load_a(0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
          start_b(0, far);
        } else {
          load_a((q + 1) / MI, (q + 1) % MI, (q + 1) & 1);
          if (q == 0) load_b(1, 1);
          __builtin_amdgcn_sched_barrier(0);   // (left to itself the compiler reads a fragment just before it is used)
        }
        if (i == 0) {
#pragma unroll
          for (int j = 0; j < NI; ++j) ob[j] = E::prepare(fb[half][j], sb[WEIGHTS ? 0 : j]);
        }
        const typename E::op oa = E::prepare(fa[q & 1], sa[i]);
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = E::mma(ob[j], sb[WEIGHTS ? 0 : j], oa, sa[i], acc[i][j]);
        if (q == Q / 4 - 1) start_b(1, more);
        if (q == Q / 2 - 1) start_a(0, far);
        if (q == 3 * Q / 4 - 1) start_a(1, far);
      }
    }
    shift_scales();
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  const std::true_type yes;
  const std::false_type no;
  // a wave whose part of the tile lies past the matrix (or the expert's rows) only transfers
  const bool idle = (wm * MI * 32 >= w.rows_a || wn * NI * 32 >= w.rows_b);
  if (idle) {
    for (int s = 0; s < ns; ++s) {
      const int far = ns - s - T::H;
      if constexpr (T::kWhole) {
        next_step(far);
        start_b(0, far); start_b(1, far);
        start_a(0, far - 1); start_a(1, far - 1);
      } else {
        start_b(1, far + 1);
        start_a(0, far); start_a(1, far);
        next_step(far);
        start_b(0, far);
      }
    }
    __syncthreads();
    return;
  }
  for (int s = 0; s < ns; ++s) {
    step(s, even, no);
    if (++s == ns) break;
    step(s, odd, no);
    if (++s == ns) break;
    step(s, even, no);
    if (++s == ns) break;
    load_scales(s + 1 < ns ? s + 1 : s - 3);
    step(s, odd, yes);
    take_scales();
  }

  // lane l, accumulator e of tile (i, j): row 32 i + l % 32 of C, column 32 j + 8 (e / 4) + 4 h + e % 4
  if (w.bias) {
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = (wn * NI + j) * 32 + 8 * q + 4 * h, left = w.rows_b - n;
        float b[4] = {};
        if (left > 0) q8::load4(w.bias + n, left, b);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += b[e];
      }
  }
  __syncthreads();
  // Tiles that begin together end together, and their stores wait for HBM.  Past the caches they do so less: over 68
  // outputs of 12 to 500 MB 7% less time on average (8192 x 8192 with 1024 positions 85 -> 72 us; 5888 x 7136 with 640
  // 39.6 -> 41.1).  With whoever reads the output right behind (a clamp, the quantizer) 1.4% less to 24 MB, 2.3% more from 40 to
  // 90 MB, which the last-level cache would have kept (5888 x 7136 with 640 66 -> 72), and 2.7% less beyond.  Not where
  // rows begin off 16 bytes: lines written in pieces have to meet in the caches (10464 x 5899 with 357 positions 52 us, 75
  // past them).  A start in turns gains nothing.
  const bool stream = T::TM == 256 && g.N * (OUT == FMM_F32 ? 4 : 2) % 16 == 0 && reinterpret_cast<uintptr_t>(w.C) % 16 == 0;
  q8::GemmProblem out = {};
  out.M = w.M;
  out.N = g.N;
  const int mw = w.m0 + wm * MI * 32, nw = w.n0 + wn * NI * 32;
  uint8_t *share = reinterpret_cast<uint8_t *>(lds_raw) + wave * (T::kLds / T::kWaves);
  if (mw + MI * 32 > out.M || nw + NI * 32 > out.N) return q8::store_tile<E, T, OUT, false>(out, w.C, acc, mw, nw, share);
  if constexpr (T::TM == 256) {
    if (stream) return q8::store_tile<E, T, OUT, true, true>(out, w.C, acc, mw, nw, share);
  }
  q8::store_tile<E, T, OUT, true>(out, w.C, acc, mw, nw, share);
}

}  // namespace f8
}  // namespace fmm
