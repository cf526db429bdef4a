// The product of the e4m3 layers: C = A B^T over rows that are contiguous along
// the contracted axis, a scale byte for each 128 of them.
#pragma once

#include <hip/hip_runtime.h>

#include "device.h"
#include "f8_types.h"

namespace fmm {
namespace f8 {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// What a workgroup has to do: a tile of C, its rows of A and B, and the steps
// of 128 codes that it contracts.
struct Work {
  const uint8_t *a, *b, *sa, *sb;   // codes and scales of the tile's first rows, from the first step on
  int rows_a, rows_b;               // rows that exist (of the tile and past it)
  int steps;
  void *C;                          // the tile's first output
  const float *bias;                // of its first column, or null
};

// fp8 matrix cores (16-bit outputs), or codes converted to bf16 and the bf16
// matrix cores (fp32 outputs): codes and their powers of two are exact in bf16 and
// the sums keep fp32's digits, where the fp8 cores keep 13 bits below the largest
// product of each group of eight.
struct F8 {
  static __device__ __forceinline__ v16f mma(v8i b, uint32_t sb, v8i a, uint32_t sa, v16f c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, 0, 0, (int)sb, 0, (int)sa);
  }
};
struct F8Exact {
  static __device__ __forceinline__ v16f mma(v8i b, uint32_t sb, v8i a, uint32_t sa, v16f c) {
    const float fa = dev::e8m0_at(sa, 0), fb = dev::e8m0_at(sb, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dev::dequant8((uint32_t)b[2 * i], (uint32_t)b[2 * i + 1], fb),
                                                  dev::dequant8((uint32_t)a[2 * i], (uint32_t)a[2 * i + 1], fa), c, 0, 0, 0);
    return c;
  }
};

// The work of workgroup `id` (wave-uniform); false: none.
template <int TM, int TN, bool WEIGHTS>
__device__ __forceinline__ bool work_of(const Product &g, int id, int out_bytes, Work &w) {
  Span s;
  int tm, tn, m0, split = 0;
  if (g.axis) {
    const int per = g.tiles_m * g.tiles_n, e = id / (per * g.splits);
    id -= e * per * g.splits;
    split = id / per;
    id -= split * per;
    tm = id % g.tiles_m;
    tn = id / g.tiles_m;
    m0 = tm * TM;
    Experts x(g.offsets, g.experts, g.rows, kBlock);
    s = x.at(e);
  } else {
    Experts x(g.offsets, g.experts, g.rows, TM);
    tm = id / g.tiles_n;
    tn = id % g.tiles_n;
    if (tm >= x.total) return false;
    s = x.find(tm);
    m0 = s.lo + (tm - s.tiles) * TM;
  }
  const int n0 = tn * TN;
  const int64_t e = s.expert;
  w.a = g.a.codes + e * g.a.expert_codes + m0 * g.a.pitch;
  w.sa = g.a.scales + e * g.a.expert_scales + m0 * g.a.scale_pitch;
  w.b = g.b.codes + e * g.b.expert_codes + n0 * g.b.pitch;
  w.sb = g.b.scales + e * g.b.expert_scales + (WEIGHTS ? n0 / kBlock : n0) * g.b.scale_pitch;
  w.rows_a = (g.axis ? g.M : s.hi) - m0;
  w.rows_b = g.N - n0;
  w.steps = g.steps;
  int64_t row = m0;
  if (g.axis) {
    w.steps = (s.hi - s.lo + kBlock - 1) / kBlock;
    w.a += (int64_t)s.tiles * kBlock;
    w.b += (int64_t)s.tiles * kBlock;
    w.sa += (int64_t)s.wides * kScalePad;
    w.sb += (int64_t)s.wides * kScalePad;
    row += e * g.M;
  }
  w.C = static_cast<uint8_t *>(g.C) + (row * g.N + n0) * out_bytes;
  w.bias = g.bias ? g.bias + e * g.N + n0 : nullptr;
  return true;
}

// One wave, one 32 x 32 tile, operands straight from memory.  Lane (r, h) takes 32 of
// a row's 64 codes; which ones does not matter as long as both sides agree.
template <class E, int OUT, bool WEIGHTS>
__device__ __forceinline__ void gemm_tile(const Product &g, const Work &w, int mw, int nw) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  if (mw >= w.rows_a || nw >= w.rows_b) return;
  const int ra = min(mw + r, w.rows_a - 1), rb = min(nw + r, w.rows_b - 1);
  const uint8_t *a = w.a + ra * g.a.pitch + 32 * h, *b = w.b + rb * g.b.pitch + 32 * h;
  const uint8_t *sa = w.sa + ra * g.a.scale_pitch, *sb = w.sb + (WEIGHTS ? rb / kBlock : rb) * g.b.scale_pitch;
  v16f acc = {};
  for (int s = 0; s < w.steps; ++s) {
    const uint32_t ea = sa[s], eb = sb[s];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const v8i fa = *reinterpret_cast<const v8i *>(a + (int64_t)s * kBlock + 64 * t);
      const v8i fb = *reinterpret_cast<const v8i *>(b + (int64_t)s * kBlock + 64 * t);
      acc = E::mma(fb, eb, fa, ea, acc);
    }
  }
  // lane (r, h), element e: row r, column 8 (e / 4) + 4 h + e % 4
  if (mw + r >= w.rows_a) return;
  elem_t<OUT> *out = static_cast<elem_t<OUT> *>(w.C) + (int64_t)(mw + r) * g.N + nw;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int n = 8 * (e >> 2) + 4 * h + (e & 3);
    if (nw + n < w.rows_b) out[n] = (elem_t<OUT>)(acc[e] + (w.bias ? w.bias[nw + n] : 0.0f));
  }
}

}  // namespace f8
}  // namespace fmm
