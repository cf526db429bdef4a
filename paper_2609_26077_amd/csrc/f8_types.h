// Device side of the e4m3 blocks: scales, codes and their values.
#pragma once

#include "f8.h"
#include "q8_types.h"

namespace fmm {
namespace f8 {

using q8::elem_t;
using q8::u32x2;
using q8::u32x4;

typedef short v2i16 __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

// |x| as bits, 0 for NaN and infinities: what a block's maximum is taken of
__device__ __forceinline__ uint32_t magnitude(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7fffffffu;
  return m < 0x7f800000u ? m : 0u;
}

// The scale byte e + 127 of a block with maximum a (its bits): the least e >= -126
// with a <= 448 2^e = 1.75 2^(e + 8); 2^0 where a = 0.  At most 247.
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  const int e = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
  return a == 0 ? 127u : (uint32_t)max(e, 1);
}

// 2^(b - 127), every byte's (0: 2^-127, 255: NaN)
__device__ __forceinline__ float scale_value(uint32_t b) {
  return __uint_as_float(b == 0 ? 0x400000u : b == 255 ? 0x7fc00000u : b << 23);
}

// Codes of four values under the scale s = 2^e, |v| <= 448 s: nearest, ties to even.
// (v_cvt_scalef32_pk_fp8_f32 divides by the power of two exactly; what is not finite is made the code NaN.)
__device__ __forceinline__ float finite_or_nan(float v) {
  return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u ? v : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ uint32_t codes4(float v0, float v1, float v2, float v3, float s) {
  v2i16 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32((v2i16){0, 0}, finite_or_nan(v0), finite_or_nan(v1), s, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, finite_or_nan(v2), finite_or_nan(v3), s, true);
  return __builtin_bit_cast(uint32_t, w);
}

// eight codes -> their values times s
__device__ __forceinline__ void values8(u32x2 w, float s, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    v[4 * i] = a[0] * s;
    v[4 * i + 1] = a[1] * s;
    v[4 * i + 2] = b[0] * s;
    v[4 * i + 3] = b[1] * s;
  }
}

// ---- experts ---------------------------------------------------------------------
// lane l of a wave: op over lanes 0 .. l
template <class F>
__device__ __forceinline__ int scan64(int v, F op, int id) {
  // (a lane without a source takes id)
  v = op(v, __builtin_amdgcn_update_dpp(id, v, 0x111, 0xf, 0xf, false));   // row_shr:1
  v = op(v, __builtin_amdgcn_update_dpp(id, v, 0x112, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(id, v, 0x114, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(id, v, 0x118, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(id, v, 0x142, 0xa, 0xf, false));   // row_bcast:15 into rows 1 and 3
  v = op(v, __builtin_amdgcn_update_dpp(id, v, 0x143, 0xc, 0xf, false));   // row_bcast:31 into rows 2 and 3
  return v;
}

// Where tiles of an expert's rows begin: its first row, the rows after its last, and
// the tiles of `unit` rows, and of `wide` of those, that come before it.
struct Span {
  int expert, lo, hi, tiles, wides;
};

// Offsets are read as if each were raised to the largest before it and cut to [0, rows], so that the
// experts' rows never overlap and lie inside the matrix whatever they hold.  Sixty-four
// experts at a time: a lane each, running maxima and counts by scans.  find(index) asks for
// the expert that holds tile `index`, at(e) for expert e; total() counts all tiles.  Every
// lane of the wave takes part.
struct Experts {
  const int32_t *offsets;
  int experts, rows, unit;
  int lo, hi, tiles, first, wides, wfirst;    // the lane's expert of the group that is held
  int group, total;

  __device__ __forceinline__ void load(int g, int &top, int &count, int &wcount) {
    const int lane = threadIdx.x & 63, e = 64 * g + lane;
    auto cut = [&](int i) { return min(max(i <= experts ? offsets[i] : rows, 0), rows); };
    const int a = cut(min(e, experts)), b = cut(min(e + 1, experts));
    const auto larger = [](int x, int y) { return max(x, y); };
    const auto sum = [](int x, int y) { return x + y; };
    lo = max(scan64(a, larger, 0), top);
    hi = max(max(lo, b), top);
    tiles = e < experts ? (hi - lo + unit - 1) / unit : 0;
    wides = (tiles + kScalePad - 1) / kScalePad;
    const int t = scan64(tiles, sum, 0) + count, w = scan64(wides, sum, 0) + wcount;
    first = t - tiles;
    wfirst = w - wides;
    top = __builtin_amdgcn_readlane(hi, 63);
    count = __builtin_amdgcn_readlane(t, 63);
    wcount = __builtin_amdgcn_readlane(w, 63);
    group = g;
  }
  __device__ __forceinline__ Experts(const int32_t *off, int experts_, int rows_, int unit_)
      : offsets(off), experts(experts_), rows(rows_), unit(unit_) {
    if (!offsets) {
      total = (rows + unit - 1) / unit;
      return;
    }
    int top = 0, count = 0, wcount = 0;
    for (int g = 0; 64 * g < experts; ++g) load(g, top, count, wcount);
    total = count;
  }
  __device__ __forceinline__ Span take(int lane) const {
    return {64 * group + lane, __builtin_amdgcn_readlane(lo, lane), __builtin_amdgcn_readlane(hi, lane),
            __builtin_amdgcn_readlane(first, lane), __builtin_amdgcn_readlane(wfirst, lane)};
  }
  // the expert of tile `index` < total (wave-uniform)
  __device__ __forceinline__ Span find(int index) {
    if (!offsets) return {0, 0, rows, 0, 0};
    if (experts > 64) {
      int top = 0, count = 0, wcount = 0;
      for (int g = 0;; ++g) {
        load(g, top, count, wcount);
        if (index < count || 64 * (g + 1) >= experts) break;
      }
    }
    const uint64_t here = __ballot(index >= first && index < first + tiles);
    return take(here ? __builtin_ctzll(here) : 0);
  }
  __device__ __forceinline__ Span at(int expert) {
    if (!offsets) return {0, 0, rows, 0, 0};
    if (experts > 64) {
      int top = 0, count = 0, wcount = 0;
      for (int g = 0; g <= expert / 64; ++g) load(g, top, count, wcount);
    }
    return take(expert & 63);
  }
};

}  // namespace f8
}  // namespace fmm
