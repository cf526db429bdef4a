// Device side of the three activation types: loads and stores of eight
// consecutive elements at any element alignment.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/fmm8.h"

namespace fmm {
namespace q8 {

template <int T>
using elem_t = std::conditional_t<T == FMM_F32, float, std::conditional_t<T == FMM_BF16, __bf16, _Float16>>;

// 16 bytes at the alignment of the element: gfx950 takes unaligned global
// accesses, so a row of any width is read and written by whole vectors.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));

// two floats -> the bits of two 16-bit elements (round to nearest even)
template <int T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  static_assert(T != FMM_F32, "16-bit types");
  const elem_t<T> x = (elem_t<T>)a, y = (elem_t<T>)b;
  return (uint32_t)__builtin_bit_cast(uint16_t, x) | (uint32_t)__builtin_bit_cast(uint16_t, y) << 16;
}

template <int T>
__device__ __forceinline__ void unpack2(uint32_t w, float &a, float &b) {
  static_assert(T != FMM_F32, "16-bit types");
  if constexpr (T == FMM_BF16) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
  } else {
    a = (float)__builtin_bit_cast(_Float16, (uint16_t)w);
    b = (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
  }
}

// eight elements as they are stored
template <int T>
struct Raw8 {
  u32x4 w[T == FMM_F32 ? 2 : 1];
};

// p[0..7], with zeros from element n on (n may be <= 0)
template <int T>
__device__ __forceinline__ Raw8<T> raw8(const elem_t<T> *p, int64_t n) {
  Raw8<T> r;
  if (n >= 8) {
    if constexpr (T == FMM_F32) {
      r.w[0] = *reinterpret_cast<const u32x4_a4 *>(p);
      r.w[1] = *reinterpret_cast<const u32x4_a4 *>(p + 4);
    } else {
      r.w[0] = *reinterpret_cast<const u32x4_a2 *>(p);
    }
  } else if constexpr (T == FMM_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i / 4][i % 4] = i < n ? __float_as_uint(p[i]) : 0u;
  } else {
    const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r.w[0][i] = (uint32_t)(2 * i < n ? q[2 * i] : 0) | (uint32_t)(2 * i + 1 < n ? q[2 * i + 1] : 0) << 16;
  }
  return r;
}

template <int T>
__device__ __forceinline__ void floats8(const Raw8<T> &r, float (&v)[8]) {
  if constexpr (T == FMM_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i / 4][i % 4]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(r.w[0][i], v[2 * i], v[2 * i + 1]);
  }
}

template <int T>
__device__ __forceinline__ void load8(const elem_t<T> *p, int64_t n, float (&v)[8]) {
  floats8<T>(raw8<T>(p, n), v);
}

template <int T>
__device__ __forceinline__ void store8(elem_t<T> *p, int64_t n, const float (&v)[8]) {
  if (n >= 8) {
    if constexpr (T == FMM_F32) {
      u32x4 a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = __float_as_uint(v[i]);
        b[i] = __float_as_uint(v[4 + i]);
      }
      *reinterpret_cast<u32x4_a4 *>(p) = a;
      *reinterpret_cast<u32x4_a4 *>(p + 4) = b;
    } else {
      u32x4 a;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
      *reinterpret_cast<u32x4_a2 *>(p) = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (elem_t<T>)v[i];
  }
}

// four consecutive elements, of which those before n exist
template <int T>
__device__ __forceinline__ void store4(elem_t<T> *p, int n, const float (&v)[4]) {
  if (n >= 4) {
    if constexpr (T == FMM_F32) {
      u32x4 a;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]);
      *reinterpret_cast<u32x4_a4 *>(p) = a;
    } else {
      u32x2 a;
      a[0] = pack2<T>(v[0], v[1]);
      a[1] = pack2<T>(v[2], v[3]);
      *reinterpret_cast<u32x2_a2 *>(p) = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = (elem_t<T>)v[i];
  }
}

// eight int8 codes -> floats
__device__ __forceinline__ void codes8(u32x2 w, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = (float)(int8_t)(w[0] >> (8 * i));
    v[4 + i] = (float)(int8_t)(w[1] >> (8 * i));
  }
}

// ---- reductions over lanes ---------------------------------------------------
template <int N>
__device__ __forceinline__ uint32_t ror16(uint32_t v) {   // lane l of 16 takes lane (l - N) mod 16
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf, false);
}
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, ror16<8>(v));
  v = max(v, ror16<4>(v));
  v = max(v, ror16<2>(v));
  return max(v, ror16<1>(v));
}
__device__ __forceinline__ float sum16(float v) {
  v += __uint_as_float(ror16<8>(__float_as_uint(v)));
  v += __uint_as_float(ror16<4>(__float_as_uint(v)));
  v += __uint_as_float(ror16<2>(__float_as_uint(v)));
  return v + __uint_as_float(ror16<1>(__float_as_uint(v)));
}
__device__ __forceinline__ uint32_t max64(uint32_t v) {
  v = max16(v);
  v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return max(v, (uint32_t)__shfl_xor((int)v, 32));
}
__device__ __forceinline__ float sum64(float v) {
  v = sum16(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

}  // namespace q8
}  // namespace fmm
