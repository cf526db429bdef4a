// Rows of 8-bit codes: quantize, dequantize, the RMS norm with the residual's
// addition and an 8-bit output, and that norm's gradient.
//
// All of these move a few bytes an element and compute a few operations on
// them, so HBM bounds them: a row is read once into registers as fp32, its
// statistics are reduced across the row's threads, and its outputs are written
// from the same registers.
//
//   v_j = x_j (quantize) or h_j g_j with h = x + res in fp32 (norm)
//   a = max(amax |v|, floor),  q_j = rne(v_j (127 / a)),  s = a / 127
//   norm: rstd = (mean h^2 + eps)^-1/2, and the stored scale is s rstd: the
//   factor rstd of y = h rstd g is common to the row, so it cancels in the
//   codes, which therefore do not depend on the order the squares are summed in.
//   The checkpoint of h: the same rule over each group of 128 columns.
//   The floor is 1e-12 for a row to quantize, and for one that is zero.  In the norm
//   it is 2^-118, the least power of two whose 127 / a is far from infinity: rstd
//   makes rows of any size ones of order 1.
//
// A magnitude is compared by its bits, where NaN exceeds infinity exceeds every
// finite value: a row (or group) that holds one of the two gets scale NaN and
// zero codes.
//
// Geometry: TPR threads share a row and hold C chunks of eight consecutive
// columns each, chunk c of thread t at column 8 (c TPR + t), so that a wave
// reads consecutive 16-byte vectors and a checkpoint group is 16 consecutive
// lanes.  Rows of up to 1024 columns take a wave each (no barrier), longer ones
// as many threads as leave each 8 to 32 elements; where there are few rows, as
// many as the row has chunks, up to 1024, which is what a single token's latency
// wants.
//
// Measured: forward with residual and checkpoint, 8192 x 4096 bf16 51 us, 5.2 TB/s
// (the rate of a 1 GiB copy), 1024 x 8192 fp32 21, one token of 4096 3.4; gradient
// from the checkpoint with dh 51 (4.6 TB/s), 26 and 3.2.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "q8.h"
#include "q8_types.h"

namespace fmm {
namespace q8 {
namespace {

constexpr uint32_t kInfBits = 0x7f800000u;

__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct RowScale {
  float r;         // 127 / a
  float s;         // a / 127, NaN where the row holds NaN or infinity
  uint32_t keep;   // all ones, or zero there
};
template <bool NORM>
__device__ __forceinline__ RowScale row_scale(uint32_t amax_bits) {
  RowScale k;
  const bool bad = amax_bits >= kInfBits;
  const float a = bad ? 1.0f : fmaxf(__uint_as_float(amax_bits), NORM && amax_bits ? 0x1p-118f : 1e-12f);
  k.r = 127.0f / a;
  k.s = bad ? __uint_as_float(0x7fc00000u) : a / 127.0f;
  k.keep = bad ? 0u : ~0u;
  return k;
}

// Eight codes.  |v r| <= 127 (1 + 2^-23): adding 1.5 2^23 leaves the nearest
// integer (ties to even) in the low byte of the sum, in two's complement.
__device__ __forceinline__ u32x2 codes_of(const float (&v)[8], const RowScale &k) {
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(v[i] * k.r + 12582912.0f);
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u);
    w[i] = (lo | hi << 16) & k.keep;
  }
  return w;
}

// the row's (sum, largest magnitude) from each thread's part; `turn` alternates
// from row to row, so that a row's values outlive the next row's barrier
template <int TPR>
__device__ __forceinline__ void reduce_row(float &sum, uint32_t &m, int turn) {
  sum = sum64(sum);
  m = max64(m);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    __shared__ float ssum[2][W];
    __shared__ uint32_t smax[2][W];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) {
      ssum[turn][wave] = sum;
      smax[turn][wave] = m;
    }
    __syncthreads();
    sum = ssum[turn][0];
    m = smax[turn][0];
#pragma unroll
    for (int i = 1; i < W; ++i) {
      sum += ssum[turn][i];
      m = max(m, smax[turn][i]);
    }
  }
}

// The checkpoint of one chunk of h (16 lanes hold a group).
__device__ __forceinline__ void save_chunk(const float (&h)[8], int8_t *codes, float *scales, int64_t col, int64_t pitch) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, mag(h[i]));
  const RowScale k = row_scale<true>(max16(m));
  if (col < pitch) {
    *reinterpret_cast<u32x2 *>(codes + col) = codes_of(h, k);
    if ((threadIdx.x & 15) == 0) scales[col / kGroup] = k.s;
  }
}

template <int T, int TPR, int C, bool NORM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rows_kernel(RowArgs a) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  using E = elem_t<T>;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const E *gain = static_cast<const E *>(a.gain);
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB, turn ^= 1) {
    const bool live = row0 + sub < a.rows;   // (waves past the last row repeat it and store nothing)
    const int64_t row = live ? row0 + sub : a.rows - 1;
    const E *x = static_cast<const E *>(a.x) + row * a.cols;
    const E *res = static_cast<const E *>(a.res) + row * a.cols;
    float h[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = 8 * (int64_t)(c * TPR + t);
      load8<T>(x + col, a.cols - col, h[c]);
    }
    if (NORM && a.res) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int64_t col = 8 * (int64_t)(c * TPR + t);
        float r[8];
        load8<T>(res + col, a.cols - col, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] += r[i];
      }
    }
    if (NORM && a.h && live) {
      E *out = static_cast<E *>(a.h) + row * a.cols;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int64_t col = 8 * (int64_t)(c * TPR + t);
        store8<T>(out + col, a.cols - col, h[c]);
      }
    }
    float sum = 0.0f;
    uint32_t m = 0;
    if (NORM) {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += h[c][i] * h[c][i];
      if (a.saved) {
#pragma unroll
        for (int c = 0; c < C; ++c)
          save_chunk(h[c], a.saved + row * a.pitch, a.saved_scales + row * (a.pitch / kGroup), 8 * (int64_t)(c * TPR + t),
                     live ? a.pitch : 0);
      }
      if (gain) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int64_t col = 8 * (int64_t)(c * TPR + t);
          float g[8];
          load8<T>(gain + col, a.cols - col, g);
#pragma unroll
          for (int i = 0; i < 8; ++i) h[c][i] *= g[i];
        }
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, mag(h[c][i]));
    reduce_row<TPR>(sum, m, turn);
    const RowScale k = row_scale<NORM>(m);
    if (live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int64_t col = 8 * (int64_t)(c * TPR + t);
        if (col < a.pitch) *reinterpret_cast<u32x2 *>(a.codes + row * a.pitch + col) = codes_of(h[c], k);
      }
      if (t == 0) {
        if (NORM) {
          const float rstd = 1.0f / sqrtf(sum / (float)a.cols + a.eps);
          a.rstd[row] = rstd;
          a.scales[row] = k.s * rstd;
        } else {
          a.scales[row] = k.s;
        }
      }
    }
  }
}

// Rows too long for registers: the statistics (and h and its checkpoint) in one
// walk over the row, the codes in a second.
template <int T, bool NORM>
__global__ __launch_bounds__(1024) void long_rows_kernel(RowArgs a) {
  using E = elem_t<T>;
  const E *gain = static_cast<const E *>(a.gain);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const E *x = static_cast<const E *>(a.x) + row * a.cols;
    const E *res = static_cast<const E *>(a.res) + row * a.cols;
    auto chunk = [&](int64_t col, float (&h)[8]) {
      load8<T>(x + col, a.cols - col, h);
      if (NORM && a.res) {
        float r[8];
        load8<T>(res + col, a.cols - col, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += r[i];
      }
    };
    auto gained = [&](int64_t col, float (&h)[8]) {
      if (NORM && gain) {
        float g[8];
        load8<T>(gain + col, a.cols - col, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] *= g[i];
      }
    };
    float sum = 0.0f;
    uint32_t m = 0;
    for (int64_t col0 = 0; col0 < a.pitch; col0 += 8 * 1024) {   // (whole waves: the groups' reductions need their 16 lanes)
      const int64_t col = col0 + 8 * (int64_t)threadIdx.x;
      float h[8];
      chunk(col, h);
      if (NORM) {
        if (a.h) store8<T>(static_cast<E *>(a.h) + row * a.cols + col, a.cols - col, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += h[i] * h[i];
        if (a.saved) save_chunk(h, a.saved + row * a.pitch, a.saved_scales + row * (a.pitch / kGroup), col, a.pitch);
        gained(col, h);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, mag(h[i]));
    }
    reduce_row<1024>(sum, m, turn);
    const RowScale k = row_scale<NORM>(m);
    for (int64_t col = 8 * (int64_t)threadIdx.x; col < a.pitch; col += 8 * 1024) {
      float h[8];
      chunk(col, h);
      gained(col, h);
      *reinterpret_cast<u32x2 *>(a.codes + row * a.pitch + col) = codes_of(h, k);
    }
    if (threadIdx.x == 0) {
      if (NORM) {
        const float rstd = 1.0f / sqrtf(sum / (float)a.cols + a.eps);
        a.rstd[row] = rstd;
        a.scales[row] = k.s * rstd;
      } else {
        a.scales[row] = k.s;
      }
    }
  }
}

// ---- dequantize: eight columns a thread ------------------------------------------
template <int T>
__global__ __launch_bounds__(256) void dequantize_kernel(DequantArgs a) {
  using E = elem_t<T>;
  const int64_t chunks = (a.cols + 7) / 8, total = a.rows * chunks;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t row = e / chunks, col = 8 * (e - row * chunks);
    float v[8];
    codes8(*reinterpret_cast<const u32x2 *>(a.codes + row * a.pitch + col), v);
    const float s = a.grouped ? a.scales[row * (a.pitch / kGroup) + col / kGroup] : a.scales[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
    store8<T>(static_cast<E *>(a.out) + row * a.cols + col, a.cols - col, v);
  }
}

// ---- the norm's gradient ---------------------------------------------------------
// With xh = h rstd and w = dy g:  c = mean_j(w_j xh_j),
//   dx = rstd (w - xh c) + dh,   dg_j = sum over rows of dy_j xh_j.
// A workgroup keeps its columns' sums of dg in registers over the rows it
// walks; the workgroups' sums are added in order by a second kernel.

// h of one chunk: stored, or codes times their group's scale
template <int T, bool SAVED>
__device__ __forceinline__ void grad_h(const NormGradArgs &a, int64_t row, int64_t col, float (&h)[8]) {
  if (SAVED) {
    if (col < a.pitch) {
      codes8(*reinterpret_cast<const u32x2 *>(a.saved + row * a.pitch + col), h);
      const float s = a.saved_scales[row * (a.pitch / kGroup) + col / kGroup];
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = col + i < a.cols ? h[i] * s : 0.0f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = 0.0f;
    }
  } else {
    load8<T>(static_cast<const elem_t<T> *>(a.h) + row * a.cols + col, a.cols - col, h);
  }
}

template <int TPR>
__device__ __forceinline__ float reduce_sum(float v, int turn) {
  uint32_t none = 0;
  reduce_row<TPR>(v, none, turn);
  return v;
}

// What a row's gradient reads, as it is stored: the next row's is on its way
// while this one's is worked on (8192 x 4096 bf16 with dh: 80 us without, 50 with).
template <int T, int C, bool SAVED>
struct GradRow {
  Raw8<T> dy[C], dh[C], h[SAVED ? 1 : C];
  u32x2 q[SAVED ? C : 1];
  float s[SAVED ? C : 1], rstd;
};

// 1024 threads a row are 4 waves a SIMD, 128 registers each; the others may have 256.
template <int T, int TPR, int C, bool SAVED>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR, TPR == 1024 ? 4 : 2) void norm_grad_kernel(NormGradArgs a) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  using E = elem_t<T>;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const E *gain = static_cast<const E *>(a.gain);
  const E *dys = static_cast<const E *>(a.dy), *dhs = static_cast<const E *>(a.dh), *hs = static_cast<const E *>(a.h);
  auto column = [&](int c) { return 8 * (int64_t)(c * TPR + t); };
  auto fetch = [&](int64_t row, GradRow<T, C, SAVED> &r) {
    r.rstd = a.rstd[row];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = column(c);
      r.dy[c] = raw8<T>(dys + row * a.cols + col, a.cols - col);
      if (SAVED) {
        const bool in = col < a.pitch;
        r.q[c] = in ? *reinterpret_cast<const u32x2 *>(a.saved + row * a.pitch + col) : (u32x2){};
        r.s[c] = in ? a.saved_scales[row * (a.pitch / kGroup) + col / kGroup] : 0.0f;
      } else {
        r.h[c] = raw8<T>(hs + row * a.cols + col, a.cols - col);
      }
      if (a.dh) r.dh[c] = raw8<T>(dhs + row * a.cols + col, a.cols - col);
    }
  };
  float g[C][8], dg[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (gain) {
      load8<T>(gain + column(c), a.cols - column(c), g[c]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[c][i] = 1.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[c][i] = 0.0f;
  }
  const float inv = 1.0f / (float)a.cols;
  const int64_t stride = (int64_t)gridDim.x * RPB, first = (int64_t)blockIdx.x * RPB + sub;
  constexpr bool kAhead = TPR < 1024;   // (at 1024 threads a second row would spill)
  GradRow<T, C, SAVED> r, next;
  if (kAhead) fetch(min(first, a.rows - 1), r);
  int turn = 0;
  // (waves past the last row repeat it and keep nothing)
  for (int64_t row = first; row - sub < a.rows; row += stride, turn ^= 1) {
    const bool live = row < a.rows;
    if (!kAhead) fetch(min(row, a.rows - 1), r);
    else if (row - sub + stride < a.rows) fetch(min(row + stride, a.rows - 1), next);
    float xh[C][8], dot = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float dy[8];
      floats8<T>(r.dy[c], dy);
      if (SAVED) {
        codes8(r.q[c], xh[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) xh[c][i] *= r.s[c];   // (codes past the last column are zero, and so is dy there)
      } else {
        floats8<T>(r.h[c], xh[c]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xh[c][i] *= r.rstd;
        const float p = dy[i] * xh[c][i];
        if (live) dg[c][i] += p;
        dot += p * g[c][i];
      }
    }
    const float m = reduce_sum<TPR>(dot, turn) * inv;
    if (live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float dy[8], o[8];
        floats8<T>(r.dy[c], dy);
        if (a.dh) {
          floats8<T>(r.dh[c], o);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] += r.rstd * (dy[i] * g[c][i] - xh[c][i] * m);
        store8<T>(static_cast<E *>(a.dx) + row * a.cols + column(c), a.cols - column(c), o);
      }
    }
    if (kAhead) r = next;
  }
  if (a.dgain) {
    if constexpr (RPB > 1) {
      // the waves' sums meet first
      __shared__ float sums[RPB][C * TPR * 8];
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[sub][column(c) + i] = dg[c][i];
      __syncthreads();
      for (int64_t col = threadIdx.x; col < a.cols; col += 256) {
        float v = sums[0][col];
#pragma unroll
        for (int i = 1; i < RPB; ++i) v += sums[i][col];
        a.partial[(int64_t)blockIdx.x * a.cols + col] = v;
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
        store8<FMM_F32>(a.partial + (int64_t)blockIdx.x * a.cols + column(c), a.cols - column(c), dg[c]);
    }
  }
}

// Small gradients: one launch.  dg does not need c, so its column sums come from
// workgroups of their own, which read dy and h again (from the caches) rather
// than wait for a second kernel: one row of 4096 6.0 -> 3.2 us, 64 rows 6.8 -> 3.4,
// 512 rows 12.5 -> 7.8 (1000 of 1302 would take 18, 12 with partial sums).  A
// workgroup of those takes 8 LANES columns, LANES threads a row and 256 / LANES
// rows at a time.
template <int T, int TPR, int C, bool SAVED, int LANES>
__global__ __launch_bounds__(256) void small_norm_grad_kernel(NormGradArgs a, int row_blocks) {
  using E = elem_t<T>;
  const E *gain = static_cast<const E *>(a.gain), *dys = static_cast<const E *>(a.dy);
  if ((int)blockIdx.x >= row_blocks) {
    constexpr int ROWS = 256 / LANES;
    __shared__ float sums[4][8 * LANES];
    const int lane = threadIdx.x % LANES, first = threadIdx.x / LANES;
    const int64_t col = 8 * ((int64_t)(blockIdx.x - row_blocks) * LANES + lane);
    float dg[8] = {};
    // four rows' reads on their way at a time (rows past the last: its, times zero)
    for (int64_t row0 = first; row0 < a.rows; row0 += 4 * ROWS) {
      Raw8<T> dy[4], h[SAVED ? 1 : 4];
      u32x2 q[SAVED ? 4 : 1];
      float s[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t row = min(row0 + u * ROWS, a.rows - 1);
        dy[u] = raw8<T>(dys + row * a.cols + col, a.cols - col);
        s[u] = a.rstd[row];
        if (SAVED) {
          const bool in = col < a.pitch;
          q[u] = in ? *reinterpret_cast<const u32x2 *>(a.saved + row * a.pitch + col) : (u32x2){};
          s[u] *= in ? a.saved_scales[row * (a.pitch / kGroup) + col / kGroup] : 0.0f;
        } else {
          h[u] = raw8<T>(static_cast<const E *>(a.h) + row * a.cols + col, a.cols - col);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (row0 + u * ROWS >= a.rows) break;
        float d[8], x[8];
        floats8<T>(dy[u], d);
        if (SAVED) codes8(q[u], x);
        else floats8<T>(h[u], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[i] += d[i] * (x[i] * s[u]);
      }
    }
    // over a wave's rows, then the four waves'
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int o = LANES; o < 64; o *= 2) dg[i] += __shfl_xor(dg[i], o);
      if ((threadIdx.x & 63) < LANES) sums[threadIdx.x >> 6][8 * lane + i] = dg[i];
    }
    __syncthreads();
    const int64_t out = 8 * (int64_t)(blockIdx.x - row_blocks) * LANES + threadIdx.x;
    if (threadIdx.x < 8 * LANES && out < a.cols)
      a.dgain[out] = sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] + sums[3][threadIdx.x];
    return;
  }
  constexpr int RPB = 256 / TPR;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const int64_t want = (int64_t)blockIdx.x * RPB + sub, row = min(want, a.rows - 1);
  const float rstd = a.rstd[row];
  float w[C][8], xh[C][8], dot = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int64_t col = 8 * (int64_t)(c * TPR + t);
    load8<T>(dys + row * a.cols + col, a.cols - col, w[c]);
    grad_h<T, SAVED>(a, row, col, xh[c]);
  }
  if (gain) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = 8 * (int64_t)(c * TPR + t);
      float g[8];
      load8<T>(gain + col, a.cols - col, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[c][i] *= g[i];
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      xh[c][i] *= rstd;
      dot += w[c][i] * xh[c][i];
    }
  const float m = reduce_sum<TPR>(dot, 0) * (1.0f / (float)a.cols);
  if (want != row) return;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int64_t col = 8 * (int64_t)(c * TPR + t);
    float o[8] = {};
    if (a.dh) load8<T>(static_cast<const E *>(a.dh) + row * a.cols + col, a.cols - col, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] += rstd * (w[c][i] - xh[c][i] * m);
    store8<T>(static_cast<E *>(a.dx) + row * a.cols + col, a.cols - col, o);
  }
}

// Long rows: two walks for dx; the gain's sums come from a kernel of their own.
template <int T, bool SAVED>
__global__ __launch_bounds__(1024) void long_norm_grad_kernel(NormGradArgs a) {
  using E = elem_t<T>;
  const E *gain = static_cast<const E *>(a.gain);
  const float inv = 1.0f / (float)a.cols;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const float rstd = a.rstd[row];
    auto chunk = [&](int64_t col, float (&w)[8], float (&xh)[8]) {
      load8<T>(static_cast<const E *>(a.dy) + row * a.cols + col, a.cols - col, w);
      grad_h<T, SAVED>(a, row, col, xh);
      if (gain) {
        float g[8];
        load8<T>(gain + col, a.cols - col, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] *= g[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) xh[i] *= rstd;
    };
    float dot = 0.0f;
    for (int64_t col = 8 * (int64_t)threadIdx.x; col < a.cols; col += 8 * 1024) {
      float w[8], xh[8];
      chunk(col, w, xh);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot += w[i] * xh[i];
    }
    const float m = reduce_sum<1024>(dot, turn) * inv;
    for (int64_t col = 8 * (int64_t)threadIdx.x; col < a.cols; col += 8 * 1024) {
      float w[8], xh[8], o[8];
      chunk(col, w, xh);
      if (a.dh) {
        load8<T>(static_cast<const E *>(a.dh) + row * a.cols + col, a.cols - col, o);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] += rstd * (w[i] - xh[i] * m);
      store8<T>(static_cast<E *>(a.dx) + row * a.cols + col, a.cols - col, o);
    }
  }
}

// the sums of dy xh over each block's rows, columns 2048 blockIdx.y + 8 t ..
template <int T, bool SAVED>
__global__ __launch_bounds__(256) void long_gain_grad_kernel(NormGradArgs a) {
  const int64_t col = 2048 * (int64_t)blockIdx.y + 8 * (int64_t)threadIdx.x;
  if (col >= a.cols) return;
  float dg[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dg[i] = 0.0f;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float dy[8], h[8];
    load8<T>(static_cast<const elem_t<T> *>(a.dy) + row * a.cols + col, a.cols - col, dy);
    grad_h<T, SAVED>(a, row, col, h);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[i] += dy[i] * (h[i] * rstd);
  }
  store8<FMM_F32>(a.partial + (int64_t)blockIdx.x * a.cols + col, a.cols - col, dg);
}

// out[j] = sum over n rows of partial[row][j]: ascending within each of 32
// interleaved sets of rows, whose sums are then added in order
__global__ __launch_bounds__(1024) void sum_partials_kernel(const float *__restrict__ partial, float *__restrict__ out,
                                                            int64_t n, int64_t cols) {
  __shared__ float part[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int64_t col = 32 * (int64_t)blockIdx.x + x;
  float s = 0.0f;
  if (col < cols) {
#pragma unroll 8
    for (int64_t r = y; r < n; r += 32) s += partial[r * cols + col];
  }
  part[y][x] = s;
  __syncthreads();
  if (y == 0 && col < cols) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += part[i][x];
    out[col] = s;
  }
}

// ---- geometry --------------------------------------------------------------------
constexpr int64_t kMaxBlocks = 1 << 20;   // (blocks times 1024 threads stay under the launch limit)
constexpr int64_t kFewRows = 512;         // up to two rows a compute unit: a row takes all the threads it can use

struct Geometry {
  int tpr, c;
};
Geometry geometry(int64_t rows, int64_t cols) {
  if (cols > kMaxHeldCols) return {0, 0};
  const bool few = rows <= kFewRows;
  if (cols <= 512) return {64, 1};
  if (cols <= 1024 && !few) return {64, 2};
  if (cols <= 2048) return {256, 1};
  if (cols <= 8192 && few) return {1024, 1};
  if (cols <= 4096) return {256, 2};
  if (cols <= 8192) return {256, 4};
  if (cols <= 16384) return {1024, 2};
  return {1024, 4};
}

template <int T, bool NORM>
void launch_rows(const RowArgs &a, hipStream_t s) {
  const Geometry g = geometry(a.rows, a.cols);
  const int rpb = g.tpr == 64 ? 4 : 1;
  const dim3 grid((unsigned)std::min<int64_t>((a.rows + rpb - 1) / rpb, kMaxBlocks));
  if (g.tpr == 0) long_rows_kernel<T, NORM><<<grid, 1024, 0, s>>>(a);
  else if (g.tpr == 64 && g.c == 1) rows_kernel<T, 64, 1, NORM><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 64) rows_kernel<T, 64, 2, NORM><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 256 && g.c == 1) rows_kernel<T, 256, 1, NORM><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 256 && g.c == 2) rows_kernel<T, 256, 2, NORM><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 256) rows_kernel<T, 256, 4, NORM><<<grid, 256, 0, s>>>(a);
  else if (g.c == 1) rows_kernel<T, 1024, 1, NORM><<<grid, 1024, 0, s>>>(a);
  else if (g.c == 2) rows_kernel<T, 1024, 2, NORM><<<grid, 1024, 0, s>>>(a);
  else rows_kernel<T, 1024, 4, NORM><<<grid, 1024, 0, s>>>(a);
}

template <bool NORM>
int launch_rows_typed(int type, const RowArgs &a, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == FMM_F32) launch_rows<FMM_F32, NORM>(a, s);
  else if (type == FMM_BF16) launch_rows<FMM_BF16, NORM>(a, s);
  else launch_rows<FMM_F16, NORM>(a, s);
  return hipGetLastError();
}

// A gradient holds more a thread, so at most two chunks each; rows of more than
// 16384 columns are read twice.
Geometry grad_geometry(int64_t cols) {
  if (cols <= 512) return {64, 1};
  if (cols <= 1024) return {64, 2};
  if (cols <= 2048) return {256, 1};
  if (cols <= 4096) return {256, 2};
  if (cols <= 8192) return {512, 2};
  if (cols <= 16384) return {1024, 2};
  return {0, 0};
}
// The workgroups that share the rows: two of 256 threads a compute unit, or three
// where that leaves each eight rows or more and their registers fit (16-bit rows).
// More of them leave more partial sums.  bf16 8192 x 4096: 52 us with 512, 47 with
// 768, 59 with 1024; 700 x 4096 13.8 with 512, 16.2 with 700; fp32 4096 x 4096 39
// with 512, 43 with 768.
int64_t grad_blocks(int type, int64_t rows, int64_t cols) {
  const Geometry g = grad_geometry(cols);
  const int64_t units = g.tpr == 64 ? (rows + 3) / 4 : rows;
  const bool three = g.tpr != 0 && g.tpr <= 256 && type != FMM_F32 && units >= 8 * 768;
  const int64_t most = g.tpr == 0 ? 64 : three ? 768 : 512 * 256 / std::max(g.tpr, 256);
  return std::max<int64_t>(1, std::min(units, most));
}

// One launch up to here: at most 8 rows a thread in the columns' workgroups, two
// round trips to memory.
bool small_grad(int64_t rows, int64_t cols) { return rows > 0 && rows <= kFewRows && cols <= 8192; }

template <int T, int TPR, int C, bool SAVED>
void launch_small(const NormGradArgs &a, hipStream_t s) {
  constexpr int RPB = 256 / TPR;
  const int rows = (int)((a.rows + RPB - 1) / RPB), chunks = (int)((a.cols + 7) / 8);
  const int wide = a.dgain ? (chunks + 7) / 8 : 0, narrow = a.dgain ? (chunks + 3) / 4 : 0;
  if (a.rows <= 128) small_norm_grad_kernel<T, TPR, C, SAVED, 8><<<dim3((unsigned)(rows + wide)), 256, 0, s>>>(a, rows);
  else small_norm_grad_kernel<T, TPR, C, SAVED, 4><<<dim3((unsigned)(rows + narrow)), 256, 0, s>>>(a, rows);
}

template <int T, bool SAVED>
void launch_grad(const NormGradArgs &a, hipStream_t s) {
  if (small_grad(a.rows, a.cols)) {
    if (a.cols <= 512) launch_small<T, 64, 1, SAVED>(a, s);
    else if (a.cols <= 1024) launch_small<T, 64, 2, SAVED>(a, s);
    else if (a.cols <= 2048) launch_small<T, 256, 1, SAVED>(a, s);
    else if (a.cols <= 4096) launch_small<T, 256, 2, SAVED>(a, s);
    else launch_small<T, 256, 4, SAVED>(a, s);
    return;
  }
  const Geometry g = grad_geometry(a.cols);
  const int64_t blocks = a.rows > 0 ? grad_blocks(T, a.rows, a.cols) : 0;
  const dim3 grid((unsigned)blocks);
  if (blocks == 0) {
    // no rows: the gain's sums are empty
  } else if (g.tpr == 0) {
    const int64_t rb = std::min<int64_t>(a.rows, kMaxBlocks);
    long_norm_grad_kernel<T, SAVED><<<dim3((unsigned)rb), 1024, 0, s>>>(a);
    if (a.dgain)
      long_gain_grad_kernel<T, SAVED><<<dim3((unsigned)blocks, (unsigned)((a.cols + 2047) / 2048)), 256, 0, s>>>(a);
  } else if (g.tpr == 64 && g.c == 1) norm_grad_kernel<T, 64, 1, SAVED><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 64) norm_grad_kernel<T, 64, 2, SAVED><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 256 && g.c == 1) norm_grad_kernel<T, 256, 1, SAVED><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 256) norm_grad_kernel<T, 256, 2, SAVED><<<grid, 256, 0, s>>>(a);
  else if (g.tpr == 512) norm_grad_kernel<T, 512, 2, SAVED><<<grid, 512, 0, s>>>(a);
  else norm_grad_kernel<T, 1024, 2, SAVED><<<grid, 1024, 0, s>>>(a);
  if (a.dgain)
    sum_partials_kernel<<<dim3((unsigned)((a.cols + 31) / 32)), 1024, 0, s>>>(a.partial, a.dgain, blocks, a.cols);
}

template <int T>
void launch_grad_source(const NormGradArgs &a, hipStream_t s) {
  if (a.h) launch_grad<T, false>(a, s);
  else launch_grad<T, true>(a, s);
}

}  // namespace

int launch_quantize(int type, const RowArgs &a, void *stream) { return launch_rows_typed<false>(type, a, stream); }
int launch_rmsnorm(int type, const RowArgs &a, void *stream) { return launch_rows_typed<true>(type, a, stream); }

int launch_dequantize(int type, const DequantArgs &a, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t total = a.rows * ((a.cols + 7) / 8);
  const dim3 grid((unsigned)std::min<int64_t>((total + 255) / 256, kMaxBlocks));
  if (type == FMM_F32) dequantize_kernel<FMM_F32><<<grid, 256, 0, s>>>(a);
  else if (type == FMM_BF16) dequantize_kernel<FMM_BF16><<<grid, 256, 0, s>>>(a);
  else dequantize_kernel<FMM_F16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

int64_t norm_grad_partials(int type, int64_t rows, int64_t cols) {
  return small_grad(rows, cols) ? 0 : grad_blocks(type, rows, cols);
}

int launch_rmsnorm_grad(int type, const NormGradArgs &a, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == FMM_F32) launch_grad_source<FMM_F32>(a, s);
  else if (type == FMM_BF16) launch_grad_source<FMM_BF16>(a, s);
  else launch_grad_source<FMM_F16>(a, s);
  return hipGetLastError();
}

}  // namespace q8
}  // namespace fmm
