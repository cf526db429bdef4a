// The linear layer's gradients from its 8-bit operands:
//   dX = (dY * sw) Qw   (M x K, contracted over N),
//   dW = (dY * sa)^T Qa (N x K, contracted over M),  dbias = column sums of dY.
//
// int8 codes are exact in bfloat16, so the bf16 matrix cores multiply them by
// dY directly; what has to be rounded is a product with a scale.
//   bf16 dY: the scale goes to the codes, bf16(q s), dY itself being exact (one
//     rounding, half an ulp of bf16, of one operand: the error is about that of
//     rounding the result to bf16).
//   fp16 and fp32 dY: the scale goes to dY, and dY s is written as the sum of two
//     or three bfloat16 parts (16 and 24 significant bits) along a longer
//     contracted axis, the codes staying exact.
//
// Two launches, or three.  The first lays the operands out along the contracted axes
// (transposes through LDS, converted on the way, padded with zeros to the
// product's 64-position step) and leaves dY's column sums by 64-row tiles.  It moves
// 3 bytes a code (1 in, 2 out) and, for an element of dY, 4 bytes in bf16 (6 where
// N is no multiple of 64: dY by rows as well), 10 in fp16 and 16 in fp32: 470 MB in 95
// of 910 us for 8192 x 8192 x 4096 bf16, 16 MB in 6.4 of 17 for 256 x 2048 x 2048, 31 MB
// in 10.4 of 41 for 1000 x 1302 x 1472 fp32.  The second runs both products' tiles and adds up the column
// sums.  Where a product has few tiles and a long axis, its tiles' axis is split
// into runs, and the third adds the runs' sums.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "q8_gemm.h"

namespace fmm {
namespace q8 {
namespace {

constexpr int kPos = 64;   // bf16 positions of a step

template <int T>
constexpr int kParts = T == FMM_BF16 ? 1 : T == FMM_F16 ? 2 : 3;

struct LayoutArgs {
  const void *dy;
  const int8_t *a, *w;
  const float *sa, *sw;
  uint16_t *dyt;      // [parts][N][Mp]: dY^T
  uint16_t *dyr;      // [parts][M][Np]: dY by rows (null: dY itself serves)
  uint16_t *at, *wt;  // [K][Mp], [K][Np]
  float *colsum;      // [M / 64][N]
  int64_t M, N, K, Mp, Np, pitch;
  int bm, bn, bk;     // 64-wide tiles of each axis
  int jobs_dy, jobs_a, jobs_w;   // blocks of each job
  int want_dx, want_dw, want_db;
};

__device__ __forceinline__ uint16_t bf16_bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// part p of v: bf16 of what the parts before leave.  EVERY: any v, else finite ones
// that bf16 does not round to infinity.  A finite v that it would is cut towards zero
// instead, and what is left of it too: the parts' sum then never exceeds v on its way.
constexpr uint32_t kFirstCut = 0x7f7f8000u;
template <int P, bool EVERY>
__device__ __forceinline__ void split_parts(float v, uint16_t (&out)[P]) {
  const uint32_t mag = __float_as_uint(v) & 0x7fffffffu;
  const bool finite = mag < 0x7f800000u, cut = finite && mag >= kFirstCut;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    out[p] = EVERY && cut ? (uint16_t)(__float_as_uint(v) >> 16) : bf16_bits(v);
    const float r = v - bf16_value(out[p]);
    v = EVERY && !finite ? 0.0f : r;   // (nothing is left of NaN and infinity)
  }
}

// q s of large scales.  A row quantized from the largest float has codes whose q s lies between it and
// 2^128 and is rounded to infinity: that is the largest float here.
__device__ __forceinline__ float code_value(float q, float s) {
  const float v = q * s;
  return fabsf(q * (0.5f * s)) <= 0x1p127f ? fminf(fmaxf(v, -0x1.fffffep127f), 0x1.fffffep127f) : v;
}

// 16 consecutive values of each part to dst + part * plane
template <int P>
__device__ __forceinline__ void store_parts(const float (&v)[16], uint16_t *dst, int64_t plane) {
  uint16_t b[16][P];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
  if (most < kFirstCut) {
#pragma unroll
    for (int i = 0; i < 16; ++i) split_parts<P, false>(v[i], b[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) split_parts<P, true>(v[i], b[i]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    u32x4 o[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i / 4][i % 4] = (uint32_t)b[2 * i][p] | (uint32_t)b[2 * i + 1][p] << 16;
    u32x4 *out = reinterpret_cast<u32x4 *>(dst + p * plane);
    out[0] = o[0];
    out[1] = o[1];
  }
}

// One 64 x 64 tile a workgroup: thread t reads 16 columns of row t / 4 and
// writes 16 rows of column t / 4.  LDS rows of 65 floats: both directions fall
// on distinct banks.
template <int T>
__global__ __launch_bounds__(256) void layout_kernel(LayoutArgs g) {
  constexpr int P = kParts<T>;
  __shared__ float tile[64][65];
  const int t = threadIdx.x, r = t >> 2, c = (t & 3) * 16;
  int id = blockIdx.x;
  if (id < g.jobs_dy) {
    // dY: rows m, columns n
    using E = elem_t<T>;
    const int64_t m0 = 64 * (int64_t)(id / g.bn), n0 = 64 * (int64_t)(id % g.bn);
    float v[16];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float x[8];
      const int64_t n = n0 + c + 8 * u;
      load8<T>(static_cast<const E *>(g.dy) + (m0 + r) * g.N + n, m0 + r < g.M ? g.N - n : 0, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[8 * u + i] = x[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) tile[r][c + i] = v[i];
    if (g.dyr && g.want_dx && m0 + r < g.M) {
      if (P > 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= n0 + c + i < g.N ? g.sw[n0 + c + i] : 0.0f;
      }
      store_parts<P>(v, g.dyr + (m0 + r) * g.Np + n0 + c, g.M * g.Np);
    }
    __syncthreads();
    const int64_t n = n0 + r;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      v[i] = tile[c + i][r];
      s += v[i];
    }
    s += __shfl_xor(s, 1);
    s += __shfl_xor(s, 2);
    if (g.want_db && (t & 3) == 0 && n < g.N) g.colsum[(m0 / 64) * g.N + n] = s;
    if (g.want_dw && n < g.N) {
      if (P > 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= m0 + c + i < g.M ? g.sa[m0 + c + i] : 0.0f;
      }
      store_parts<P>(v, g.dyt + n * g.Mp + m0 + c, g.N * g.Mp);
    }
    return;
  }
  // codes: rows x K -> K x rows
  id -= g.jobs_dy;
  const bool is_a = id < g.jobs_a;
  if (!is_a) id -= g.jobs_a;
  const int8_t *q = is_a ? g.a : g.w;
  const float *sc = is_a ? g.sa : g.sw;
  uint16_t *out = is_a ? g.at : g.wt;
  const int64_t rows = is_a ? g.M : g.N, rp = is_a ? g.Mp : g.Np;
  const int64_t r0 = 64 * (int64_t)(id / g.bk), k0 = 64 * (int64_t)(id % g.bk);
  float v[16];
  if (r0 + r < rows) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(q + (r0 + r) * g.pitch + k0 + c);
    const float s = P == 1 ? sc[r0 + r] : 1.0f;   // (else it goes to dY)
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4)));
    if (P == 1 && fabsf(s) > 0x1p119f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = code_value(v[i], s);
    } else if (P == 1) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] *= s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.0f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) tile[r][c + i] = v[i];
  __syncthreads();
  const int64_t k = k0 + r;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = tile[c + i][r];
  if (k < g.K) store_parts<1>(v, out + k * rp + r0 + c, 0);
}

struct GradGemms {
  GemmProblem p[2];
  int items0, items;         // blocks of p[0], of both
  const float *colsum;
  float *dbias;
  int64_t N;
  int tiles;                 // rows of colsum
};

// Tiles TX of dX and TW of dW (equal workgroups).
template <class TX, class TW, int OUT>
__global__ __launch_bounds__(TX::kThreads, 2) void grad_kernel(GradGemms g) {
  static_assert(TX::kThreads == TW::kThreads, "one launch");
  __shared__ uint4 lds[(TX::kLds > TW::kLds ? TX::kLds : TW::kLds) / 16];
  const int id = blockIdx.x;
  if (id < g.items) {
    if (id < g.items0) gemm_tile<Bf16, TX, OUT>(g.p[0], id, lds);
    else gemm_tile<Bf16, TW, OUT>(g.p[1], id - g.items0, lds);
    return;
  }
  const int64_t n = (int64_t)(id - g.items) * TX::kThreads + threadIdx.x;
  if (n >= g.N) return;
  float s = 0.0f;
#pragma unroll 4
  for (int i = 0; i < g.tiles; ++i) s += g.colsum[(int64_t)i * g.N + n];
  g.dbias[n] = s;
}

// The sums of a split product's runs, added in order, eight elements a thread.
template <int OUT>
__device__ __forceinline__ void add_runs(const GemmProblem &p, int64_t at) {
  const int64_t n = (int64_t)p.M * p.N;
  float v[8], w[8];
  load8<FMM_F32>(p.partial + at, n - at, v);
  for (int s = 1; s < p.splits; ++s) {
    load8<FMM_F32>(p.partial + s * n + at, n - at, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += w[i];
  }
  store8<OUT>(static_cast<elem_t<OUT> *>(p.C) + at, n - at, v);
}
template <int OUT>
__global__ __launch_bounds__(256) void add_runs_kernel(GradGemms g, int64_t chunks0, int64_t chunks) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e < chunks0) add_runs<OUT>(g.p[0], 8 * e);
  else if (e < chunks) add_runs<OUT>(g.p[1], 8 * (e - chunks0));
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {
  size_t dyt, dyr, at, wt, colsum, total;
  bool rows;   // dY is laid out by rows too
};
Layout layout_of(int type, int64_t M, int64_t N, int64_t K) {
  const int64_t Mp = round_up(M, kPos), Np = round_up(N, kPos);
  const int parts = type == FMM_BF16 ? 1 : type == FMM_F16 ? 2 : 3;
  Layout l;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at = align256(at + (size_t)bytes);
    return here;
  };
  l.rows = parts > 1 || N % kPos != 0;
  l.dyt = take(2 * parts * N * Mp);
  l.dyr = take(l.rows ? 2 * parts * M * Np : 0);
  l.at = take(2 * K * Mp);
  l.wt = take(2 * K * Np);
  l.colsum = take(4 * (Mp / 64) * N);
  l.total = at;
  return l;
}

// How the products are cut: the tile of each, and the runs that its contracted
// axis is split into.
struct Cut {
  int tile[2];     // 0: 64, 1: 128, 2: 256, 3: 128 with the longer ring (2 and 3 of both, or
                   // neither: their workgroups are larger)
  int splits[2];
};

// t = max(start + chain steps of a run, of either; start + work of both / CUs) us,
// a product's work being its tile's `work` times steps and tiles; runs cost a launch
// and the traffic of their sums besides.  The form is the int8 product's (a step moves
// and multiplies as much).  Against all cuts (up to 24 of them a shape, drawn where
// there are more) on 1917 shapes of the three types, with either product and with both:
// 3.6% over the fastest on average, more than 10% on 13% of them, 59% at worst (11874 x
// 323 x 4468 fp16, 358 us for 225 with dW in four runs: dW's tiles come after dX's, so
// that a long chain of theirs begins late, which the cost does not know).
// Without runs few tiles with a long axis leave most of the chip idle: 8192 tokens of
// 512 x 512 channels 42 -> 32 us, of 1024 x 1024 87 -> 65 to 69.  A tile for each, not
// one for both: 2000 tokens of 300 x 2000 in fp16 37.6 -> 32.1.  The longer ring where
// each CU has a workgroup at most: 1000 x 1302 x 1472 fp32 49 -> 43, 2048^3 bf16 54 ->
// 47; but 13436 tokens of 2023 x 124 69 -> 74.
Cut cut_of(const int64_t (&m)[2], const int64_t (&n)[2], const int64_t (&steps)[2], int ncu) {
  constexpr int kEdge[4] = {64, 128, 256, 128};
  constexpr double kStart[4] = {3.2, 4.5, 7.5, 4.0}, kChain[4] = {0.20, 0.47, 1.2, 0.36},
                   kWork[4] = {0.29, 0.60, 2.0, 0.36};
  constexpr double kMostSums = 1 << 24;   // floats of sums: 64 MB
  double tiles[2][4], work[2][4];
  for (int k = 0; k < 2; ++k)
    for (int i = 0; i < 4; ++i) {
      tiles[k][i] = (double)((m[k] + kEdge[i] - 1) / kEdge[i]) * (double)((n[k] + kEdge[i] - 1) / kEdge[i]);
      work[k][i] = kWork[i] * steps[k] * tiles[k][i] / ncu;
    }
  Cut best = {};
  double least = 1e300;
  for (int t0 = 0; t0 < 4; ++t0)
    for (int t1 = 0; t1 < 4; ++t1) {
      if (t0 != t1 && (t0 > 1 || t1 > 1)) continue;
      const double busy = std::max(m[0] ? kStart[t0] : 0, m[1] ? kStart[t1] : 0) + work[0][t0] + work[1][t1];
      for (int s0 = 1; s0 <= 16; s0 *= 2)
        for (int s1 = 1; s1 <= 16; s1 *= 2) {
          if ((s0 > 1 && s0 * 4 > steps[0]) || (s1 > 1 && s1 * 4 > steps[1])) continue;
          if (t0 == 3 && s0 * tiles[0][3] + s1 * tiles[1][3] > ncu) continue;
          const double sums = (s0 > 1 ? (double)m[0] * n[0] * s0 : 0) + (s1 > 1 ? (double)m[1] * n[1] * s1 : 0);
          if (sums > kMostSums) continue;
          const double chain = std::max(kStart[t0] + kChain[t0] * ((steps[0] + s0 - 1) / s0),
                                        kStart[t1] + kChain[t1] * ((steps[1] + s1 - 1) / s1));
          const double t = std::max(chain, busy) + (sums > 0 ? 3.0 + sums * 8 / 4e6 : 0);
          if (t < least) {
            least = t;
            best = {{t0, t1}, {s0, s1}};
          }
        }
    }
  return best;
}

// (a product that is not wanted has no rows and no steps: it is left in one run)
Cut cut_of(int type, int64_t M, int64_t N, int64_t K, bool dx, bool dw, int ncu) {
  const int64_t parts = type == FMM_BF16 ? 1 : type == FMM_F16 ? 2 : 3;
  return cut_of({dx ? M : 0, dw ? N : 0}, {K, K},
                {dx ? parts * ((N + kPos - 1) / kPos) : 0, dw ? parts * ((M + kPos - 1) / kPos) : 0}, ncu);
}

template <int T, class TX, class TW>
void launch_gemms(GradGemms g, const GradArgs &a, hipStream_t s) {
  constexpr int kEdge[2] = {TX::TM, TW::TM};
  for (int i = 0; i < 2; ++i) {
    g.p[i].tiles_m = (g.p[i].M + kEdge[i] - 1) / kEdge[i];
    g.p[i].tiles_n = (g.p[i].N + kEdge[i] - 1) / kEdge[i];
  }
  const int64_t dx = a.dx ? (int64_t)g.p[0].tiles_m * g.p[0].tiles_n * g.p[0].splits : 0;
  const int64_t dw = a.dw ? (int64_t)g.p[1].tiles_m * g.p[1].tiles_n * g.p[1].splits : 0;
  const int64_t db = a.dbias ? (a.N + TX::kThreads - 1) / TX::kThreads : 0;
  g.items0 = (int)dx;
  g.items = (int)(dx + dw);
  if (dx + dw + db > 0) grad_kernel<TX, TW, T><<<dim3((unsigned)(dx + dw + db)), TX::kThreads, 0, s>>>(g);
  int64_t chunks[2];
  for (int i = 0; i < 2; ++i)
    chunks[i] = (i ? dw : dx) > 0 && g.p[i].splits > 1 ? ((int64_t)g.p[i].M * g.p[i].N + 7) / 8 : 0;
  const int64_t all = chunks[0] + chunks[1];
  if (all > 0) add_runs_kernel<T><<<dim3((unsigned)((all + 255) / 256)), 256, 0, s>>>(g, chunks[0], all);
}

template <int T>
int launch(const GradArgs &a, int ncu, hipStream_t s) {
  const Layout l = layout_of(T, a.M, a.N, a.K);
  LayoutArgs g = {};
  g.dy = a.dy; g.a = a.a; g.w = a.w; g.sa = a.sa; g.sw = a.sw;
  g.dyt = reinterpret_cast<uint16_t *>(a.ws + l.dyt);
  g.dyr = l.rows ? reinterpret_cast<uint16_t *>(a.ws + l.dyr) : nullptr;
  g.at = reinterpret_cast<uint16_t *>(a.ws + l.at);
  g.wt = reinterpret_cast<uint16_t *>(a.ws + l.wt);
  g.colsum = reinterpret_cast<float *>(a.ws + l.colsum);
  g.M = a.M; g.N = a.N; g.K = a.K;
  g.Mp = round_up(a.M, kPos); g.Np = round_up(a.N, kPos); g.pitch = pitch_of(a.K);
  g.bm = (int)(g.Mp / 64); g.bn = (int)(g.Np / 64); g.bk = (int)((a.K + 63) / 64);
  g.want_dx = a.dx != nullptr; g.want_dw = a.dw != nullptr; g.want_db = a.dbias != nullptr;
  g.jobs_dy = g.want_dw || g.want_db || (g.want_dx && l.rows) ? g.bm * g.bn : 0;
  g.jobs_a = g.want_dw ? g.bm * g.bk : 0;
  g.jobs_w = g.want_dx ? g.bn * g.bk : 0;
  const int jobs = g.jobs_dy + g.jobs_a + g.jobs_w;
  if (jobs > 0) layout_kernel<T><<<dim3((unsigned)jobs), 256, 0, s>>>(g);

  constexpr int P = kParts<T>;
  GradGemms q = {};
  GemmProblem &x = q.p[0], &w = q.p[1];
  x.A = l.rows ? reinterpret_cast<const uint8_t *>(g.dyr) : static_cast<const uint8_t *>(a.dy);
  x.pitch_a = 2 * g.Np; x.part_a = 2 * a.M * g.Np;
  x.B = reinterpret_cast<const uint8_t *>(g.wt); x.pitch_b = 2 * g.Np;
  x.C = a.dx; x.M = (int)a.M; x.N = (int)a.K; x.steps = g.bn; x.parts = P;
  w.A = reinterpret_cast<const uint8_t *>(g.dyt);
  w.pitch_a = 2 * g.Mp; w.part_a = 2 * a.N * g.Mp;
  w.B = reinterpret_cast<const uint8_t *>(g.at); w.pitch_b = 2 * g.Mp;
  w.C = a.dw; w.M = (int)a.N; w.N = (int)a.K; w.steps = g.bm; w.parts = P;
  q.colsum = g.colsum; q.dbias = a.dbias; q.N = a.N; q.tiles = g.bm;
  const Cut cut = cut_of(T, a.M, a.N, a.K, a.dx, a.dw, ncu);
  x.splits = cut.splits[0];
  w.splits = cut.splits[1];
  x.partial = reinterpret_cast<float *>(a.ws + l.total);
  w.partial = x.partial + (x.splits > 1 ? (int64_t)x.splits * a.M * a.K : 0);
  if (cut.tile[0] == 2) launch_gemms<T, Tile256, Tile256>(q, a, s);
  else if (cut.tile[0] == 3) launch_gemms<T, Tile128Ahead, Tile128Ahead>(q, a, s);
  else if (cut.tile[0] == 1 && cut.tile[1] == 1) launch_gemms<T, Tile128, Tile128>(q, a, s);
  else if (cut.tile[0] == 1) launch_gemms<T, Tile128, Tile64>(q, a, s);
  else if (cut.tile[1] == 1) launch_gemms<T, Tile64, Tile128>(q, a, s);
  else launch_gemms<T, Tile64, Tile64>(q, a, s);
  return hipGetLastError();
}

}  // namespace

// (what is wanted is not known here: the most that any choice of it takes)
size_t grad_scratch(int type, int64_t M, int64_t N, int64_t K, int ncu) {
  size_t sums = 0;
  for (int want = 1; want < 4; ++want) {
    const Cut c = cut_of(type, M, N, K, want & 1, want & 2, ncu);
    size_t n = 0;
    if ((want & 1) && c.splits[0] > 1) n += sizeof(float) * c.splits[0] * M * K;
    if ((want & 2) && c.splits[1] > 1) n += sizeof(float) * c.splits[1] * N * K;
    sums = std::max(sums, n);
  }
  return layout_of(type, M, N, K).total + align256(sums);
}

const char *linear_grad_kernel_name(int type, int64_t M, int64_t N, int64_t K, bool dx, bool dw, int ncu, int32_t *runs) {
  static const char *const small[2][2] = {{"grad_kernel 64x64 64x64", "grad_kernel 64x64 128x128"},
                                          {"grad_kernel 128x128 64x64", "grad_kernel 128x128 128x128"}};
  const Cut c = cut_of(type, M, N, K, dx, dw, ncu);
  if (runs) {
    runs[0] = c.splits[0];
    runs[1] = c.splits[1];
  }
  if (c.tile[0] == 2) return "grad_kernel 256x256 256x256";
  if (c.tile[0] == 3) return "grad_kernel 128x128 128x128 ahead";
  return small[c.tile[0]][c.tile[1]];
}

int launch_linear_grad(int type, const GradArgs &a, int ncu, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == FMM_F32) return launch<FMM_F32>(a, ncu, s);
  if (type == FMM_BF16) return launch<FMM_BF16>(a, ncu, s);
  return launch<FMM_F16>(a, ncu, s);
}

}  // namespace q8
}  // namespace fmm
