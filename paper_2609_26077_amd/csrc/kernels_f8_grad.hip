// The gradients of the e4m3 linear layers, on e4m3 operands throughout:
//   dX = Q(dY) W, blocks of Q(dY) along a row;  dW = Q(dY)^T Q(X), blocks of 128 rows
// counted from the expert's first row, X being the codes of the forward pass.
//
// The layout pass brings dY and X into rows along their contracted axes: dY
// by rows (dyr) and by columns (dyt), X by columns (xt).  W's codes stay where they are: dX's product reads them by
// columns from LDS (turning them first, 268 MB of 600 for 16384 x 4096 x 2048 of 16 experts, took 40 us of
// 125; 26 tokens of 24 experts' 390 x 1664 44 us for 29), and a 128 x 128 block's scale is that of its
// transpose, so only the table of scales (swt) is turned.
// X's codes are rounded again where the new block's scale is larger than the old one
// (codes below 2^-15 of the block's largest).  It also leaves dY's column sums by block.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "f8_gemm.h"

namespace fmm {
namespace f8 {
namespace {

struct LayoutArgs {
  const void *dy;
  const uint8_t *a, *sa, *sw;
  const int32_t *offsets;
  uint8_t *dyr, *sdyr;      // [rows][Np], [rows][spn]
  uint8_t *dyt, *sdyt;      // of each expert [N][128 blocks], [N][blocks, padded to 16], blocks: of 128 of its rows
  uint8_t *xt, *sxt;        // the same with K
  uint8_t *swt;             // [experts][K / 128][spn]
  float *colsum;            // [blocks][N]
  int64_t Np, Kp, spn, spk;
  int rows, experts, N, K;
  int blocks, bn, bk;                // blocks of rows (at most), of N, of K
  int jobs_dy, jobs_a, jobs_w;
  int want_dx, want_dw, want_db;
};

// One 128 x 128 tile a workgroup: thread t has eight columns of R rows from R (t / 16) on.  R is 4 where
// a CU has few tiles and their latency counts, else 8 (with W's tiles beside dY's and X's: 1000 x 1302 x 1472
// fp32 11.0 us for 11.9, 16384 x 4096 x 2048 bf16 of 16 experts 120 us for 137; without them, and with the
// columns' maxima by LDS atomics, 9.4 and 78, 335 MB at 4.3 TB/s, half of them written).
// The transpose goes through LDS in pieces of four bytes (four rows of a column);
// piece p of column n sits at p ^ 2 (n / 8), so that both directions spread over the banks
// and sixteen bytes stay together but for their order.
template <int R>
struct Turn {
  static constexpr int kThreads = 2048 / R, kWaves = kThreads / 64;
  uint32_t out[128][32];
  uint32_t most[128];
  float sum[kWaves][128];
};
__device__ __forceinline__ int piece(int p, int n) { return p ^ (2 * (n >> 3) & 31); }

// the tile's columns n < cols to rows of dst
template <int R>
__device__ __forceinline__ void store_columns(const Turn<R> &tile, uint8_t *dst, int64_t pitch, int cols) {
  const int t = threadIdx.x, c = t & 7;
#pragma unroll
  for (int p = 0; p < R / 2; ++p) {
    const int n = Turn<R>::kThreads / 8 * p + (t >> 3);
    if (n < cols) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(&tile.out[n][piece(4 * c, n) & ~3]);
      *reinterpret_cast<u32x4 *>(dst + n * pitch + 16 * c) = n >> 3 & 1 ? (u32x4){v[2], v[3], v[0], v[1]} : v;
    }
  }
}

// codes by columns of v, and their scales to scales[n * pitch]; tile.most is zero
template <int R>
__device__ __forceinline__ void columns(Turn<R> &tile, const float (&v)[R][8], uint8_t *dst, int64_t pitch, uint8_t *scales,
                                        int64_t scale_pitch, int cols) {
  const int t = threadIdx.x, lane = t & 63, rg = t >> 4, cg = t & 15;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t a = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) a = max(a, magnitude(v[r][i]));
    a = max(a, (uint32_t)__shfl_xor((int)a, 16));
    a = max(a, (uint32_t)__shfl_xor((int)a, 32));
    if (lane < 16) atomicMax(&tile.most[8 * cg + i], a);
  }
  __syncthreads();
  if (t < 128 && t < cols) scales[t * scale_pitch] = (uint8_t)scale_byte(tile.most[t]);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int n = 8 * cg + i;
    const float s = scale_value(scale_byte(tile.most[n]));
#pragma unroll
    for (int r = 0; r < R; r += 4)
      tile.out[n][piece((R * rg + r) / 4, n)] = codes4(v[r][i], v[r + 1][i], v[r + 2][i], v[r + 3][i], s);
  }
  __syncthreads();
  store_columns(tile, dst, pitch, cols);
}

template <int T, int R>
__global__ __launch_bounds__(Turn<R>::kThreads) void layout_kernel(LayoutArgs g) {
  __shared__ Turn<R> tile;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, rg = t >> 4, cg = t & 15;
  int id = blockIdx.x;
  if (id >= g.jobs_dy + g.jobs_a) {
    // an expert's scales of W
    id -= g.jobs_dy + g.jobs_a;
    for (int i = t; i < g.bn * g.bk; i += Turn<R>::kThreads) {
      const int kb = i / g.bn, nb = i - kb * g.bn;
      g.swt[((int64_t)id * g.bk + kb) * g.spn + nb] = g.sw[((int64_t)id * g.bn + nb) * g.spk + kb];
    }
    return;
  }
  const bool is_dy = id < g.jobs_dy;
  if (!is_dy) id -= g.jobs_dy;
  const int bc = is_dy ? g.bn : g.bk, block = id / bc, cb = id % bc, c0 = cb * kBlock, cols = (is_dy ? g.N : g.K) - c0;
  Experts x(g.offsets, g.experts, g.rows, kBlock);
  if (block >= x.total) return;
  const Span s = x.find(block);
  const int row0 = s.lo + (block - s.tiles) * kBlock, rows = s.hi - row0;
  // where the expert's codes by columns and their scales begin (bytes of a row before them), the rows' bytes
  const int64_t before = (int64_t)s.tiles * kBlock, scales_before = (int64_t)s.wides * kScalePad;
  const int mine = (s.hi - s.lo + kBlock - 1) / kBlock, at = block - s.tiles;
  const int64_t Bp = (int64_t)mine * kBlock, sbp = (mine + kScalePad - 1) / kScalePad * kScalePad;
  float v[R][8];
  if (t < 128) tile.most[t] = 0;
  __syncthreads();
  if (is_dy) {
    const elem_t<T> *src = static_cast<const elem_t<T> *>(g.dy) + (int64_t)(row0 + R * rg) * g.N + c0 + 8 * cg;
    q8::Raw8<T> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r] = q8::raw8<T>(src + (int64_t)r * g.N, R * rg + r < rows ? cols - 8 * cg : 0);
#pragma unroll
    for (int r = 0; r < R; ++r) q8::floats8<T>(raw[r], v[r]);
    if (g.want_dx) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, magnitude(v[r][i]));
        const uint32_t b = scale_byte(q8::max16(a));
        const float sc = scale_value(b);
        const int64_t row = row0 + R * rg + r;
        if (R * rg + r < rows) {
          u32x2 q;
          q[0] = codes4(v[r][0], v[r][1], v[r][2], v[r][3], sc);
          q[1] = codes4(v[r][4], v[r][5], v[r][6], v[r][7], sc);
          *reinterpret_cast<u32x2 *>(g.dyr + row * g.Np + c0 + 8 * cg) = q;
          if (cg == 0) g.sdyr[row * g.spn + cb] = (uint8_t)b;
        }
      }
    }
    if (g.want_db) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float c = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) c += v[r][i];
        c += __shfl_xor(c, 16);
        c += __shfl_xor(c, 32);
        if (lane < 16) tile.sum[wave][8 * cg + i] = c;
      }
      __syncthreads();
      if (t < 128 && t < cols) {
        float c = 0.0f;
#pragma unroll
        for (int k = 0; k < Turn<R>::kWaves; ++k) c += tile.sum[k][t];
        g.colsum[(int64_t)block * g.N + c0 + t] = c;
      }
    }
    if (g.want_dw)
      columns(tile, v, g.dyt + before * g.N + c0 * Bp + at * kBlock, Bp, g.sdyt + scales_before * g.N + c0 * sbp + at, sbp, cols);
  } else {
    const uint8_t *src = g.a + (int64_t)(row0 + R * rg) * g.Kp + c0 + 8 * cg;
    const uint8_t *scales = g.sa + (int64_t)(row0 + R * rg) * g.spk + cb;
    u32x2 q[R];
    uint32_t b[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool some = R * rg + r < rows;
      q[r] = some ? *reinterpret_cast<const u32x2 *>(src + r * g.Kp) : (u32x2){0, 0};
      b[r] = some ? scales[r * g.spk] : 127u;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) values8(q[r], scale_value(b[r]), v[r]);
    columns(tile, v, g.xt + before * g.K + c0 * Bp + at * kBlock, Bp, g.sxt + scales_before * g.K + c0 * sbp + at, sbp, cols);
  }
}

struct GradGemms {
  Product x, w;              // dX, dW
  int x_first;               // dX's tiles come before dW's: the ones with the longer chain
  int items0, items;         // workgroups of the first, of both
  const float *colsum;
  float *dbias;
};

// Tiles TX of dX and TW of dW (equal workgroups), then dY's column sums by expert.
template <class E, class TX, class TW, int OUT>
__global__ __launch_bounds__(TX::kThreads, 2) void grad_kernel(GradGemms g) {
  static_assert(TX::kThreads == TW::kThreads, "one launch");
  __shared__ uint4 lds[(TX::kLds > TW::kLds ? TX::kLds : TW::kLds) / 16];
  int id = blockIdx.x;
  if (id < g.items) {
    Work w;
    const bool first = id < g.items0;
    if (!first) id -= g.items0;
    if (first == (g.x_first != 0)) {
      if (work_of<TX::TM, TX::TN, true, true>(g.x, id, w)) gemm_tile<E, TX, OUT, true, true>(g.x, w, lds);
    } else {
      if (work_of<TW::TM, TW::TN, false>(g.w, id, w)) gemm_tile<E, TW, OUT, false>(g.w, w, lds);
    }
    return;
  }
  const int N = g.w.M, per = (N + TX::kThreads - 1) / TX::kThreads;
  id -= g.items;
  const int e = id / per, n = (id - e * per) * TX::kThreads + threadIdx.x;
  Experts x(g.w.offsets, g.w.experts, g.w.rows, kBlock);
  const Span s = x.at(e);
  if (n >= N) return;
  const int blocks = (s.hi - s.lo + kBlock - 1) / kBlock;
  float c = 0.0f;
#pragma unroll 4
  for (int i = 0; i < blocks; ++i) c += g.colsum[(int64_t)(s.tiles + i) * N + n];
  g.dbias[(int64_t)e * N + n] = c;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {
  size_t dyr, sdyr, dyt, sdyt, xt, sxt, swt, colsum, total;
  int64_t blocks, Np, spn;
};
Layout layout_of(int64_t rows, int64_t experts, int64_t N, int64_t K) {
  Layout l;
  const int64_t full = std::min(experts, rows);      // experts that may have rows
  l.blocks = rows / kBlock + full;
  l.Np = pitch_of(N);
  l.spn = scale_pitch_of(N);
  const int64_t Bp = l.blocks * kBlock, sbp = kScalePad * (l.blocks / kScalePad + full);   // rows of all experts' blocks
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at = align256(at + (size_t)bytes);
    return here;
  };
  l.dyr = take(rows * l.Np);
  l.sdyr = take(rows * l.spn);
  l.dyt = take(N * Bp);
  l.sdyt = take(N * sbp);
  l.xt = take(K * Bp);
  l.sxt = take(K * sbp);
  l.swt = take(experts * (pitch_of(K) / kBlock) * l.spn);
  l.colsum = take(4 * l.blocks * N);
  l.total = at;
  return l;
}

// The tile of each product: 0: 64, 1: 128, 2: 256, 3: 128 with the longer ring (2 and 3 of both, or
// neither: their workgroups are larger).
struct Cut {
  int x, w;
};

// t = max(start + chain steps, of either; start + work of both / CUs) + tile tiles / CUs us, as for the forward
// products.  Against all cuts on 2384 shapes that it was not fitted on (rows 16 to 16384, N to 8192, K to 4096, single
// weights and up to 64 experts): 1.0% over the fastest on average in 16 bits and 0.5% in fp32, more than 10% on 3%
// and 1.5% of them, 34% and 15% at worst (thousands of rows over a few experts).  Each is the fastest somewhere, us (64:
// of both, 64/128: dX's and dW's, ...):
//   rows x N x K of experts          64     64/128  128/64  128    128 ahead  256
//   16384 x 4096 x 2048 of 16 bf16   814    596     660     455    581        379
//   4096 x 4096 x 2048 fp32          224    186     183     153    178        -
//   1000 x 1302 x 1472 fp32          30.8   28.6    29.0    29.1   28.5       -
//   114 x 440 x 754 of 16 bf16       23.3   21.9    22.9    18.9   21.0       22.4
//   2229 x 1664 x 354 bf16           25.9   30.2    28.3    31.6   28.6       42.6
//   5668 x 133 x 1536 of 4 bf16      37.7   37.4    29.9    35.4   34.0       48.8
Cut cut_of(int type, int64_t rows, int64_t experts, int64_t N, int64_t K, bool dx, bool dw, int ncu) {
  constexpr int kEdge[4] = {64, 128, 256, 128};
  struct Cost {
    double start, chain, work, tile;
  };
  constexpr Cost kCost[2][4] = {{{3.29, 0.03, 0.329, 0.0}, {3.56, 0.616, 0.56, 0.0}, {8.54, 1.05, 1.76, 0.0}, {3.55, 0.448, 0.698, 0.51}},
                                {{3.11, 0.243, 0.395, 0.2}, {3.71, 0.957, 0.731, 0.0}, {0.0, 0.0, 0.0, 0.0}, {4.11, 0.688, 0.899, 0.92}}};
  const Cost(&cost)[4] = kCost[type == FMM_F32];
  // experts with rows, at most, and each one's rows if they were even
  const double full = std::max<double>(1, std::min(experts, rows)), each = rows / full;
  const double steps_x = dx ? (N + kBlock - 1) / kBlock : 0, steps_w = dw ? std::ceil(each / kBlock) : 0;
  Cut best = {};
  double least = 1e300;
  for (int x = 0; x < 4; ++x)
    for (int w = 0; w < 4; ++w) {
      if (x != w && (x > 1 || w > 1)) continue;
      if (x == 2 && type == FMM_F32) continue;
      const double tx = dx ? full * std::ceil(each / kEdge[x]) * std::ceil((double)K / kEdge[x]) : 0;
      const double tw = dw ? full * std::ceil((double)N / kEdge[w]) * std::ceil((double)K / kEdge[w]) : 0;
      if (x == 3 && tx + tw > ncu) continue;
      const Cost &cx = cost[x], &cw = cost[w];
      const double chain = std::max(dx ? cx.start + cx.chain * steps_x : 0, dw ? cw.start + cw.chain * steps_w : 0);
      const double busy = std::max(dx ? cx.start : 0, dw ? cw.start : 0) + (cx.work * steps_x * tx + cw.work * steps_w * tw) / ncu;
      const double t = std::max(chain, busy) + (cx.tile * tx + cw.tile * tw) / ncu;
      if (t < least) {
        least = t;
        best = {x, w};
      }
    }
  return best;
}

template <class E, int T, class TX, class TW>
void launch_gemms(GradGemms g, const GradArgs &a, hipStream_t s) {
  g.x.tiles_n = (g.x.N + TX::TN - 1) / TX::TN;
  g.x.tiles_m = g.x.rows / TX::TM + std::min(g.x.experts, g.x.rows);
  g.w.tiles_n = (g.w.N + TW::TN - 1) / TW::TN;
  g.w.tiles_m = (g.w.M + TW::TM - 1) / TW::TM;
  const int x = a.dx ? g.x.tiles_m * g.x.tiles_n : 0, w = a.dw ? g.w.experts * (int)round_up(g.w.tiles_m * g.w.tiles_n, 8) : 0;
  const int db = a.dbias ? g.w.experts * ((g.w.M + TX::kThreads - 1) / TX::kThreads) : 0;
  g.x_first = g.x.steps * g.w.experts >= g.w.steps;
  // (whole turns over the XCDs, so that the second's order is the first's)
  g.items0 = (int)round_up(g.x_first ? x : w, 8);
  g.items = g.items0 + (g.x_first ? w : x);
  if (g.items + db > 0) grad_kernel<E, TX, TW, T><<<dim3((unsigned)(g.items + db)), TX::kThreads, 0, s>>>(g);
}

template <class E, int T>
int launch(const GradArgs &a, int ncu, hipStream_t s) {
  const Cut cut = cut_of(T, a.rows, a.experts, a.N, a.K, a.dx, a.dw, ncu);
  const Layout l = layout_of(a.rows, a.experts, a.N, a.K);
  LayoutArgs g = {};
  g.dy = a.dy; g.a = a.a; g.sa = a.sa; g.sw = a.sw; g.offsets = a.offsets;
  g.dyr = a.ws + l.dyr; g.sdyr = a.ws + l.sdyr;
  g.dyt = a.ws + l.dyt; g.sdyt = a.ws + l.sdyt;
  g.xt = a.ws + l.xt; g.sxt = a.ws + l.sxt;
  g.swt = a.ws + l.swt;
  g.colsum = reinterpret_cast<float *>(a.ws + l.colsum);
  g.Np = l.Np; g.Kp = pitch_of(a.K); g.spn = l.spn; g.spk = scale_pitch_of(a.K);
  g.rows = (int)a.rows; g.experts = (int)a.experts; g.N = (int)a.N; g.K = (int)a.K;
  g.blocks = (int)l.blocks; g.bn = (int)(l.Np / kBlock); g.bk = (int)(g.Kp / kBlock);
  g.want_dx = a.dx != nullptr; g.want_dw = a.dw != nullptr; g.want_db = a.dbias != nullptr;
  g.jobs_dy = g.want_dx || g.want_dw || g.want_db ? g.blocks * g.bn : 0;
  g.jobs_a = g.want_dw ? g.blocks * g.bk : 0;
  g.jobs_w = g.want_dx && a.rows > 0 ? g.experts : 0;
  const int jobs = g.jobs_dy + g.jobs_a + g.jobs_w;
  if (jobs > 4 * ncu) layout_kernel<T, 8><<<dim3((unsigned)jobs), Turn<8>::kThreads, 0, s>>>(g);
  else if (jobs > 0) layout_kernel<T, 4><<<dim3((unsigned)jobs), Turn<4>::kThreads, 0, s>>>(g);

  GradGemms q = {};
  q.colsum = g.colsum; q.dbias = a.dbias;
  q.x.offsets = a.offsets; q.x.experts = g.experts; q.x.rows = g.rows; q.x.N = g.K; q.x.out_bytes = type_bytes(T);
  q.w = q.x;
  q.x.a = {g.dyr, g.sdyr, g.Np, g.spn, 0, 0};
  q.x.b = {a.w, g.swt, g.Kp, g.spn, a.N * g.Kp, (int64_t)g.bk * g.spn};
  q.x.turned = g.N;
  q.x.C = a.dx; q.x.M = g.rows; q.x.steps = g.bn;
  q.w.a.codes = g.dyt; q.w.a.scales = g.sdyt;
  q.w.b.codes = g.xt; q.w.b.scales = g.sxt;
  q.w.C = a.dw; q.w.M = g.N; q.w.steps = g.blocks; q.w.axis = 1;
  if (cut.x == 3) launch_gemms<E, T, q8::Tile128Ahead, q8::Tile128Ahead>(q, a, s);
  else if (cut.x == 1 && cut.w == 1) launch_gemms<E, T, q8::Tile128, q8::Tile128>(q, a, s);
  else if (cut.x == 1) launch_gemms<E, T, q8::Tile128, q8::Tile64>(q, a, s);
  else if (cut.x == 0 && cut.w == 1) launch_gemms<E, T, q8::Tile64, q8::Tile128>(q, a, s);
  else if (cut.x == 0) launch_gemms<E, T, q8::Tile64, q8::Tile64>(q, a, s);
  else if constexpr (T != FMM_F32) launch_gemms<E, T, q8::Tile256, q8::Tile256>(q, a, s);
  return hipGetLastError();
}

}  // namespace

size_t grad_scratch(int, int64_t rows, int64_t experts, int64_t N, int64_t K, int) {
  return layout_of(rows, experts, N, K).total;
}

const char *grad_kernel_name(int type, int64_t rows, int64_t experts, int64_t N, int64_t K, bool dx, bool dw, int ncu) {
  static const char *const small[2][2] = {{"grad_kernel 64x64 64x64", "grad_kernel 64x64 128x128"},
                                          {"grad_kernel 128x128 64x64", "grad_kernel 128x128 128x128"}};
  const Cut c = cut_of(type, rows, experts, N, K, dx, dw, ncu);
  if (c.x == 2) return "grad_kernel 256x256 256x256";
  if (c.x == 3) return "grad_kernel 128x128 128x128 ahead";
  return small[c.x][c.w];
}

int launch_grad(int type, const GradArgs &a, int ncu, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == FMM_F32) return launch<F8Exact, FMM_F32>(a, ncu, s);
  if (type == FMM_BF16) return launch<F8, FMM_BF16>(a, ncu, s);
  return launch<F8, FMM_F16>(a, ncu, s);
}

}  // namespace f8
}  // namespace fmm
