// The int8 product with a scale for each token and channel.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "q8_gemm.h"

namespace fmm {
namespace q8 {
namespace {

template <class T, int OUT>
__global__ __launch_bounds__(T::kThreads, 2) void matmul_kernel(GemmProblem g) {
  __shared__ uint4 lds[T::kLds / 16];
  gemm_tile<Int8, T, OUT>(g, blockIdx.x, lds);
}

// Few tokens: the weights are read once and that bounds it, so what counts is
// bytes in flight.  A workgroup takes 16 NT channels and 16 MT tokens and splits
// the contracted axis over its W waves, each of which brings its own 128-byte
// pieces of those rows into its own part of LDS, D pieces ahead, whole lines at
// a time, and waits for nobody until the waves' (exact) sums meet in LDS at the
// end.  v_mfma_i32_16x16x64_i8 takes 16 bytes a lane of 16 rows; rows in LDS are
// swizzled as in the tile kernel.  Loading the operands' lanes straight from
// memory instead touches half lines: one token of 8192 x 8192 took 16.4 us (14).
template <int MT, int NT, int W, int D, int OUT>
__global__ __launch_bounds__(64 * W) void few_tokens_kernel(GemmProblem g) {
  constexpr int kPiece = 16 * (MT + NT) * kStep;
  constexpr int kMoves = 2 * (MT + NT);            // transfers of a piece: eight rows each
  constexpr int kLds = W * D * kPiece;
  static_assert(MT * NT * 1024 <= D * kPiece && kLds <= 160 * 1024, "the sums fit, and the pieces");
  __shared__ uint4 lds_raw[kLds / 16];
  const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles_n = (g.N + 16 * NT - 1) / (16 * NT);
  const int n0 = 16 * NT * (blockIdx.x % tiles_n), m0 = 16 * MT * (blockIdx.x / tiles_n);
  const uint32_t base = dma::lds_addr(lds_raw) + wave * D * kPiece;
  const uint8_t *mine = reinterpret_cast<const uint8_t *>(lds_raw) + wave * D * kPiece;
  // rows past the end repeat the last one
  const int lrow = lane >> 3, lpos = lane & 7;
  uint32_t offw[2 * NT], offa[2 * MT];
#pragma unroll
  for (int j = 0; j < 2 * NT; ++j) {
    const int row = 8 * j + lrow;
    offw[j] = (uint32_t)(min(row, g.N - 1 - n0) * g.pitch_b) + 16u * (uint32_t)(lpos ^ swz128(row));
  }
#pragma unroll
  for (int j = 0; j < 2 * MT; ++j) {
    const int row = 8 * j + lrow;
    offa[j] = (uint32_t)(min(row, g.M - 1 - m0) * g.pitch_a) + 16u * (uint32_t)(lpos ^ swz128(row));
  }
  const uint8_t *pw = g.B + (int64_t)n0 * g.pitch_b, *pa = g.A + (int64_t)m0 * g.pitch_a;
  auto start = [&](int k, int slot) {
    const uint32_t dst = base + slot * kPiece;
#pragma unroll
    for (int j = 0; j < 2 * NT; ++j) dma::copy16(offw[j], pw + (int64_t)k * kStep, dst + j * 1024);
#pragma unroll
    for (int j = 0; j < 2 * MT; ++j) dma::copy16(offa[j], pa + (int64_t)k * kStep, dst + (2 * NT + j) * 1024);
  };
  // byte of chunk 4 u + h of row r of the first 16
  uint32_t chunk[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) chunk[u] = r * kStep + 16u * (uint32_t)((4 * u + h) ^ swz128(r));

  v4i acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = (v4i){};
#pragma unroll
  for (int d = 0; d < D; ++d)
    if (wave + d * W < g.steps) start(wave + d * W, d);
  int slot = 0;
  for (int k = wave; k < g.steps; k += W) {
    // this piece has landed; the D - 1 after it, if there are as many, may be on their way
    if (k + (D - 1) * W < g.steps) dma::wait_vmcnt<(D - 1) * kMoves>(); else dma::wait_vmcnt<0>();
    const uint8_t *p = mine + slot * kPiece;
    v4i fw[NT][2], fa[MT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u) fw[j][u] = *reinterpret_cast<const v4i *>(p + 16 * j * kStep + chunk[u]);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) fa[i][u] = *reinterpret_cast<const v4i *>(p + 16 * (NT + i) * kStep + chunk[u]);
    // the slot has been read: fill it again
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (k + D * W < g.steps) start(k + D * W, slot);
    slot = slot + 1 == D ? 0 : slot + 1;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[j][u], fa[i][u], acc[i][j], 0, 0, 0);
  }
  // (a wave's sums go where its pieces were)
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
      *reinterpret_cast<v4i *>(const_cast<uint8_t *>(mine) + ((i * NT + j) * 64 + lane) * 16) = acc[i][j];
  __syncthreads();
  // lane l, element e of tile (i, j): token 16 i + l % 16, channel 16 j + 4 (l / 16) + e
  for (int e = wave; e < MT * NT; e += W) {
    const int m = m0 + 16 * (e / NT) + r, n = n0 + 16 * (e % NT) + 4 * h;
    const uint8_t *p = reinterpret_cast<const uint8_t *>(lds_raw) + (e * 64 + lane) * 16;
    v4i s = *reinterpret_cast<const v4i *>(p);
#pragma unroll
    for (int i = 1; i < W; ++i) s += *reinterpret_cast<const v4i *>(p + i * D * kPiece);
    if (m < g.M && n < g.N) {
      float sw[4], bias[4] = {}, v[4];
      load4(g.sw + n, g.N - n, sw);
      if (g.bias) load4(g.bias + n, g.N - n, bias);
      const float sa = g.sa[m];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = (float)s[q] * sa * sw[q] + bias[q];
      store4<OUT>(static_cast<elem_t<OUT> *>(g.C) + (int64_t)m * g.N + n, g.N - n, v);
    }
  }
}

template <int MT, int NT, int W, int D, int OUT>
void launch_few(const GemmProblem &g, hipStream_t s) {
  const int64_t groups = (int64_t)((g.N + 16 * NT - 1) / (16 * NT)) * ((g.M + 16 * MT - 1) / (16 * MT));
  few_tokens_kernel<MT, NT, W, D, OUT><<<dim3((unsigned)groups), 64 * W, 0, s>>>(g);
}

// The shapes of workgroup the product comes in, and what each takes: t = start +
// max(chain pieces, work pieces groups / CUs) us, pieces being the 128-byte steps
// that a wave walks.  `chain` is a piece's time where the chip is not full, `work`
// where it is.  On 1400 shapes (1 to 32768 tokens, 1 to 65536 channels) the one that it
// picks is 1.1% slower than the fastest on average, with operands that the last-level
// cache holds or with weights from HBM; 4% of the shapes are off by more than 10%, the
// worst (8749 x 65 x 447, 7.1 us for 4.8) by 50%.  On decode's shapes, up to 384 tokens,
// 2% on average.  Each shape is the fastest somewhere, us (operands in the last-level
// cache / weights from HBM; 128+: where there are no more tiles than CUs, the 128 tile
// with a longer ring):
//   tokens x channels x channels   16x16      32x32      48x32      64x64      128+       128        256
//   1 x 8192 x 8192                13.0/17.8  18.6/22.0  18.9/22.3  14.8/23.4  24.3/35.1  34.5/56.6  70.4/93.8
//   48 x 7168 x 2048               8.6/9.8    5.9/7.8    5.3/7.2    6.7/8.8    9.7/12.6   12.8/17.8  23.9/29.2
//   64 x 4096 x 4096               11.0/12.4  6.2/8.6    7.1/8.6    8.8/13.6   14.6/20.4  19.7/29.5  39.9/50.6
//   64 x 8192 x 8192               43.0/43.4  30.4/30.7  31.2/32.2  14.9/26.1  24.6/38.1  34.7/56.6  71.3/96.6
//   256 x 4096 x 4096              31.1/32.4  15.9/18.0  14.7/16.9  9.7/13.2   14.7/22.4  19.3/28.8  39.2/52.9
//   1000 x 1302 x 1472             21.1/21.8  11.9/12.2  11.2/11.6  8.0/9.8    9.2/11.9   11.1/14.4  21.9/24.9
//   3000 x 1000 x 4000             106/104    36.2/37.6  31.1/32.7  21.8/24.5  17.3/20.3  20.9/28.6  40.0/49.7
//   2048 x 4096 x 4096             199/202    93.8/98.6  77.5/81.9  52.3/62.0  -          34.9/38.4  42.7/51.1
//   2048 x 8192 x 8192             1167/1173  634/648    501/513    232/232    -          143/147    113/115
// (A 64 x 32 shape was the cheapest by this rule on 1 shape in 4000 and is not kept.  It
// would be the fastest by up to 30% for about 256 tokens of 2048 channels and a long
// contracted axis, which start, chain and work do not tell from 64 x 8192 x 8192: there
// it takes 21.2 us for 14.9 with cached operands, 23.1 for 26.1 from HBM.)
struct Shape {
  int tm, tn, waves;            // tile, and the waves that share its contracted axis
  float start, chain, work;
  bool one;                     // only where each CU has one group at most
};
constexpr Shape kShapes[] = {
    {16, 16, 8, 1.7f, 0.30f, 0.57f, false}, {32, 32, 4, 2.2f, 0.37f, 0.61f, false},
    {48, 32, 4, 2.4f, 0.58f, 0.76f, false}, {64, 64, 1, 3.2f, 0.19f, 0.28f, false},
    {128, 128, 1, 3.3f, 0.45f, 0.60f, true}, {128, 128, 1, 3.6f, 0.47f, 0.62f, false},
    {256, 256, 1, 8.7f, 1.2f, 1.8f, false},
};

constexpr int kShapeCount = sizeof(kShapes) / sizeof(kShapes[0]);

// (a launch takes fewer than 2^32 threads; the largest tile stays below that by the limit on M N)
constexpr double kMaxGroups = 1 << 22;

int pick(const GemmProblem &g, int ncu) {
  int best = kShapeCount - 1;
  double least = 1e300;
  for (int i = 0; i < kShapeCount; ++i) {
    const Shape &p = kShapes[i];
    const double groups = (double)((g.M + p.tm - 1) / p.tm) * ((g.N + p.tn - 1) / p.tn);
    if (groups > kMaxGroups || (p.one && groups > ncu)) continue;
    const double pieces = (g.steps + p.waves - 1) / p.waves;
    const double t = p.start + std::max(p.chain * pieces, p.work * pieces * groups / ncu);
    if (t < least) {
      best = i;
      least = t;
    }
  }
  return best;
}

template <class T, int OUT>
void launch_tiles(GemmProblem g, hipStream_t s) {
  g.tiles_m = (g.M + T::TM - 1) / T::TM;
  g.tiles_n = (g.N + T::TN - 1) / T::TN;
  g.splits = 1;
  matmul_kernel<T, OUT><<<dim3((unsigned)(g.tiles_m * g.tiles_n)), T::kThreads, 0, s>>>(g);
}

template <int OUT>
void launch(const GemmProblem &g, int ncu, hipStream_t s) {
  switch (pick(g, ncu)) {
    case 0: return launch_few<1, 1, 8, 2, OUT>(g, s);
    case 1: return launch_few<2, 2, 4, 2, OUT>(g, s);
    case 2: return launch_few<3, 2, 4, 2, OUT>(g, s);
    case 3: return launch_tiles<Tile64, OUT>(g, s);
    case 4: return launch_tiles<Tile128Ahead, OUT>(g, s);
    case 5: return launch_tiles<Tile128, OUT>(g, s);
    default: return launch_tiles<Tile256, OUT>(g, s);
  }
}

}  // namespace

const char *matmul_kernel_name(const GemmProblem &p, int ncu) {
  static const char *const names[kShapeCount] = {
      "few_tokens_kernel 16x16", "few_tokens_kernel 32x32",      "few_tokens_kernel 48x32", "matmul_kernel 64x64",
      "matmul_kernel 128x128 ahead", "matmul_kernel 128x128", "matmul_kernel 256x256"};
  return names[pick(p, ncu)];
}

int launch_matmul(int type, const GemmProblem &p, int ncu, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == FMM_F32) launch<FMM_F32>(p, ncu, s);
  else if (type == FMM_BF16) launch<FMM_BF16>(p, ncu, s);
  else launch<FMM_F16>(p, ncu, s);
  return hipGetLastError();
}

}  // namespace q8
}  // namespace fmm
