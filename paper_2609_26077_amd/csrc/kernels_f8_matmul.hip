// Products of e4m3 activations and weights, by expert or not.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "f8_gemm.h"

namespace fmm {
namespace f8 {
namespace {

template <class E, class T, int OUT>
__global__ __launch_bounds__(T::kThreads, 2) void matmul_kernel(Product g) {
  __shared__ uint4 lds[T::kLds / 16];
  Work w;
  if (!work_of<T::TM, T::TN, true>(g, blockIdx.x, w)) return;
  gemm_tile<E, T, OUT, true>(g, w, lds);
}

// Few tokens: the weights are read once and that bounds it, so what counts is
// bytes in flight.  A workgroup takes 16 NT channels and 16 MT tokens (of one expert) and splits
// the contracted axis over its W waves, each of which brings its own 128-byte
// pieces of those rows into its own part of LDS, D pieces ahead, whole lines at
// a time, and waits for nobody until the waves' sums meet in LDS at the end, where they
// are added in the waves' order.  Rows in LDS are swizzled as in the tile kernel.
// The scales of 128 steps go through LDS too, wave 0 bringing them before its
// first pieces.  One token of 8192 x 8192: 13.2 us, 67 MB at 5.1 TB/s; 64 tokens over 32 experts of 2048 x 4096: 41 us,
// the weights of the experts with rows at 6 TB/s.
template <class E, int MT, int NT, int W, int D, int OUT>
__global__ __launch_bounds__(64 * W) void few_tokens_kernel(Product g) {
  constexpr int kPiece = 16 * (MT + NT) * kStep;
  constexpr int kMoves = 2 * (MT + NT);            // transfers of a piece: eight rows each
  constexpr int kLds = W * D * kPiece, kSeg = 128, kScales = 16 * MT * kSeg;
  static_assert(MT * NT * 1024 <= D * kPiece && kLds + kScales + 1024 <= 160 * 1024, "the sums fit, and the pieces");
  static_assert(kBlock % (16 * NT) == 0 && kSeg % W == 0, "one scale of the weights, whole turns of the waves");
  __shared__ uint4 lds_raw[(kLds + kScales + 1024) / 16];
  const int lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Experts x(g.offsets, g.experts, g.rows, 16 * MT);
  const int tm = blockIdx.x / g.tiles_n, n0 = 16 * NT * (blockIdx.x - tm * g.tiles_n);
  if (tm >= x.total) return;
  const Span s = x.find(tm);
  const int m0 = s.lo + 16 * MT * (tm - s.tiles), rows_a = s.hi - m0, rows_b = g.N - n0;
  const int64_t ex = s.expert;
  const uint8_t *pa = g.a.codes + m0 * g.a.pitch, *pw = g.b.codes + ex * g.b.expert_codes + n0 * g.b.pitch;
  const uint8_t *psa = g.a.scales + m0 * g.a.scale_pitch;
  const uint8_t *psw = g.b.scales + ex * g.b.expert_scales + n0 / kBlock * g.b.scale_pitch;
  const uint32_t base0 = dma::lds_addr(lds_raw), base = base0 + wave * D * kPiece;
  const uint8_t *lds = reinterpret_cast<const uint8_t *>(lds_raw), *mine = lds + wave * D * kPiece;
  // rows past the end repeat the last one
  const int lrow = lane >> 3, lpos = lane & 7;
  uint32_t offw[2 * NT], offa[2 * MT];
#pragma unroll
  for (int j = 0; j < 2 * NT; ++j) {
    const int row = 8 * j + lrow;
    offw[j] = (uint32_t)(min(row, rows_b - 1) * g.b.pitch) + 16u * (uint32_t)(lpos ^ swz128(row));
  }
#pragma unroll
  for (int j = 0; j < 2 * MT; ++j) {
    const int row = 8 * j + lrow;
    offa[j] = (uint32_t)(min(row, rows_a - 1) * g.a.pitch) + 16u * (uint32_t)(lpos ^ swz128(row));
  }
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

  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = (v4f){};
  for (int seg = 0; seg < g.steps; seg += kSeg) {
    const int end = min(seg + kSeg, g.steps);
    if (seg > 0) __syncthreads();   // (everyone has read the last scales)
    if (wave == 0) {
      // 16-byte chunk c of a row of scales sits at c ^ (row mod 8); chunks past the row's end repeat its last
      const int last = (int)((g.a.scale_pitch - seg) / 16) - 1;
#pragma unroll
      for (int j = 0; j < 2 * MT; ++j)
        dma::copy16((uint32_t)(min(8 * j + lrow, rows_a - 1) * g.a.scale_pitch) + 16u * (uint32_t)min(lpos ^ lrow, last),
                    psa + seg, base0 + kLds + j * 1024);
      dma::copy16(16u * (uint32_t)min(lpos, last), psw + seg, base0 + kLds + kScales);
    }
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (seg + wave + d * W < end) start(seg + wave + d * W, d);
    if (wave == 0) {
      if (seg + (D - 1) * W < end) dma::wait_vmcnt<D * kMoves>(); else dma::wait_vmcnt<0>();
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    int slot = 0;
    for (int k = seg + wave; k < end; k += W) {
      // this piece has landed; the D - 1 after it, if there are as many, may be on their way
      if (k + (D - 1) * W < end) dma::wait_vmcnt<(D - 1) * kMoves>(); else dma::wait_vmcnt<0>();
      const uint8_t *p = mine + slot * kPiece;
      const int kk = k - seg;
      uint32_t ea[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) ea[i] = lds[kLds + (16 * i + r) * kSeg + 16 * ((kk >> 4) ^ (r & 7)) + (kk & 15)];
      const uint32_t ew = lds[kLds + kScales + kk];
      v8i fw[NT], fa[MT];
      auto read = [&](int row) {
        const v4i lo = *reinterpret_cast<const v4i *>(p + row * kStep + chunk[0]);
        const v4i hi = *reinterpret_cast<const v4i *>(p + row * kStep + chunk[1]);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      };
#pragma unroll
      for (int j = 0; j < NT; ++j) fw[j] = read(16 * j);
#pragma unroll
      for (int i = 0; i < MT; ++i) fa[i] = read(16 * (NT + i));
      // the slot has been read: fill it again
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (k + D * W < end) start(k + D * W, slot);
      slot = slot + 1 == D ? 0 : slot + 1;
      typename E::op ow[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) ow[j] = E::prepare(fw[j], ew);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const typename E::op oa = E::prepare(fa[i], ea[i]);
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = E::mma16(ow[j], ew, oa, ea[i], acc[i][j]);
      }
    }
  }
  // (a wave's sums go where its pieces were)
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
      *reinterpret_cast<v4f *>(const_cast<uint8_t *>(mine) + ((i * NT + j) * 64 + lane) * 16) = acc[i][j];
  __syncthreads();
  // lane l, element e of tile (i, j): token 16 i + l % 16, channel 16 j + 4 (l / 16) + e
  for (int e = wave; e < MT * NT; e += W) {
    const int m = 16 * (e / NT) + r, n = 16 * (e % NT) + 4 * h;
    const uint8_t *p = lds + (e * 64 + lane) * 16;
    v4f c = *reinterpret_cast<const v4f *>(p);
#pragma unroll
    for (int i = 1; i < W; ++i) c += *reinterpret_cast<const v4f *>(p + i * D * kPiece);
    if (m < rows_a && n < rows_b) {
      float bias[4] = {}, v[4];
      if (g.bias) q8::load4(g.bias + ex * g.N + n0 + n, rows_b - n, bias);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = c[q] + bias[q];
      q8::store4<OUT>(static_cast<elem_t<OUT> *>(g.C) + (int64_t)(m0 + m) * g.N + n0 + n, rows_b - n, v);
    }
  }
}

// The shapes of workgroup: t = start + max(chain pieces, work pieces groups / CUs) + group groups / CUs us, pieces
// being the 128-byte steps that a wave walks.  `chain` is a piece's time where the chip is not full, `work` where
// it is, `group` what each group costs besides: one set where several rows of tiles share a weight's tiles (through L2), one
// where a weight's tiles come for a single row of them.  Fitted on 6187 shapes, each counting alike, and checked on 3609
// others (1 to 16384 tokens; N and K to 8192, with 32 M weights and more to 16384; single weights and up to 256 experts with uneven
// rows, which the rule takes to be even).  On the latter the one that it picks is, over the fastest, 1.8% slower on average in
// 16 bits and 1.2% in fp32, more than 10% on 6% and 4% of them, 38% and 32% at worst; for few tokens over many experts 3.3%
// and 2.4% on average.  (One set of costs for both, fitted alike: 1.8% and 1.2%, of the latter 3.6% and 2.5%, and 64 x 2048 x
// 4096 of 32 gets the 128 tile.  Either way the shapes that the tests name keep their kernels.)  Each is the fastest somewhere, us:
//   tokens x N x K                   16x16   32x32   64x64   128 ahead  128     256
//   1 x 8192 x 8192 bf16             14.1    19.5    19.8    25.0       36.6    48.6
//   64 x 8192 x 8192 bf16            43.5    21.7    23.9    28.6       37.8    52.1
//   256 x 4096 x 4096 bf16           32.4    17.7    14.5    20.4       22.9    41.6
//   1000 x 1302 x 1472 fp32          26.3    15.1    12.7    15.6       15.9    -
//   2001 x 1030 x 1472 of 7 bf16     43.4    23.0    15.5    11.5       12.7    21.3
//   2048 x 4096 x 4096 bf16          208     98.0    58.4    44.1       36.0    45.2
//   16384 x 4096 x 4096 of 16 bf16   1992    906     576     426        339     286
//   64 x 2048 x 4096 of 32 bf16      40.9    38.7    54.2    55.7       51.4    55.0
struct Shape {
  int tm, tn, waves;            // tile, and the waves that share its contracted axis
  bool one;                     // only where each CU has one group at most
  struct Cost {
    float start;
    struct {
      float chain, work, group;
    } of[2];                    // several rows of tiles for each expert, one
  } cost[2];                    // of 16-bit outputs, of fp32
};
constexpr Shape kShapes[] = {
    {16, 16, 8, false, {{3.28f, {{0.665f, 0.79f, 0.0f}, {0.322f, 0.364f, 0.412f}}}, {3.56f, {{0.2f, 0.724f, 0.0f}, {0.368f, 0.61f, 0.29f}}}}},
    {32, 32, 4, false, {{3.46f, {{0.521f, 0.745f, 0.08f}, {0.511f, 0.637f, 0.09f}}}, {3.62f, {{0.632f, 0.819f, 0.02f}, {0.765f, 0.7f, 0.18f}}}}},
    {64, 64, 1, false, {{3.67f, {{0.376f, 0.296f, 0.0f}, {0.377f, 0.283f, 0.0f}}}, {3.73f, {{0.541f, 0.431f, 0.0f}, {0.553f, 0.789f, 0.04f}}}}},
    {128, 128, 1, true, {{3.75f, {{0.568f, 0.636f, 0.0f}, {0.422f, 0.44f, 0.56f}}}, {3.77f, {{0.831f, 1.09f, 0.07f}, {0.806f, 1.65f, 0.02f}}}}},
    {128, 128, 1, false, {{3.6f, {{0.672f, 0.579f, 0.0f}, {0.677f, 0.51f, 0.005f}}}, {3.6f, {{0.951f, 0.361f, 0.28f}, {1.21f, 0.815f, 0.2f}}}}},
    {256, 256, 1, false, {{6.85f, {{1.08f, 1.73f, 1.36f}, {0.767f, 1.7f, 2.87f}}}, {0.0f, {{0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f}}}}},
};
constexpr int kShapeCount = sizeof(kShapes) / sizeof(kShapes[0]);
// (a launch takes fewer than 2^32 threads, and tiles of uneven experts may be twice as many as of even ones)
constexpr double kMaxGroups = 1 << 21;

int pick(int type, const Product &g, int ncu) {
  const int shapes = type == FMM_F32 ? kShapeCount - 1 : kShapeCount;
  // experts with rows, at most, and each one's rows if they were even
  const double experts = std::max(1, std::min(g.experts, g.rows)), rows = g.rows / experts;
  int best = shapes - 1;
  double least = 1e300;
  for (int i = 0; i < shapes; ++i) {
    const Shape &p = kShapes[i];
    const double groups = experts * std::ceil(rows / p.tm) * ((g.N + p.tn - 1) / p.tn);
    if (groups > kMaxGroups || (p.one && groups > ncu)) continue;
    const double pieces = (g.steps + p.waves - 1) / p.waves;
    const float start = p.cost[type == FMM_F32].start;
    const auto &c = p.cost[type == FMM_F32].of[rows <= p.tm];
    const double t = start + std::max(c.chain * pieces, c.work * pieces * groups / ncu) + c.group * groups / ncu;
    if (t < least) {
      best = i;
      least = t;
    }
  }
  return best;
}

template <class E, int MT, int NT, int W, int D, int OUT>
void launch_few(Product g, hipStream_t s) {
  g.tiles_n = (g.N + 16 * NT - 1) / (16 * NT);
  g.tiles_m = g.rows / (16 * MT) + std::min(g.experts, g.rows);
  few_tokens_kernel<E, MT, NT, W, D, OUT><<<dim3((unsigned)(g.tiles_m * g.tiles_n)), 64 * W, 0, s>>>(g);
}

template <class E, class T, int OUT>
void launch_tiles(Product g, hipStream_t s) {
  g.tiles_n = (g.N + T::TN - 1) / T::TN;
  g.tiles_m = g.rows / T::TM + std::min(g.experts, g.rows);
  matmul_kernel<E, T, OUT><<<dim3((unsigned)(g.tiles_m * g.tiles_n)), T::kThreads, 0, s>>>(g);
}

template <class E, int OUT>
void launch(int shape, const Product &g, hipStream_t s) {
  switch (shape) {
    case 0: return launch_few<E, 1, 1, 8, 2, OUT>(g, s);
    case 1: return launch_few<E, 2, 2, 4, 2, OUT>(g, s);
    case 2: return launch_tiles<E, q8::Tile64, OUT>(g, s);
    case 3: return launch_tiles<E, q8::Tile128Ahead, OUT>(g, s);
    case 4: return launch_tiles<E, q8::Tile128, OUT>(g, s);
  }
  if constexpr (OUT != FMM_F32) launch_tiles<E, q8::Tile256, OUT>(g, s);
}

}  // namespace

const char *matmul_kernel_name(int type, const Product &p, int ncu) {
  static const char *const names[kShapeCount] = {
      "few_tokens_kernel 16x16", "few_tokens_kernel 32x32", "matmul_kernel 64x64", "matmul_kernel 128x128 ahead",
      "matmul_kernel 128x128", "matmul_kernel 256x256"};
  return names[pick(type, p, ncu)];
}

int launch_matmul(int type, const Product &p, int ncu, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int shape = pick(type, p, ncu);
  if (type == FMM_F32) launch<F8Exact, FMM_F32>(shape, p, s);
  else if (type == FMM_BF16) launch<F8, FMM_BF16>(shape, p, s);
  else launch<F8, FMM_F16>(shape, p, s);
  return hipGetLastError();
}

}  // namespace f8
}  // namespace fmm
