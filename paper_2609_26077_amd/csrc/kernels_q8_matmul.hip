// The int8 product with a scale for each token and channel.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "q8_gemm.h"

namespace fmm {
namespace q8 {
namespace {

template <class T, int OUT>
__global__ __launch_bounds__(T::kThreads, T::kThreads == 512 ? 2 : 1) void matmul_kernel(GemmProblem g) {
  __shared__ uint4 lds[2 * T::kSlot / 16];
  gemm_tile<Int8, T, OUT>(g, blockIdx.x, lds);
}

template <int OUT>
void launch(GemmProblem g, int ncu, hipStream_t s) {
  auto tiles = [&](int edge) {
    g.tiles_m = (g.M + edge - 1) / edge;
    g.tiles_n = (g.N + edge - 1) / edge;
    return (int64_t)g.tiles_m * g.tiles_n;
  };
  g.splits = 1;
  if (tiles(256) >= ncu) {
    matmul_kernel<Tile256, OUT><<<dim3((unsigned)tiles(256)), Tile256::kThreads, 0, s>>>(g);
  } else if (tiles(128) >= ncu) {
    matmul_kernel<Tile128, OUT><<<dim3((unsigned)tiles(128)), Tile128::kThreads, 0, s>>>(g);
  } else {
    const unsigned n = (unsigned)tiles(64);
    matmul_kernel<Tile64, OUT><<<dim3(n), Tile64::kThreads, 0, s>>>(g);
  }
}

}  // namespace

size_t matmul_scratch(int64_t, int64_t, int64_t, int) { return 0; }

int launch_matmul(int type, const GemmProblem &p, int ncu, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == FMM_F32) launch<FMM_F32>(p, ncu, s);
  else if (type == FMM_BF16) launch<FMM_BF16>(p, ncu, s);
  else launch<FMM_F16>(p, ncu, s);
  return hipGetLastError();
}

}  // namespace q8
}  // namespace fmm
