// Products of e4m3 activations and weights, by expert or not.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "f8_gemm.h"

namespace fmm {
namespace f8 {
namespace {

template <class E, int OUT>
__global__ __launch_bounds__(256) void matmul_kernel(Product g) {
  Work w;
  if (!work_of<64, 64, true>(g, blockIdx.x, OUT == FMM_F32 ? 4 : 2, w)) return;
  const int wave = threadIdx.x >> 6;
  gemm_tile<E, OUT, true>(g, w, 32 * (wave >> 1), 32 * (wave & 1));
}

}  // namespace

int launch_matmul(int type, const Product &p, int ncu, void *stream) {
  Product g = p;
  g.tiles_n = (g.N + 63) / 64;
  g.tiles_m = g.rows / 64 + std::min(g.experts, g.rows);
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (type == FMM_F32) matmul_kernel<F8Exact, FMM_F32><<<grid, 256, 0, s>>>(g);
  else if (type == FMM_BF16) matmul_kernel<F8, FMM_BF16><<<grid, 256, 0, s>>>(g);
  else matmul_kernel<F8, FMM_F16><<<grid, 256, 0, s>>>(g);
  return hipGetLastError();
}

const char *matmul_kernel_name(int, const Product &, int) { return "matmul_kernel 64x64"; }

}  // namespace f8
}  // namespace fmm
