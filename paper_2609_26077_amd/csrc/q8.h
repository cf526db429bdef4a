// The 8-bit linear layer: what its host side and its kernels share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/fmm8.h"

namespace fmm {
namespace q8 {

constexpr int kGroup = 128;              // code rows are padded to, and checkpoints scaled by, groups of this many columns
constexpr int64_t kMaxK = 131071;        // int8 products: K 2^14 < 2^31, so an int32 sum cannot overflow
// what keeps every launch under 2^32 threads and a tile's byte offsets in 32 bits
constexpr int64_t kMaxRows = 1ll << 30, kMaxCols = 1ll << 24;
constexpr int64_t kMaxOutputs = 1ll << 37;
constexpr int64_t kMaxGradDim = 1ll << 22, kMaxGradElements = 1ll << 34;

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline int64_t pitch_of(int64_t cols) { return round_up(cols, kGroup); }
inline int type_bytes(int type) { return type == FMM_F32 ? 4 : 2; }

// ---- rows: quantize, dequantize, RMS norm (kernels_q8_rows.hip) -------------
struct RowArgs {
  const void *x, *res, *gain;   // rows x cols, rows x cols or null, cols or null
  void *h;                      // rows x cols or null: x + res rounded to the type
  int8_t *codes;                // rows x pitch
  float *scales;                // rows
  int8_t *saved;                // rows x pitch or null: the checkpoint of x + res
  float *saved_scales;          // rows x pitch / 128
  float *rstd;                  // rows (norm only)
  int64_t rows, cols, pitch;
  float eps;
};
int launch_quantize(int type, const RowArgs &a, void *stream);
int launch_rmsnorm(int type, const RowArgs &a, void *stream);
// widest row that stays in registers (longer ones are read twice)
constexpr int64_t kMaxHeldCols = 32768;

struct DequantArgs {
  const int8_t *codes;
  const float *scales;   // one per row, or one per row and group
  void *out;             // rows x cols
  int64_t rows, cols, pitch;
  int grouped;
};
int launch_dequantize(int type, const DequantArgs &a, void *stream);

struct NormGradArgs {
  const void *dy, *dh, *h, *gain;   // dh, gain may be null; h null: saved
  const int8_t *saved;
  const float *saved_scales, *rstd;
  void *dx;
  float *dgain;       // cols or null
  float *partial;     // blocks x cols
  int64_t rows, cols, pitch;
};
// rows of partial sums that the gradient of the gain goes through
int64_t norm_grad_partials(int type, int64_t rows, int64_t cols);
int launch_rmsnorm_grad(int type, const NormGradArgs &a, void *stream);

// ---- products (q8_gemm.h, kernels_q8_matmul.hip, kernels_q8_grad.hip) -------
// C = A B^T over K-contiguous rows: `parts` planes of A (one after the other
// along the contracted axis) against the same B.
struct GemmProblem {
  const uint8_t *A, *B;             // M rows of pitch_a bytes, N rows of pitch_b bytes
  int64_t pitch_a, pitch_b, part_a; // part_a: bytes from one plane of A to the next
  const float *sa, *sw, *bias;      // int8: C = acc sa[m] sw[n] + bias[n] (bias null: 0)
  void *C;                          // M x N
  int M, N;
  int steps, parts;                 // 128-byte steps of a plane, planes
  int tiles_m, tiles_n;
  int splits;                       // the contracted axis in this many runs of steps;
  float *partial;                   // if more than one, their sums go here: [splits][M][N] (bf16 only)
};

int launch_matmul(int type, const GemmProblem &p, int ncu, void *stream);
const char *matmul_kernel_name(const GemmProblem &p, int ncu);

struct GradArgs {
  const void *dy;
  const int8_t *a, *w;
  const float *sa, *sw;
  void *dx, *dw;
  float *dbias;
  uint8_t *ws;
  int64_t M, N, K;
};
size_t grad_scratch(int type, int64_t M, int64_t N, int64_t K, int ncu);
const char *linear_grad_kernel_name(int type, int64_t M, int64_t N, int64_t K, bool dx, bool dw, int ncu, int32_t *runs);
int launch_linear_grad(int type, const GradArgs &a, int ncu, void *stream);

}  // namespace q8
}  // namespace fmm
