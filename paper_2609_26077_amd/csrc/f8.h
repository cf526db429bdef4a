// Linear layers on e4m3 operands with a power-of-two scale for each block of
// 128, by expert or not: what the host side and the kernels share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "q8.h"

namespace fmm {
namespace f8 {

using q8::pitch_of;
using q8::round_up;
using q8::type_bytes;

constexpr int kBlock = 128;
// rows of scale bytes are padded to this: the products read them eight at a time
constexpr int kScalePad = 16;
// what keeps launches below 2^32 threads and a tile's byte offsets in 32 bits; the
// elements are those of a matrix with its sides padded to 128, rows for each expert
constexpr int64_t kMaxDim = 1ll << 22, kMaxElements = 1ll << 34;
constexpr int64_t kMaxExperts = 4096;

inline int64_t scale_pitch_of(int64_t cols) { return round_up((cols + kBlock - 1) / kBlock, kScalePad); }

// ---- codes (kernels_f8_rows.hip) ----------------------------------------------
struct CodeArgs {
  void *x;                   // count x rows x cols
  uint8_t *codes, *scales;   // rows of pitch and scale_pitch bytes
  int64_t count, rows, cols, pitch, scale_pitch;
};
int launch_quantize(int type, const CodeArgs &a, void *stream);
int launch_quantize_blocks(int type, const CodeArgs &a, void *stream);
int launch_dequantize(int type, const CodeArgs &a, int block_rows, void *stream);

// ---- products (f8_gemm.h, kernels_f8_matmul.hip, kernels_f8_grad.hip) -----------
// One operand: rows of codes that are contiguous along the contracted axis.
struct Side {
  const uint8_t *codes, *scales;
  int64_t pitch, scale_pitch;              // bytes of a row
  int64_t expert_codes, expert_scales;     // from one expert's to the next one's (0: shared)
};

// C = A B^T.  Either A's rows belong to the experts, each with a B of its own
// (axis false), or the contracted axis does, and each expert has a C (axis true; the rows of its operands
// then lie together, those of one expert after those of another, as long as its blocks are).
struct Product {
  Side a, b;
  void *C;
  const float *bias;         // [experts][N] or null
  const int32_t *offsets;    // [experts + 1]: rows of expert e, or null: one expert with all of them
  int experts, rows;         // rows: of A, or of the contracted axis
  int M, N;                  // rows of C (axis: of each C), columns
  int steps;                 // 128-byte steps of the contracted axis (axis: at most)
  int axis, out_bytes;       // out_bytes: of an element of C
  int turned;                // rows of a B that lies along the contracted axis
  int tiles_m, tiles_n;      // (tiles_m with experts and not axis: at most)
};

int launch_matmul(int type, const Product &p, int ncu, void *stream);
const char *matmul_kernel_name(int type, const Product &p, int ncu);

struct GradArgs {
  const void *dy;                          // rows x N
  const uint8_t *a, *sa, *w, *sw;
  const int32_t *offsets;
  void *dx, *dw;
  float *dbias;
  uint8_t *ws;
  int64_t rows, experts, N, K;
};
size_t grad_scratch(int type, int64_t rows, int64_t experts, int64_t N, int64_t K, int ncu);
int launch_grad(int type, const GradArgs &a, int ncu, void *stream);
const char *grad_kernel_name(int type, int64_t rows, int64_t experts, int64_t N, int64_t K, bool dx, bool dw, int ncu);

// ---- clipping (kernels_clip.hip) -------------------------------------------------
struct Tensor {
  const void *in;
  void *out;
  int64_t n;
  int type;
};
constexpr int kClipBlocks = 2048;          // partial sums of a call
constexpr int kClipTable = 120;            // tensors of a launch
constexpr int64_t kMaxClipTensors = 1024 * kClipTable, kMaxClipElements = 1ll << 42;
static_assert(kMaxClipTensors <= (int64_t)kClipTable * kClipBlocks, "a partial sum for each launch");
int launch_clip(const Tensor *t, int count, float most, float *norm, double *partial, void *stream);

}  // namespace f8
}  // namespace fmm
