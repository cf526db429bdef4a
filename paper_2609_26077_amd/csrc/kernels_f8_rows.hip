// e4m3 codes with a power-of-two scale for each block of 128: of rows (1 x 128)
// and of weights (128 x 128), and back.
//
// HBM bounds them where the data is large (weights of eight 1301 x 2050 in fp32: 22 us, 107 MB at 4.8 TB/s, and
// back 19 us, 5.6 TB/s), the launch where it is small (one row of 4096: 2.4 us of 8 that a call takes on the host).
// A block's maximum is taken on bits, and one instruction divides by the power of two and rounds.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "f8_types.h"

namespace fmm {
namespace f8 {
namespace {

// A group of sixteen lanes has one block of a row, eight elements a lane.  A
// workgroup's sixteen groups are 2^shift blocks side by side of 16 >> shift rows, so
// that narrow matrices leave few of them idle.
struct Walk {
  int shift, chunks;           // chunks: of 2^shift blocks in a row
  int64_t row_groups, groups;  // of 16 >> shift rows in a matrix, workgroups
};
Walk walk_of(const CodeArgs &a) {
  const int64_t blocks = a.pitch / kBlock;
  Walk w = {};
  // the widest that wastes little: chunks that reach past a row's end leave their groups idle
  // (eight weights of 1301 x 2050, 17 blocks a row, back to fp32: 31 us by 16 blocks)
  for (w.shift = 4; w.shift > 0 && round_up(blocks, 1 << w.shift) * 8 > blocks * 9; --w.shift) {}
  w.chunks = (int)((blocks + (1 << w.shift) - 1) >> w.shift);
  const int rows = 16 >> w.shift;
  w.row_groups = (a.rows + rows - 1) / rows;
  w.groups = a.count * w.row_groups * w.chunks;
  return w;
}
// the lane's matrix, row and first column; false past the end
__device__ __forceinline__ bool place(const CodeArgs &g, const Walk &w, int64_t id, int64_t &m, int64_t &row, int64_t &col) {
  const int64_t rg = id / w.chunks;
  m = rg / w.row_groups;
  const int t = threadIdx.x >> 4;
  row = ((rg - m * w.row_groups) << (4 - w.shift)) + (t >> w.shift);
  col = (((id - rg * w.chunks) << w.shift) + (t & ((1 << w.shift) - 1))) * kBlock + 8 * (threadIdx.x & 15);
  return row < g.rows && col < g.pitch;
}

template <int T>
__global__ __launch_bounds__(256) void quantize_kernel(CodeArgs g, Walk w) {
  int64_t m, row, col;
  if (!place(g, w, blockIdx.x, m, row, col)) return;   // (whole groups of sixteen leave)
  const int64_t at = m * g.rows + row;
  float v[8];
  q8::load8<T>(static_cast<const elem_t<T> *>(g.x) + at * g.cols + col, g.cols - col, v);
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, magnitude(v[i]));
  const uint32_t b = scale_byte(q8::max16(a));
  const float s = scale_value(b);
  u32x2 q;
  q[0] = codes4(v[0], v[1], v[2], v[3], s);
  q[1] = codes4(v[4], v[5], v[6], v[7], s);
  *reinterpret_cast<u32x2 *>(g.codes + at * g.pitch + col) = q;
  uint8_t *scales = g.scales + at * g.scale_pitch;
  const int lane = threadIdx.x & 15;
  if (lane == 0) scales[col / kBlock] = (uint8_t)b;
  // the bytes that pad the row of scales
  const int64_t pad = g.pitch / kBlock + lane;
  if (col < kBlock && pad < g.scale_pitch) scales[pad] = 127;
}

// A workgroup a block: thread t has eight columns of rows 8 (t / 16) .. + 7.
template <int T>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(CodeArgs g) {
  __shared__ uint32_t most[4];
  const int nb = (int)(g.pitch / kBlock), rb = (int)((g.rows + kBlock - 1) / kBlock);
  const int64_t id = blockIdx.x, m = id / ((int64_t)nb * rb);
  const int in = (int)(id - m * nb * rb), kr = in / nb, kc = in - kr * nb;
  const int t = threadIdx.x;
  const int64_t row0 = (int64_t)kr * kBlock + 8 * (t >> 4), col = (int64_t)kc * kBlock + 8 * (t & 15);
  const int64_t at = m * g.rows + row0;
  q8::Raw8<T> raw[8];
#pragma unroll
  for (int r = 0; r < 8; ++r)
    raw[r] = q8::raw8<T>(static_cast<const elem_t<T> *>(g.x) + (at + r) * g.cols + col, row0 + r < g.rows ? g.cols - col : 0);
  uint32_t a = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    float v[8];
    q8::floats8<T>(raw[r], v);
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, magnitude(v[i]));
  }
  a = q8::max64(a);
  if ((t & 63) == 0) most[t >> 6] = a;
  __syncthreads();
  a = max(max(most[0], most[1]), max(most[2], most[3]));
  const uint32_t b = scale_byte(a);
  const float s = scale_value(b);
#pragma unroll
  for (int r = 0; r < 8; ++r)
    if (row0 + r < g.rows) {
      float v[8];
      q8::floats8<T>(raw[r], v);
      u32x2 q;
      q[0] = codes4(v[0], v[1], v[2], v[3], s);
      q[1] = codes4(v[4], v[5], v[6], v[7], s);
      *reinterpret_cast<u32x2 *>(g.codes + (at + r) * g.pitch + col) = q;
    }
  uint8_t *scales = g.scales + (m * rb + kr) * g.scale_pitch;
  if (t == 0) scales[kc] = (uint8_t)b;
  if (kc == 0 && nb + t < g.scale_pitch && t < kScalePad) scales[nb + t] = 127;
}

template <int T>
__global__ __launch_bounds__(256) void dequantize_kernel(CodeArgs g, Walk w, int shift) {
  int64_t m, row, col;
  if (!place(g, w, blockIdx.x, m, row, col)) return;
  const int64_t at = m * g.rows + row, srows = ((g.rows - 1) >> shift) + 1;
  const u32x2 q = *reinterpret_cast<const u32x2 *>(g.codes + at * g.pitch + col);
  const float s = scale_value(g.scales[(m * srows + (row >> shift)) * g.scale_pitch + col / kBlock]);
  float v[8];
  values8(q, s, v);
  q8::store8<T>(static_cast<elem_t<T> *>(g.x) + at * g.cols + col, g.cols - col, v);
}

constexpr int64_t kMaxGroups = (1ll << 32) / 256 - 1;   // a launch takes fewer than 2^32 threads

}  // namespace

#define FMM_TYPES(type, CALL)           \
  do {                                  \
    if ((type) == FMM_F32) CALL(FMM_F32); \
    else if ((type) == FMM_BF16) CALL(FMM_BF16); \
    else CALL(FMM_F16);                 \
  } while (0)

int launch_quantize(int type, const CodeArgs &a, void *stream) {
  const Walk w = walk_of(a);
  if (w.groups > kMaxGroups) return hipErrorInvalidConfiguration;
#define CALL(T) quantize_kernel<T><<<dim3((unsigned)w.groups), 256, 0, static_cast<hipStream_t>(stream)>>>(a, w)
  FMM_TYPES(type, CALL);
#undef CALL
  return hipGetLastError();
}

int launch_quantize_blocks(int type, const CodeArgs &a, void *stream) {
  const int64_t groups = a.count * (a.pitch / kBlock) * ((a.rows + kBlock - 1) / kBlock);
  if (groups > kMaxGroups) return hipErrorInvalidConfiguration;
#define CALL(T) quantize_blocks_kernel<T><<<dim3((unsigned)groups), 256, 0, static_cast<hipStream_t>(stream)>>>(a)
  FMM_TYPES(type, CALL);
#undef CALL
  return hipGetLastError();
}

int launch_dequantize(int type, const CodeArgs &a, int block_rows, void *stream) {
  const Walk w = walk_of(a);
  if (w.groups > kMaxGroups) return hipErrorInvalidConfiguration;
  const int shift = block_rows == 1 ? 0 : 7;
#define CALL(T) dequantize_kernel<T><<<dim3((unsigned)w.groups), 256, 0, static_cast<hipStream_t>(stream)>>>(a, w, shift)
  FMM_TYPES(type, CALL);
#undef CALL
  return hipGetLastError();
}

}  // namespace f8
}  // namespace fmm
