// The e4m3 linear layers' and the clipping's entry points: argument checks and launches.
#include <cmath>
#include <new>
#include <vector>

#include "f8.h"
#include "internal.h"

namespace {

using namespace fmm::f8;

bool is_type(int type) { return type == FMM_F32 || type == FMM_BF16 || type == FMM_F16; }
bool aligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
bool good(const void *p, size_t bytes) { return p && aligned(p, bytes); }

// a matrix with its sides padded
bool fits(int64_t rows, int64_t cols) {
  return rows <= kMaxElements && (rows == 0 || pitch_of(cols) <= kMaxElements / rows);
}

int check_codes(int type, int64_t count, int64_t rows, int64_t cols) {
  if (!is_type(type) || count < 0 || rows < 0 || cols < 0) return FMM_ERR_ARG;
  if (count > kMaxDim || rows > (1ll << 30) || cols > kMaxDim) return FMM_ERR_UNSUPPORTED;
  // (weights of a block each are padded to 128 rows)
  if (count > 1 ? !fits(count * round_up(rows, kBlock), cols) : !fits(rows, cols)) return FMM_ERR_UNSUPPORTED;
  return FMM_OK;
}

int check(const fmm_f8_desc *d, const int32_t *offsets, bool call) {
  if (!d || !is_type(d->type) || d->rows < 0 || d->N < 0 || d->K < 0 || d->experts < 1) return FMM_ERR_ARG;
  if (d->rows > kMaxDim || d->N > kMaxDim || d->K > kMaxDim || d->experts > kMaxExperts) return FMM_ERR_UNSUPPORTED;
  const int64_t rows = round_up(d->rows, kBlock) + kBlock * d->experts;
  if (!fits(rows, d->N) || !fits(rows, d->K) || !fits(d->experts * pitch_of(d->N), d->K)) return FMM_ERR_UNSUPPORTED;
  if (call && ((!offsets && d->experts > 1) || !aligned(offsets, 4))) return FMM_ERR_ARG;
  return FMM_OK;
}

Product product(const fmm_f8_desc &d) {
  Product p = {};
  p.a.pitch = p.b.pitch = pitch_of(d.K);
  p.a.scale_pitch = p.b.scale_pitch = scale_pitch_of(d.K);
  p.b.expert_codes = d.N * p.b.pitch;
  p.b.expert_scales = (d.N + kBlock - 1) / kBlock * p.b.scale_pitch;
  p.experts = (int)d.experts;
  p.rows = p.M = (int)d.rows;
  p.N = (int)d.N;
  p.steps = (int)(p.a.pitch / kBlock);
  p.out_bytes = type_bytes(d.type);
  return p;
}

}  // namespace

extern "C" {

int64_t fmm_f8_scale_pitch(int64_t cols) { return cols < 0 ? -1 : scale_pitch_of(cols); }

int fmm_f8_quantize(int type, int64_t rows, int64_t cols, const void *dX, uint8_t *dCodes, uint8_t *dScales, void *stream) {
  const int st = check_codes(type, 1, rows, cols);
  if (st != FMM_OK) return st;
  if (rows == 0 || cols == 0) return FMM_OK;
  if (!good(dX, type_bytes(type)) || !good(dCodes, 16) || !good(dScales, 16)) return FMM_ERR_ARG;
  const CodeArgs a = {const_cast<void *>(dX), dCodes, dScales, 1, rows, cols, pitch_of(cols), scale_pitch_of(cols)};
  return fmm::hip_status(launch_quantize(type, a, stream));
}

int fmm_f8_quantize_weight(int type, int64_t count, int64_t rows, int64_t cols, const void *dX, uint8_t *dCodes,
                           uint8_t *dScales, void *stream) {
  const int st = check_codes(type, count, rows, cols);
  if (st != FMM_OK) return st;
  if (count == 0 || rows == 0 || cols == 0) return FMM_OK;
  if (!good(dX, type_bytes(type)) || !good(dCodes, 16) || !good(dScales, 16)) return FMM_ERR_ARG;
  const CodeArgs a = {const_cast<void *>(dX), dCodes, dScales, count, rows, cols, pitch_of(cols), scale_pitch_of(cols)};
  return fmm::hip_status(launch_quantize_blocks(type, a, stream));
}

int fmm_f8_dequantize(int type, int64_t count, int64_t rows, int64_t cols, int block_rows, const uint8_t *dCodes,
                      const uint8_t *dScales, void *dOut, void *stream) {
  const int st = check_codes(type, count, rows, cols);
  if (st != FMM_OK) return st;
  if (block_rows != 1 && block_rows != kBlock) return FMM_ERR_ARG;
  if (count == 0 || rows == 0 || cols == 0) return FMM_OK;
  if (!good(dCodes, 16) || !good(dScales, 16) || !good(dOut, type_bytes(type))) return FMM_ERR_ARG;
  const CodeArgs a = {dOut, const_cast<uint8_t *>(dCodes), const_cast<uint8_t *>(dScales), count, rows, cols,
                      pitch_of(cols), scale_pitch_of(cols)};
  return fmm::hip_status(launch_dequantize(type, a, block_rows, stream));
}

int fmm_f8_matmul(const fmm_f8_desc *desc, const uint8_t *dA, const uint8_t *dSa, const uint8_t *dW, const uint8_t *dSw,
                  const int32_t *dOffsets, const float *dBias, void *dC, void *stream) {
  const int st = check(desc, dOffsets, true);
  if (st != FMM_OK) return st;
  if (desc->rows == 0 || desc->N == 0) return FMM_OK;
  if (desc->K > 0 && (!good(dA, 16) || !good(dW, 16) || !good(dSa, 16) || !good(dSw, 16))) return FMM_ERR_ARG;
  if (!aligned(dBias, 4) || !good(dC, type_bytes(desc->type))) return FMM_ERR_ARG;
  Product p = product(*desc);
  p.a.codes = dA;
  p.a.scales = dSa;
  p.b.codes = dW;
  p.b.scales = dSw;
  p.offsets = dOffsets;
  p.bias = dBias;
  p.C = dC;
  return fmm::hip_status(launch_matmul(desc->type, p, fmm::compute_units(), stream));
}

const char *fmm_f8_matmul_kernel(const fmm_f8_desc *desc) {
  if (check(desc, nullptr, false) != FMM_OK) return nullptr;
  return matmul_kernel_name(desc->type, product(*desc), fmm::compute_units());
}

int fmm_f8_linear_backward_scratch_size(const fmm_f8_desc *desc, size_t *bytes) {
  if (!bytes) return FMM_ERR_ARG;
  const int st = check(desc, nullptr, false);
  if (st != FMM_OK) return st;
  *bytes = grad_scratch(desc->type, desc->rows, desc->experts, desc->N, desc->K, fmm::compute_units());
  return FMM_OK;
}

int fmm_f8_linear_backward(const fmm_f8_desc *desc, const void *dDy, const uint8_t *dA, const uint8_t *dSa,
                           const uint8_t *dW, const uint8_t *dSw, const int32_t *dOffsets, void *dDx, void *dDw,
                           float *dDbias, void *dScratch, size_t scratch_bytes, void *stream) {
  const int st = check(desc, dOffsets, true);
  if (st != FMM_OK) return st;
  const int64_t rows = desc->rows, N = desc->N, K = desc->K;
  const size_t e = type_bytes(desc->type);
  if (!aligned(dDx, e) || !aligned(dDw, e) || !aligned(dDbias, 4)) return FMM_ERR_ARG;
  // an empty gradient is not wanted
  if (rows * K == 0) dDx = nullptr;
  if (N * K == 0) dDw = nullptr;
  if (N == 0) dDbias = nullptr;
  if (!dDx && !dDw && !dDbias) return FMM_OK;
  if (rows > 0 && N > 0) {
    if (!good(dDy, e)) return FMM_ERR_ARG;
    if (dDx && (!good(dW, 16) || !good(dSw, 16))) return FMM_ERR_ARG;
    if (dDw && (!good(dA, 16) || !good(dSa, 16))) return FMM_ERR_ARG;
  }
  const int ncu = fmm::compute_units();
  const size_t need = grad_scratch(desc->type, rows, desc->experts, N, K, ncu);
  if (need > 0 && (!good(dScratch, 256) || scratch_bytes < need)) return FMM_ERR_WORKSPACE;
  const GradArgs a = {dDy, dA, dSa, dW, dSw, dOffsets, dDx, dDw, dDbias, static_cast<uint8_t *>(dScratch),
                      rows, desc->experts, N, K};
  return fmm::hip_status(launch_grad(desc->type, a, ncu, stream));
}

const char *fmm_f8_linear_backward_kernel(const fmm_f8_desc *desc, int want_dx, int want_dw) {
  if (check(desc, nullptr, false) != FMM_OK) return nullptr;
  return grad_kernel_name(desc->type, desc->rows, desc->experts, desc->N, desc->K, want_dx && desc->rows * desc->K > 0,
                          want_dw && desc->N * desc->K > 0, fmm::compute_units());
}

size_t fmm_clip_scratch_size(void) { return kClipBlocks * sizeof(double); }

int fmm_clip(const int32_t *types, const int64_t *sizes, void *const *dIn, void *const *dOut, int64_t count, float most,
             float *dNorm, void *dScratch, size_t scratch_bytes, void *stream) {
  if (count < 0 || !(most >= 0.0f) || !good(dNorm, 4)) return FMM_ERR_ARG;
  if (count > kMaxClipTensors) return FMM_ERR_UNSUPPORTED;
  if (count > 0 && (!types || !sizes || !dIn || !dOut)) return FMM_ERR_ARG;
  std::vector<Tensor> t;
  try {
    t.resize((size_t)count);
  } catch (const std::bad_alloc &) {
    return FMM_ERR_NOMEM;
  }
  int64_t left = kMaxClipElements;
  for (int64_t i = 0; i < count; ++i) {
    if (!is_type(types[i]) || sizes[i] < 0) return FMM_ERR_ARG;
    if (sizes[i] > left) return FMM_ERR_UNSUPPORTED;
    left -= sizes[i];
    const size_t e = type_bytes(types[i]);
    if (sizes[i] > 0 && (!good(dIn[i], e) || !good(dOut[i], e))) return FMM_ERR_ARG;
    t[(size_t)i] = {dIn[i], dOut[i], sizes[i], types[i]};
  }
  if (!good(dScratch, 8) || scratch_bytes < fmm_clip_scratch_size()) return FMM_ERR_WORKSPACE;
  return fmm::hip_status(launch_clip(t.data(), (int)count, most, dNorm, static_cast<double *>(dScratch), stream));
}

}  // extern "C"
