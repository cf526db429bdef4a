// The 8-bit linear layer's entry points: argument checks and launches.
#include <cmath>

#include "internal.h"
#include "q8.h"

namespace {

using namespace fmm::q8;

bool is_type(int type) { return type == FMM_F32 || type == FMM_BF16 || type == FMM_F16; }
bool aligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// a buffer that is read or written whole: there, and aligned
bool good(const void *p, size_t bytes) { return p && aligned(p, bytes); }
// one that may be left out
bool fine(const void *p, size_t bytes) { return aligned(p, bytes); }

int check_scratch(const void *p, size_t have, size_t need, size_t align) {
  if (need == 0) return FMM_OK;
  return good(p, align) && have >= need ? FMM_OK : FMM_ERR_WORKSPACE;
}

int check_norm(const fmm_norm_desc *d) {
  if (!d || !is_type(d->type) || d->rows < 0 || d->cols < 0) return FMM_ERR_ARG;
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return FMM_ERR_ARG;
  if (d->cols == 0) return FMM_ERR_SHAPE;
  if (d->rows > kMaxRows || d->cols > kMaxCols) return FMM_ERR_UNSUPPORTED;
  return FMM_OK;
}

int check_linear(const fmm_q8_desc *d) {
  if (!d || !is_type(d->type) || d->M < 0 || d->N < 0 || d->K < 0) return FMM_ERR_ARG;
  if (d->K > kMaxK || d->M > kMaxRows || d->N > kMaxRows) return FMM_ERR_UNSUPPORTED;
  if (d->M * d->N > kMaxOutputs) return FMM_ERR_UNSUPPORTED;
  return FMM_OK;
}

int check_grad(const fmm_q8_desc *d) {
  const int st = check_linear(d);
  if (st != FMM_OK) return st;
  if (d->M > kMaxGradDim || d->N > kMaxGradDim) return FMM_ERR_UNSUPPORTED;
  const int64_t most = kMaxGradElements;
  return d->M * d->N > most || d->M * d->K > most || d->N * d->K > most ? FMM_ERR_UNSUPPORTED : FMM_OK;
}

// the int8 product's sizes
GemmProblem product(const fmm_q8_desc &d) {
  GemmProblem p = {};
  p.pitch_a = p.pitch_b = pitch_of(d.K);
  p.M = (int)d.M;
  p.N = (int)d.N;
  p.steps = (int)(pitch_of(d.K) / kGroup);
  p.parts = 1;
  return p;
}

size_t norm_grad_scratch(const fmm_norm_desc &d) {
  return d.rows == 0 ? 0 : sizeof(float) * (size_t)norm_grad_partials(d.type, d.rows, d.cols) * (size_t)d.cols;
}

}  // namespace

extern "C" {

int64_t fmm_q8_pitch(int64_t cols) { return cols < 0 ? -1 : pitch_of(cols); }

int fmm_q8_quantize(int type, int64_t rows, int64_t cols, const void *dX, int8_t *dCodes, float *dScales, void *stream) {
  if (!is_type(type) || rows < 0 || cols < 0) return FMM_ERR_ARG;
  if (rows > kMaxRows || cols > kMaxCols) return FMM_ERR_UNSUPPORTED;
  if (rows == 0) return FMM_OK;
  if (!good(dScales, 4)) return FMM_ERR_ARG;
  if (cols > 0 && (!good(dX, type_bytes(type)) || !good(dCodes, 16))) return FMM_ERR_ARG;
  RowArgs a = {};
  a.x = dX;
  a.codes = dCodes;
  a.scales = dScales;
  a.rows = rows;
  a.cols = cols;
  a.pitch = pitch_of(cols);
  return fmm::hip_status(launch_quantize(type, a, stream));
}

int fmm_q8_dequantize(int type, int64_t rows, int64_t cols, int group, const int8_t *dCodes, const float *dScales,
                      void *dOut, void *stream) {
  if (!is_type(type) || rows < 0 || cols < 0 || (group != 0 && group != kGroup)) return FMM_ERR_ARG;
  if (rows > kMaxRows || cols > kMaxCols) return FMM_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return FMM_OK;
  if (!good(dCodes, 16) || !good(dScales, 4) || !good(dOut, type_bytes(type))) return FMM_ERR_ARG;
  DequantArgs a = {dCodes, dScales, dOut, rows, cols, pitch_of(cols), group};
  return fmm::hip_status(launch_dequantize(type, a, stream));
}

int fmm_rmsnorm_q8(const fmm_norm_desc *desc, const void *dX, const void *dResidual, const void *dGain, void *dH,
                   int8_t *dCodes, float *dScales, int8_t *dSaved, float *dSavedScales, float *dRstd, void *stream) {
  const int st = check_norm(desc);
  if (st != FMM_OK) return st;
  if (desc->rows == 0) return FMM_OK;
  const size_t e = type_bytes(desc->type);
  if (!good(dX, e) || !fine(dResidual, e) || !fine(dGain, e) || !fine(dH, e)) return FMM_ERR_ARG;
  if (!good(dCodes, 16) || !good(dScales, 4) || !good(dRstd, 4)) return FMM_ERR_ARG;
  if (!dSaved != !dSavedScales || !fine(dSaved, 16) || !fine(dSavedScales, 4)) return FMM_ERR_ARG;
  if (desc->cols > kMaxHeldCols && dH && (dH == dX || dH == dResidual)) return FMM_ERR_UNSUPPORTED;
  RowArgs a = {dX, dResidual, dGain, dH, dCodes, dScales, dSaved, dSavedScales, dRstd,
               desc->rows, desc->cols, pitch_of(desc->cols), desc->eps};
  return fmm::hip_status(launch_rmsnorm(desc->type, a, stream));
}

int fmm_rmsnorm_q8_backward_scratch_size(const fmm_norm_desc *desc, size_t *bytes) {
  if (!bytes) return FMM_ERR_ARG;
  const int st = check_norm(desc);
  if (st != FMM_OK) return st;
  *bytes = norm_grad_scratch(*desc);
  return FMM_OK;
}

int fmm_rmsnorm_q8_backward(const fmm_norm_desc *desc, const void *dDy, const void *dDh, const void *dH,
                            const int8_t *dSaved, const float *dSavedScales, const float *dRstd, const void *dGain,
                            void *dDx, float *dDgain, void *dScratch, size_t scratch_bytes, void *stream) {
  const int st = check_norm(desc);
  if (st != FMM_OK) return st;
  if (!fine(dDgain, 4)) return FMM_ERR_ARG;
  const size_t e = type_bytes(desc->type);
  if (desc->rows > 0) {
    if (!good(dDy, e) || !fine(dDh, e) || !fine(dH, e) || !fine(dGain, e) || !good(dRstd, 4) || !good(dDx, e))
      return FMM_ERR_ARG;
    if (!dH && (!good(dSaved, 16) || !good(dSavedScales, 4))) return FMM_ERR_ARG;
    if (dDx == dDy || dDx == dH) return FMM_ERR_ARG;
    const int ws = dDgain ? check_scratch(dScratch, scratch_bytes, norm_grad_scratch(*desc), 16) : FMM_OK;
    if (ws != FMM_OK) return ws;
  }
  NormGradArgs a = {dDy, dDh, dH, dGain, dSaved, dSavedScales, dRstd, dDx, dDgain, static_cast<float *>(dScratch),
                    desc->rows, desc->cols, pitch_of(desc->cols)};
  return fmm::hip_status(launch_rmsnorm_grad(desc->type, a, stream));
}

const char *fmm_q8_matmul_kernel(const fmm_q8_desc *desc) {
  if (check_linear(desc) != FMM_OK) return nullptr;
  return matmul_kernel_name(product(*desc), fmm::compute_units());
}

int fmm_q8_matmul(const fmm_q8_desc *desc, const int8_t *dA, const float *dSa, const int8_t *dW, const float *dSw,
                  const float *dBias, void *dC, void *stream) {
  const int st = check_linear(desc);
  if (st != FMM_OK) return st;
  const int64_t M = desc->M, N = desc->N, K = desc->K;
  if (M == 0 || N == 0) return FMM_OK;
  if (K > 0 && (!good(dA, 16) || !good(dW, 16))) return FMM_ERR_ARG;
  if (!good(dSa, 4) || !good(dSw, 4) || !fine(dBias, 4) || !good(dC, type_bytes(desc->type))) return FMM_ERR_ARG;
  GemmProblem p = product(*desc);
  p.A = reinterpret_cast<const uint8_t *>(dA);
  p.B = reinterpret_cast<const uint8_t *>(dW);
  p.sa = dSa;
  p.sw = dSw;
  p.bias = dBias;
  p.C = dC;
  return fmm::hip_status(launch_matmul(desc->type, p, fmm::compute_units(), stream));
}

int fmm_q8_linear_backward_scratch_size(const fmm_q8_desc *desc, size_t *bytes) {
  if (!bytes) return FMM_ERR_ARG;
  const int st = check_grad(desc);
  if (st != FMM_OK) return st;
  *bytes = grad_scratch(desc->type, desc->M, desc->N, desc->K, fmm::compute_units());
  return FMM_OK;
}

int fmm_q8_linear_backward(const fmm_q8_desc *desc, const void *dDy, const int8_t *dA, const float *dSa,
                           const int8_t *dW, const float *dSw, void *dDx, void *dDw, float *dDbias, void *dScratch,
                           size_t scratch_bytes, void *stream) {
  const int st = check_grad(desc);
  if (st != FMM_OK) return st;
  const int64_t M = desc->M, N = desc->N, K = desc->K;
  const size_t e = type_bytes(desc->type);
  if (!fine(dDx, e) || !fine(dDw, e) || !fine(dDbias, 4)) return FMM_ERR_ARG;
  // an empty gradient is not wanted
  if (M * K == 0) dDx = nullptr;
  if (N * K == 0) dDw = nullptr;
  if (N == 0) dDbias = nullptr;
  if (!dDx && !dDw && !dDbias) return FMM_OK;
  if (M > 0 && N > 0) {
    if (!good(dDy, 16)) return FMM_ERR_ARG;
    if (dDx && (!good(dW, 16) || !good(dSw, 4))) return FMM_ERR_ARG;
    if (dDw && (!good(dA, 16) || !good(dSa, 4))) return FMM_ERR_ARG;
  }
  const int ncu = fmm::compute_units();
  const int ws = check_scratch(dScratch, scratch_bytes, grad_scratch(desc->type, M, N, K, ncu), 256);
  if (ws != FMM_OK) return ws;
  GradArgs a = {dDy, dA, dW, dSa, dSw, dDx, dDw, dDbias, static_cast<uint8_t *>(dScratch), M, N, K};
  return fmm::hip_status(launch_linear_grad(desc->type, a, ncu, stream));
}

const char *fmm_q8_linear_backward_kernel(const fmm_q8_desc *desc, int want_dx, int want_dw, int32_t runs[2]) {
  if (check_grad(desc) != FMM_OK) return nullptr;
  const int64_t M = desc->M, N = desc->N, K = desc->K;
  return linear_grad_kernel_name(desc->type, M, N, K, want_dx && M * K > 0, want_dw && N * K > 0, fmm::compute_units(), runs);
}

}  // extern "C"
