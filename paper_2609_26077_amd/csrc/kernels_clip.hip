// The global norm of many tensors and clipping by it:
//   norm = sqrt(sum over all elements of squares), out = in min(1, most / (norm + 1e-6)).
//
// Two passes over the data, so HBM bounds them: squares are summed in binary64 (no
// magnitude that fp32 holds overflows or is lost) by at most kClipBlocks workgroups into a
// partial sum each; every workgroup of the second pass adds the partial sums in
// the same order and scales.  The second pass walks the tensors backwards, from
// what the first left in the last-level cache.  The tensors' addresses travel in the kernels'
// arguments, kTable of them a launch: nothing is copied to the device, and a captured call
// keeps its own.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "f8.h"
#include "q8_types.h"

namespace fmm {
namespace f8 {
namespace {

using q8::elem_t;
using q8::u32x4;

constexpr int kTable = kClipTable;
constexpr int kChunk = 8192;       // elements of a tensor that a workgroup takes at a time
constexpr int kScaleBlocks = 8192; // workgroups of the second pass, at most

struct Table {
  const void *in[kTable];
  void *out[kTable];
  int64_t n[kTable];
  int32_t first[kTable + 1];       // chunks before each tensor
  uint8_t type[kTable];
  int32_t count, chunks;
};
static_assert(sizeof(Table) <= 3900, "kernel arguments");

// the tensor of a chunk: the last one whose first chunk is not past it
__device__ __forceinline__ int tensor_of(const Table &t, int chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// A whole chunk's loads are under way at once: kLoads vectors a thread.
constexpr int kLoads = kChunk / (8 * 256);

template <int T>
struct Part {
  q8::Raw8<T> raw[kLoads];
  __device__ __forceinline__ Part(const void *in, int64_t n) {
    const elem_t<T> *p = static_cast<const elem_t<T> *>(in);
    const int at = 8 * threadIdx.x;
    if (n == kChunk) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) raw[u] = q8::raw8<T>(p + at + 2048 * u, 8);
    } else {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) raw[u] = q8::raw8<T>(p + at + 2048 * u, n - at - 2048 * u);
    }
  }
};

template <int T>
__device__ __forceinline__ double squares(const void *in, int64_t n) {
  const Part<T> x(in, n);
  double s = 0.0;
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    float v[8];
    q8::floats8<T>(x.raw[u], v);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fma((double)v[k], (double)v[k], s);
  }
  return s;
}

// eight consecutive elements, of which those before n exist; past the caches, but for tensors that begin
// off 16 bytes, whose lines are written in pieces that have to meet there
template <int T>
__device__ __forceinline__ void store(elem_t<T> *p, int64_t n, const float (&v)[8], bool stream) {
  if (n < 8 || !stream) {
    q8::store8<T>(p, n, v);
  } else if constexpr (T == FMM_F32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 w = {__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
      __builtin_nontemporal_store(w, reinterpret_cast<q8::u32x4_a4 *>(p + 4 * h));
    }
  } else {
    const u32x4 w = {q8::pack2<T>(v[0], v[1]), q8::pack2<T>(v[2], v[3]), q8::pack2<T>(v[4], v[5]), q8::pack2<T>(v[6], v[7])};
    __builtin_nontemporal_store(w, reinterpret_cast<q8::u32x4_a2 *>(p));
  }
}

// times c, or, where c is below fp32's normal numbers and would lose digits as one, times `ratio`
template <int T>
__device__ __forceinline__ void scale(const void *in, void *out, int64_t n, float c, double ratio) {
  const Part<T> x(in, n);
  elem_t<T> *q = static_cast<elem_t<T> *>(out) + 8 * threadIdx.x;
  const bool stream = reinterpret_cast<uintptr_t>(out) % 16 == 0;
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    float v[8];
    q8::floats8<T>(x.raw[u], v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = ratio < 0x1p-126 ? (float)(v[k] * ratio) : v[k] * c;
    store<T>(q + 2048 * u, n - 8 * (int)threadIdx.x - 2048 * u, v, stream);
  }
}

// the sum over the workgroup's 256 threads, in all of them
__device__ __forceinline__ double sum256(double s, double *share) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 63) == 0) share[threadIdx.x >> 6] = s;
  __syncthreads();
  s = (share[0] + share[1]) + (share[2] + share[3]);
  __syncthreads();
  return s;
}

__global__ __launch_bounds__(256) void squares_kernel(Table t, double *partial) {
  __shared__ double share[4];
  double s = 0.0;
  for (int c = blockIdx.x, i = tensor_of(t, c); c < t.chunks; c += gridDim.x) {
    while (c >= t.first[i + 1]) ++i;
    const int type = t.type[i];
    const int64_t at = (int64_t)(c - t.first[i]) * kChunk, n = min(t.n[i] - at, (int64_t)kChunk);
    const uint8_t *p = static_cast<const uint8_t *>(t.in[i]) + at * (type == FMM_F32 ? 4 : 2);
    s += type == FMM_F32 ? squares<FMM_F32>(p, n) : type == FMM_BF16 ? squares<FMM_BF16>(p, n) : squares<FMM_F16>(p, n);
  }
  s = sum256(s, share);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void clip_kernel(Table t, const double *partial, int partials, float most, float *norm) {
  __shared__ double share[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < partials; i += 256) s += partial[i];
  s = sqrt(sum256(s, share));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)s;
  const double ratio = s < INFINITY || isnan(s) ? (double)most / (s + 1e-6) : 0.0;   // (0 for a limit of infinity too)
  const float f = ratio > 1.0 ? 1.0f : (float)ratio;     // (NaN stays)
  for (int c = t.chunks - 1 - blockIdx.x, i = tensor_of(t, c); c >= 0; c -= gridDim.x) {
    while (c < t.first[i]) --i;
    const int type = t.type[i];
    if (f == 1.0f && t.in[i] == t.out[i]) continue;
    const int64_t at = (int64_t)(c - t.first[i]) * kChunk, n = min(t.n[i] - at, (int64_t)kChunk);
    const int64_t bytes = at * (type == FMM_F32 ? 4 : 2);
    const uint8_t *p = static_cast<const uint8_t *>(t.in[i]) + bytes;
    uint8_t *q = static_cast<uint8_t *>(t.out[i]) + bytes;
    if (type == FMM_F32) scale<FMM_F32>(p, q, n, f, ratio);
    else if (type == FMM_BF16) scale<FMM_BF16>(p, q, n, f, ratio);
    else scale<FMM_F16>(p, q, n, f, ratio);
  }
}

// The next launch's tensors, from `at` on (empty ones need no chunk).
int fill(const Tensor *t, int count, int at, Table &b) {
  b.count = b.chunks = 0;
  for (; at < count && b.count < kTable; ++at) {
    if (t[at].n == 0) continue;
    const int64_t chunks = (t[at].n + kChunk - 1) / kChunk;
    b.in[b.count] = t[at].in;
    b.out[b.count] = t[at].out;
    b.n[b.count] = t[at].n;
    b.type[b.count] = (uint8_t)t[at].type;
    b.first[b.count++] = b.chunks;
    b.chunks += (int)chunks;
  }
  b.first[b.count] = b.chunks;
  return at;
}

}  // namespace

int launch_clip(const Tensor *t, int count, float most, float *norm, double *partial, void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Table b;
  // Each launch's partial sums after those before it, kClipBlocks in all, so the first pass has fewer workgroups a launch
  // the more tensors there are, and gets slower (tensors of 1 M bf16 elements, all passes by their bytes: 120 in 127 us, 6.0
  // TB/s; 300 in 407, 4.6; 1000 in 1640, 3.9; 5000 in 21600, 1.5).
  const int each = kClipBlocks / std::max(1, (count + kTable - 1) / kTable);
  int partials = 0;
  for (int at = 0; at < count;) {
    at = fill(t, count, at, b);
    if (b.chunks == 0) continue;
    const int blocks = std::min(b.chunks, each);
    squares_kernel<<<dim3((unsigned)blocks), 256, 0, s>>>(b, partial + partials);
    partials += blocks;
  }
  bool told = false;
  for (int at = 0; at < count || !told;) {
    at = fill(t, count, at, b);
    if (b.chunks == 0 && told) continue;
    clip_kernel<<<dim3((unsigned)std::max(1, std::min(b.chunks, kScaleBlocks))), 256, 0, s>>>(b, partial, partials, most,
                                                                                      told ? nullptr : norm);
    told = true;
  }
  return hipGetLastError();
}

}  // namespace f8
}  // namespace fmm
