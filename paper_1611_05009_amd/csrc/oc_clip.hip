// Global norm of many gradients, and their clipping.
//
//   norm = sqrt(sum over all tensors of g^2),
//   out = g min(1, max_norm / (norm + 1e-6)).
//
// Memory bound: no output can be written before every input has been read, so
// the inputs are read twice (the second time from the cache where they fit)
// and the outputs written once.  The tensors' addresses travel in the
// launch's arguments, up to kClipBatch of them at a time; a launch treats
// its tensors as one sequence of chunks.  Squares are added up in double: a
// float's square can exceed float, and double addition costs nothing beside
// the loads.  The partial sums are added in one fixed order.
#include "oc_rows.h"
#include "oc_sequence.h"

namespace oci {
namespace {

using namespace ocr;

// Calls f(tensor, first element, elements) for the workgroup's chunks, in
// ascending order or from the end backwards.
template <bool BACK, class F>
__device__ __forceinline__ void each_chunk(const ClipBatch& b, F f) {
  const uint32_t n = b.first[b.n];
  int t = BACK ? b.n - 1 : 0;
  for (uint32_t k = blockIdx.x; k < n; k += gridDim.x) {
    const uint32_t c = BACK ? n - 1 - k : k;
    if constexpr (BACK) {
      while (b.first[t] > c) --t;
    } else {
      while (b.first[t + 1] <= c) ++t;
    }
    const int64_t at = (int64_t)(c - b.first[t]) * kClipChunk;
    const int64_t left = b.count[t] - at;
    f(t, at, (int)(left < kClipChunk ? left : kClipChunk));
  }
}

template <class T>
__device__ __forceinline__ double square_sum(const T* p, int n) {
  double s = 0;
  const bool vec = ((uintptr_t)p & 15) == 0;
  const int body = vec ? n / 8 : 0;
#pragma unroll 4
  for (int v = (int)threadIdx.x; v < body; v += 256) {
    const f32x8 x = load8(p + 8 * v);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fma((double)x[i], (double)x[i], s);
  }
  for (int i = 8 * body + (int)threadIdx.x; i < n; i += 256) s = __builtin_fma((double)(float)p[i], (double)(float)p[i], s);
  return s;
}

// Sum over the workgroup, in every thread.
__device__ __forceinline__ double block_sum(double s) {
  __shared__ double part[4];
  for (int i = 32; i; i >>= 1) s += __shfl_xor(s, i);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(256) void k_square_sums(ClipBatch b, double* parts) {
  double s = 0;
  each_chunk<false>(b, [&](int t, int64_t at, int n) {
    if (b.type[t] == kF32) s += square_sum((const float*)b.in[t] + at, n);
    else if (b.type[t] == kF16) s += square_sum((const _Float16*)b.in[t] + at, n);
    else s += square_sum((const __bf16*)b.in[t] + at, n);
  });
  s = block_sum(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

template <class T>
__device__ __forceinline__ void scale_to(const T* p, T* q, int n, float f) {
  const int body = (((uintptr_t)p | (uintptr_t)q) & 15) == 0 ? n / 8 : 0;
#pragma unroll 4
  for (int v = (int)threadIdx.x; v < body; v += 256) store8(q + 8 * v, load8(p + 8 * v) * f);
  for (int i = 8 * body + (int)threadIdx.x; i < n; i += 256) store1(q + i, (float)p[i] * f);
}

__global__ __launch_bounds__(256) void k_clip(ClipBatch b, const double* parts, int n_parts, float max_norm, float* norm) {
  double s = 0;
  for (int i = (int)threadIdx.x; i < n_parts; i += 256) s += parts[i];
  const double root = sqrt(block_sum(s));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)root;
  const double r = (double)max_norm / (root + 1e-6);
  const float f = r < 1.0 ? (float)r : r != r ? __builtin_nanf("") : 1.f;
  // What the sums read last is what the caches still hold.
  each_chunk<true>(b, [&](int t, int64_t at, int n) {
    // A factor of one leaves what is clipped in place as it is.
    if (f == 1.f && b.in[t] == b.out[t]) return;
    if (b.type[t] == kF32) scale_to((const float*)b.in[t] + at, (float*)b.out[t] + at, n, f);
    else if (b.type[t] == kF16) scale_to((const _Float16*)b.in[t] + at, (_Float16*)b.out[t] + at, n, f);
    else scale_to((const __bf16*)b.in[t] + at, (__bf16*)b.out[t] + at, n, f);
  });
}

}  // namespace

hipError_t launch_square_sums(const ClipBatch& b, double* parts, int groups, hipStream_t s) {
  k_square_sums<<<(unsigned)groups, 256, 0, s>>>(b, parts);
  return hipGetLastError();
}

hipError_t launch_clip(const ClipBatch& b, const double* parts, int n_parts, float max_norm, float* norm, int groups,
                       hipStream_t s) {
  k_clip<<<(unsigned)groups, 256, 0, s>>>(b, parts, n_parts, max_norm, norm);
  return hipGetLastError();
}

}  // namespace oci
