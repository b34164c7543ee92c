// The norm over all gradients of a model, and clipping by it.
//
//   norm = sqrt(sum over every element of every tensor of x^2)
//   out  = x min(1, max_norm / (norm + 1e-6))
//
// Two launches over the same chunks of the tensors. The first sums squares: a
// thread adds a chunk's in fp32 (up to 256, in eight sums) and the chunks' in fp64,
// and each CTA leaves one fp64 sum in the caller's workspace. The second adds those
// in a fixed order (every CTA for itself: a few hundred numbers) and scales,
// walking the chunks from the last to the first, so that what the first launch read
// last is still in L2; where nothing changes (no clipping, in place) it ends there.
// A chunk whose fp32 squares may have over- or underflowed (|x| above about 2^60,
// or all of it below 2^-40) is summed again in fp64. The tensors' addresses travel
// as kernel parameters, so a captured call needs no copy of a table.
#include <cuda_bf16.h>

#include <cstdint>

#include "dlm_common.cuh"
#include "dlm_internal.h"

namespace dlm {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = kThreads * 8;  // chunks are multiples of this many elements

struct Tensor {
  const void* in;
  void* out;
  int64_t n;
  int first;  // its first chunk
  int flags;  // kBf16, kVectors
};
constexpr int kBf16 = 1, kVectors = 2;

// Size 16, 128 or kGradTable: a call's parameters are copied whatever part of them is used.
template <int kTensors>
struct Table {
  Tensor t[kTensors];
  int count, chunks, chunk;   // tensors, chunks in all, elements a chunk
  double* part;               // this launch's sums, one a CTA
  const double* parts;        // every launch's
  int n_parts;
  float max_norm;
  float* norm;                // written by the first CTA of the launch that has it
};

__device__ __forceinline__ float f32_of(float x) { return x; }
__device__ __forceinline__ float f32_of(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T>
struct alignas(16) Vec {
  T e[16 / sizeof(T)];
};

template <typename Tab>
__device__ __forceinline__ const Tensor& find(const Tab& tab, int chunk) {
  int lo = 0, hi = tab.count - 1;  // the last tensor whose first chunk is not after `chunk`
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.t[mid].first <= chunk)
      lo = mid;
    else
      hi = mid - 1;
  }
  return tab.t[lo];
}

__device__ __forceinline__ uint32_t bits_of(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// This thread's share of the squares of x[0, n).
template <typename T>
__device__ double squares(const T* x, int64_t n, bool vectors) {
  constexpr int kPer = 16 / sizeof(T);
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  uint32_t any = 0;
  const int64_t whole = vectors ? n / kPer * kPer : 0;
#pragma unroll 4
  for (int64_t i = static_cast<int64_t>(threadIdx.x) * kPer; i < whole; i += kThreads * kPer) {
    const Vec<T> v = *reinterpret_cast<const Vec<T>*>(x + i);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const float f = f32_of(v.e[k]);
      acc[k] = fmaf(f, f, acc[k]);
      any |= bits_of(f);
    }
  }
#pragma unroll 4
  for (int64_t i = whole + threadIdx.x; i < n; i += kThreads) {
    const float f = f32_of(x[i]);
    acc[0] = fmaf(f, f, acc[0]);
    any |= bits_of(f);
  }
  const float s = ((acc[0] + acc[1]) + (acc[2] + acc[3])) + ((acc[4] + acc[5]) + (acc[6] + acc[7]));
  if (any == 0 || (s >= 0x1p-80f && s <= 0x1p120f)) return s;
  double t = 0.0;
  for (int64_t i = static_cast<int64_t>(threadIdx.x) * kPer; i < whole; i += kThreads * kPer)
    for (int k = 0; k < kPer; ++k) t += static_cast<double>(f32_of(x[i + k])) * f32_of(x[i + k]);
  for (int64_t i = whole + threadIdx.x; i < n; i += kThreads) t += static_cast<double>(f32_of(x[i])) * f32_of(x[i]);
  return t;
}

// Scales x[0, n) by c1 c2 (c2 = 1 unless the factor is below fp32's normal range).
template <typename T>
__device__ void scale(const T* x, T* out, int64_t n, bool vectors, float c1, float c2) {
  constexpr int kPer = 16 / sizeof(T);
  const int64_t whole = vectors ? n / kPer * kPer : 0;
#pragma unroll 4
  for (int64_t i = static_cast<int64_t>(threadIdx.x) * kPer; i < whole; i += kThreads * kPer) {
    Vec<T> v = *reinterpret_cast<const Vec<T>*>(x + i);
#pragma unroll
    for (int k = 0; k < kPer; ++k) v.e[k] = static_cast<T>(f32_of(v.e[k]) * c1 * c2);
    *reinterpret_cast<Vec<T>*>(out + i) = v;
  }
  for (int64_t i = whole + threadIdx.x; i < n; i += kThreads) out[i] = static_cast<T>(f32_of(x[i]) * c1 * c2);
}

// The sum of v over the block, in every thread.
__device__ double block_sum(double v) {
  __shared__ double sums[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) v += sums[i];
  return v;
}

template <int kTensors>
__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const __grid_constant__ Table<kTensors> tab) {
  wait_for_previous();
  double s = 0.0;
  for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
    const Tensor& t = find(tab, c);
    const int64_t at = static_cast<int64_t>(c - t.first) * tab.chunk;
    const int64_t n = t.n - at < tab.chunk ? t.n - at : tab.chunk;
    s += t.flags & kBf16 ? squares(static_cast<const __nv_bfloat16*>(t.in) + at, n, t.flags & kVectors)
                         : squares(static_cast<const float*>(t.in) + at, n, t.flags & kVectors);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) tab.part[blockIdx.x] = s;
}

template <int kTensors>
__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const __grid_constant__ Table<kTensors> tab) {
  wait_for_previous();
  double s = 0.0;
  for (int i = threadIdx.x; i < tab.n_parts; i += kThreads) s += tab.parts[i];
  const double norm = sqrt(block_sum(s));
  if (tab.norm && blockIdx.x == 0 && threadIdx.x == 0) *tab.norm = static_cast<float>(norm);
  double c = static_cast<double>(tab.max_norm) / (norm + 1e-6);
  if (c >= 1.0) c = 1.0;  // a NaN stays one
  // A factor below 2^-100 as two: it may be below fp32's normal range.
  const float c2 = c < 0x1p-100 ? 0x1p-100f : 1.f, c1 = static_cast<float>(c < 0x1p-100 ? c * 0x1p100 : c);
  for (int k = tab.chunks - 1 - static_cast<int>(blockIdx.x); k >= 0; k -= gridDim.x) {
    const Tensor& t = find(tab, k);
    if (c1 == 1.f && t.in == t.out) continue;
    const int64_t at = static_cast<int64_t>(k - t.first) * tab.chunk;
    const int64_t n = t.n - at < tab.chunk ? t.n - at : tab.chunk;
    if (t.flags & kBf16)
      scale(static_cast<const __nv_bfloat16*>(t.in) + at, static_cast<__nv_bfloat16*>(t.out) + at, n, t.flags & kVectors, c1, c2);
    else
      scale(static_cast<const float*>(t.in) + at, static_cast<float*>(t.out) + at, n, t.flags & kVectors, c1, c2);
  }
}

template <int kTensors>
void fill(const GradArgs& a, int first, Table<kTensors>* tab, int64_t target) {
  tab->count = a.count - first < kTensors ? a.count - first : kTensors;
  int64_t total = 0;
  for (int i = 0; i < tab->count; ++i) total += a.grads[first + i].n;
  int64_t chunk = (total / target + kUnit - 1) / kUnit * kUnit;
  if (chunk < kUnit) chunk = kUnit;
  if (chunk > 32 * kUnit) chunk = 32 * kUnit;
  int64_t chunks = 0;
  for (;; chunk *= 2) {  // until the chunks' number is an int
    chunks = 0;
    for (int i = 0; i < tab->count; ++i) chunks += (a.grads[first + i].n + chunk - 1) / chunk;
    if (chunks <= (1 << 30) || chunk >= (1 << 29)) break;
  }
  tab->chunk = static_cast<int>(chunk);
  tab->chunks = static_cast<int>(chunks);
  int at = 0;
  for (int i = 0; i < tab->count; ++i) {
    const GradTensor& g = a.grads[first + i];
    const bool vectors = ((reinterpret_cast<uintptr_t>(g.in) | reinterpret_cast<uintptr_t>(g.out)) & 15) == 0;
    tab->t[i] = {g.in, g.out, g.n, at, (g.is_bf16 ? kBf16 : 0) | (vectors ? kVectors : 0)};
    at += static_cast<int>((g.n + chunk - 1) / chunk);
  }
}

// The launches of one phase, kTensors tensors each.
template <int kTensors>
int launch_phase(const GradArgs& a, bool scale_phase, cudaStream_t stream) {
  const int launches = a.count > 0 ? (a.count + kTensors - 1) / kTensors : 1;
  int written = 0;
  Table<kTensors> tab;
  for (int l = 0; l < launches; ++l) {
    fill(a, l * kTensors, &tab, 4 * kGradParts);
    int ctas = tab.chunks < kGradParts ? tab.chunks : kGradParts;
    if (ctas < 1) ctas = 1;
    tab.part = a.workspace + written;
    written += ctas;
    tab.parts = a.workspace;
    tab.n_parts = a.parts;
    tab.max_norm = a.max_norm;
    tab.norm = l == 0 ? a.norm : nullptr;
    if (scale_phase && !a.scale) {
      tab.chunks = 0;
      ctas = 1;
    }
    const cudaError_t e = scale_phase ? launch_overlapped(grad_scale_kernel<kTensors>, dim3(ctas), kThreads, 0, stream, 1, true, tab)
                                      : launch_overlapped(grad_squares_kernel<kTensors>, dim3(ctas), kThreads, 0, stream, 1, true, tab);
    if (e != cudaSuccess) return fail(DLM_ERR_CUDA, "gradient norm launch: %s", cudaGetErrorString(e));
    if (scale_phase && !a.scale) break;
  }
  return written;
}

template <int kTensors>
int launch_both(GradArgs a, cudaStream_t stream) {
  const int parts = launch_phase<kTensors>(a, false, stream);
  if (parts < 0) return parts;
  a.parts = parts;
  const int st = launch_phase<kTensors>(a, true, stream);
  return st < 0 ? st : DLM_OK;
}

}  // namespace

int launch_clip_grad_norm(const GradArgs& a, cudaStream_t stream) {
  if (a.count <= 16) return launch_both<16>(a, stream);
  if (a.count <= 128) return launch_both<128>(a, stream);
  return launch_both<kGradTable>(a, stream);
}

}  // namespace dlm
