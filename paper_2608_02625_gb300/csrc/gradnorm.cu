// The norm over all gradients of a model, and clipping by it.
//
//   norm = sqrt(sum over every element of every tensor of x^2)
//   out  = x min(1, max_norm / (norm + 1e-6))
//
// Two launches over the same chunks of the tensors. The first sums squares: a
// thread adds a chunk's in fp32 (up to 128, in eight sums) and the chunks' in fp64,
// and each CTA leaves one fp64 sum in the caller's workspace. The second adds those
// in a fixed order (every CTA for itself: a thousand numbers) and scales, walking the
// chunks from the last to the first, so that what the first launch read last may still
// be in L2; where nothing changes (no clipping, in place) it ends there. (Both in one
// launch, a cluster of 16 CTAs for a few small tensors, took 9.9 us for 48 of 2000 fp32
// elements, the two launches 8.9.)
// A chunk whose fp32 squares may have over- or underflowed (|x| above about 2^60,
// or all of it below 2^-40) is summed again in fp64. The tensors' addresses travel
// as kernel parameters, so a captured call needs no copy of a table.
//
// HBM bounds it: two reads and a write of everything. 310 M bf16 elements (621 MB): the
// squares 91 us (eight CTAs an SM; four: 98), the scaling about 200 (three CTAs, whose
// eight vectors a thread in flight take 80 registers), of 274 at the copy rate.
#include <cuda_bf16.h>

#include <cstdint>

#include "dlm_common.cuh"
#include "dlm_internal.h"

namespace dlm {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = kThreads * 8;  // chunks are multiples of this many elements
constexpr int kScaleCtas = 3 * 152;

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

// This thread's share of the squares of x[0, n): at most 17 in each of eight sums, whatever the
// type and alignment. (Four sums of 32 for fp32: 155 M elements, norm and scaling, 300 instead of
// 304 us, and up to 18 roundings of the norm instead of 11. Single elements in one sum: 68, and
// 310 M of bf16 460 us instead of 300, the norm alone.)
template <typename T>
__device__ double squares(const T* x, int64_t n, bool vectors) {
  constexpr int kPer = 16 / sizeof(T), kLoads = 4;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  uint32_t any = 0;
  const int vecs = vectors ? static_cast<int>(n / kPer) : 0, whole = vecs * kPer;
  const Vec<T>* xv = reinterpret_cast<const Vec<T>*>(x);
  for (int i = threadIdx.x; i < vecs; i += kThreads * kLoads) {
    Vec<T> v[kLoads] = {};
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (i + k * kThreads < vecs) v[k] = xv[i + k * kThreads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const float f = f32_of(v[k].e[e]);
        float& a = acc[(k * kPer + e) % 8];
        a = fmaf(f, f, a);
        any |= bits_of(f);
      }
  }
  for (int i = whole + threadIdx.x; i < n; i += kThreads * 8) {
    float f[8] = {};
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i + k * kThreads < n) f[k] = f32_of(x[i + k * kThreads]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      acc[k] = fmaf(f[k], f[k], acc[k]);
      any |= bits_of(f[k]);
    }
  }
  const float s = ((acc[0] + acc[1]) + (acc[2] + acc[3])) + ((acc[4] + acc[5]) + (acc[6] + acc[7]));
  if (any == 0 || (s >= 0x1p-80f && s <= 0x1p120f)) return s;
  double t = 0.0;
  for (int i = threadIdx.x; i < vecs; i += kThreads)
    for (int e = 0; e < kPer; ++e) t += static_cast<double>(f32_of(x[i * kPer + e])) * f32_of(x[i * kPer + e]);
  for (int i = whole + threadIdx.x; i < n; i += kThreads) t += static_cast<double>(f32_of(x[i])) * f32_of(x[i]);
  return t;
}

__device__ __forceinline__ Vec<float> scaled(const Vec<float>& v, float c1, float c2) {
  Vec<float> o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o.e[e] = v.e[e] * c1 * c2;
  return o;
}
__device__ __forceinline__ Vec<__nv_bfloat16> scaled(const Vec<__nv_bfloat16>& v, float c1, float c2) {
  Vec<__nv_bfloat16> o;
  uint32_t* w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
  for (int e = 0; e < 8; e += 2) w[e / 2] = pack_bf16x2(f32_of(v.e[e]) * c1 * c2, f32_of(v.e[e + 1]) * c1 * c2);
  return o;
}

// Scales x[0, n) by c1 c2 (c2 = 1 unless the factor is below fp32's normal range).
template <typename T>
__device__ void scale(const T* x, T* out, int64_t n, bool vectors, float c1, float c2) {
  constexpr int kPer = 16 / sizeof(T), kLoads = 8;
  const int vecs = vectors ? static_cast<int>(n / kPer) : 0, whole = vecs * kPer;
  const float4* xv = reinterpret_cast<const float4*>(x);
  float4* ov = reinterpret_cast<float4*>(out);
  for (int i = threadIdx.x; i < vecs; i += kThreads * kLoads) {
    float4 v[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (i + k * kThreads < vecs) v[k] = __ldcs(xv + i + k * kThreads);
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (i + k * kThreads < vecs) {
        const Vec<T> o = scaled(*reinterpret_cast<const Vec<T>*>(&v[k]), c1, c2);
        __stcs(ov + i + k * kThreads, *reinterpret_cast<const float4*>(&o));
      }
  }
  for (int i = whole + threadIdx.x; i < n; i += kThreads) out[i] = static_cast<T>(f32_of(x[i]) * c1 * c2);
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

// The squares of chunk c.
template <typename Tab>
__device__ double chunk_squares(const Tab& tab, int c) {
  const Tensor& t = find(tab, c);
  const int64_t at = static_cast<int64_t>(c - t.first) * tab.chunk;
  const int64_t n = t.n - at < tab.chunk ? t.n - at : tab.chunk;
  return t.flags & kBf16 ? squares(static_cast<const __nv_bfloat16*>(t.in) + at, n, t.flags & kVectors)
                         : squares(static_cast<const float*>(t.in) + at, n, t.flags & kVectors);
}

// The factor as two numbers: below 2^-100 it may be below fp32's normal range.
struct Factor {
  float c1, c2;
};
__device__ __forceinline__ Factor factor_of(double norm, float max_norm) {
  double c = static_cast<double>(max_norm) / (norm + 1e-6);
  if (c >= 1.0) c = 1.0;  // a NaN stays one
  return {static_cast<float>(c < 0x1p-100 ? c * 0x1p100 : c), c < 0x1p-100 ? 0x1p-100f : 1.f};
}

template <typename Tab>
__device__ void chunk_scale(const Tab& tab, int c, const Factor& f) {
  const Tensor& t = find(tab, c);
  if (f.c1 == 1.f && t.in == t.out) return;
  const int64_t at = static_cast<int64_t>(c - t.first) * tab.chunk;
  const int64_t n = t.n - at < tab.chunk ? t.n - at : tab.chunk;
  if (t.flags & kBf16)
    scale(static_cast<const __nv_bfloat16*>(t.in) + at, static_cast<__nv_bfloat16*>(t.out) + at, n, t.flags & kVectors, f.c1, f.c2);
  else
    scale(static_cast<const float*>(t.in) + at, static_cast<float*>(t.out) + at, n, t.flags & kVectors, f.c1, f.c2);
}

template <int kTensors>
__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const __grid_constant__ Table<kTensors> tab) {
  wait_for_previous();
  double s = 0.0;
  for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) s += chunk_squares(tab, c);
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
  const Factor f = factor_of(norm, tab.max_norm);
  for (int c = tab.chunks - 1 - static_cast<int>(blockIdx.x); c >= 0; c -= gridDim.x) chunk_scale(tab, c, f);
}

template <int kTensors>
void fill(const GradArgs& a, int first, Table<kTensors>* tab, int64_t target) {
  tab->count = a.count - first < kTensors ? a.count - first : kTensors;
  int64_t total = 0;
  for (int i = 0; i < tab->count; ++i) total += a.grads[first + i].n;
  int64_t chunk = (total / target + kUnit - 1) / kUnit * kUnit;
  if (chunk < kUnit) chunk = kUnit;
  if (chunk > 16 * kUnit) chunk = 16 * kUnit;
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
    fill(a, l * kTensors, &tab, 2 * kGradParts);
    int ctas = tab.chunks < kGradParts ? tab.chunks : kGradParts;
    if (ctas < 1) ctas = 1;
    tab.part = a.workspace + written;
    written += ctas;  // (of the first phase)
    tab.parts = a.workspace;
    tab.n_parts = a.parts;
    tab.max_norm = a.max_norm;
    tab.norm = l == 0 ? a.norm : nullptr;
    // As many CTAs as run at once: a second wave would wait for the first one's chunks (53 MB:
    // 49 us with 1216, 34).
    if (scale_phase && ctas > kScaleCtas) ctas = kScaleCtas;
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
