// Layer norm in front of the output projection, and its gradients.
//
//   mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps)
//   out  = xhat w + b              with xhat = (x - mean) rstd
//   dx   = rstd (a - (sum a + xhat sum a xhat) / d)      with a = dout w
//   dw   = sum over rows of dout xhat,   db = sum over rows of dout
//
// One pass over the rows: a row lives in the registers of a group of threads (a
// part of a warp, a warp, or a CTA), which takes its two sums over the centred
// values (not from sums of x and x^2, which cancel where the mean is large). Every
// group walks rows a grid apart, its weights kept in registers, the next row's
// loads issued before the sums of this one. In the gradient each thread also
// keeps the sums of its columns over the rows of its group; the CTAs' sums go to
// the caller's workspace and a second launch adds them in a fixed order, so the
// results do not depend on scheduling. All sums are fp32. Rows too wide for the
// registers of a CTA are read once for each sum, their columns' sums by a launch
// of their own.
#include <cuda_bf16.h>

#include <cstdint>

#include "dlm_common.cuh"
#include "dlm_internal.h"

namespace dlm {
namespace {

constexpr int kRowThreads = 256;    // a CTA of the kernels that hold rows in registers
constexpr int kWideThreads = 1024;  // a CTA of those that read a row again
constexpr int kHeldWidth = 8192;    // widest row held: 32 values of each kind a thread

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
  T e[VEC];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ float load_param(const void* p, int bf16, int i) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}

// The sums of v over the G threads of a row. G: a power of two up to 32 (groups
// inside a warp), or the whole block (a multiple of 32). `red` is not written
// again before every thread of the block has passed another barrier.
template <int NS>
__device__ __forceinline__ void row_sums(float (&v)[NS], int G, float (*red)[32]) {
  const int top = G < 32 ? G : 32;
  for (int o = top >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < NS; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (G <= 32) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < NS; ++k) red[k][warp] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NS; ++k) v[k] = lane < warps ? red[k][lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < NS; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
}

struct NormParams {
  const void* x;
  const void* w;
  const void* b;    // may be null
  const void* dy;   // gradient only
  void* out;        // out, or dx
  float* mean;      // written (may be null), or read
  float* rstd;
  float* part;      // gradient: [CTAs][2][d]; null where neither dw nor db is wanted
  int64_t N, s_x, s_dy, s_out;
  int d, G, w_bf16;
  float eps;
};

template <typename T, int VEC, int NV>
__device__ __forceinline__ void load_row(Pack<T, VEC> (&r)[NV], const void* base, int64_t off, int tid, int G, int d, bool any) {
  const T* p = static_cast<const T*>(base) + off;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (tid + i * G) * VEC;
    if (any && e < d)
      r[i] = *reinterpret_cast<const Pack<T, VEC>*>(p + e);
    else
#pragma unroll
      for (int k = 0; k < VEC; ++k) r[i].e[k] = from_f32<T>(0.f);
  }
}

// VEC: elements per load (16 bytes, or one where a base, a stride or d is not a
// multiple of that); NV: loads per thread and row.
template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(kRowThreads) norm_kernel(const NormParams p) {
  __shared__ float red[2][1][32];
  const int G = p.G, R = blockDim.x / G, g = threadIdx.x / G, tid = threadIdx.x % G, d = p.d;
  const float inv_d = 1.f / static_cast<float>(d);
  wait_for_previous();
  float w[NV * VEC], b[NV * VEC];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const int e = (tid + i * G) * VEC + k;
      w[i * VEC + k] = e < d ? load_param(p.w, p.w_bf16, e) : 0.f;
      b[i * VEC + k] = e < d && p.b ? load_param(p.b, p.w_bf16, e) : 0.f;
    }
  const int64_t step = static_cast<int64_t>(gridDim.x) * R;
  int64_t row = static_cast<int64_t>(blockIdx.x) * R + g;
  Pack<T, VEC> x[NV], next[NV];
  load_row<T, VEC, NV>(x, p.x, row * p.s_x, tid, G, d, row < p.N);
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * R; first < p.N; first += step, row += step) {
    load_row<T, VEC, NV>(next, p.x, (row + step) * p.s_x, tid, G, d, row + step < p.N);
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < VEC; ++k) s[0] += to_f32(x[i].e[k]);
    row_sums<1>(s, G, red[0]);
    const float mean = s[0] * inv_d;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if ((tid + i * G) * VEC < d)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float c = to_f32(x[i].e[k]) - mean;
          s[0] = fmaf(c, c, s[0]);
        }
    row_sums<1>(s, G, red[1]);
    const float rstd = 1.f / sqrtf(s[0] * inv_d + p.eps);
    if (row < p.N) {
      T* o = static_cast<T*>(p.out) + row * p.s_out;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int e = (tid + i * G) * VEC;
        if (e < d) {
          Pack<T, VEC> y;
#pragma unroll
          for (int k = 0; k < VEC; ++k)
            y.e[k] = from_f32<T>(fmaf((to_f32(x[i].e[k]) - mean) * rstd, w[i * VEC + k], b[i * VEC + k]));
          *reinterpret_cast<Pack<T, VEC>*>(o + e) = y;
        }
      }
      if (tid == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = next[i];
  }
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(kRowThreads) norm_grad_kernel(const NormParams p) {
  extern __shared__ float cols[];  // G <= 32: [2][R][G * NV * VEC]
  __shared__ float red[2][2][32];
  const int G = p.G, R = blockDim.x / G, g = threadIdx.x / G, tid = threadIdx.x % G, d = p.d;
  const float inv_d = 1.f / static_cast<float>(d);
  wait_for_previous();
  float w[NV * VEC], dw[NV * VEC], db[NV * VEC];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const int e = (tid + i * G) * VEC + k;
      w[i * VEC + k] = e < d ? load_param(p.w, p.w_bf16, e) : 0.f;
      dw[i * VEC + k] = db[i * VEC + k] = 0.f;
    }
  const int64_t step = static_cast<int64_t>(gridDim.x) * R;
  int64_t row = static_cast<int64_t>(blockIdx.x) * R + g;
  Pack<T, VEC> x[NV], dy[NV], next_x[NV], next_dy[NV];
  load_row<T, VEC, NV>(x, p.x, row * p.s_x, tid, G, d, row < p.N);
  load_row<T, VEC, NV>(dy, p.dy, row * p.s_dy, tid, G, d, row < p.N);
  float mean = row < p.N ? p.mean[row] : 0.f, rstd = row < p.N ? p.rstd[row] : 0.f;
  int parity = 0;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * R; first < p.N; first += step, row += step, parity ^= 1) {
    const int64_t after = row + step;
    load_row<T, VEC, NV>(next_x, p.x, after * p.s_x, tid, G, d, after < p.N);
    load_row<T, VEC, NV>(next_dy, p.dy, after * p.s_dy, tid, G, d, after < p.N);
    const float next_mean = after < p.N ? p.mean[after] : 0.f, next_rstd = after < p.N ? p.rstd[after] : 0.f;
    float s[2] = {0.f, 0.f};
    if (row < p.N) {  // a group without a row adds nothing
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((tid + i * G) * VEC < d)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float xhat = (to_f32(x[i].e[k]) - mean) * rstd, t = to_f32(dy[i].e[k]), a = t * w[i * VEC + k];
            s[0] += a;
            s[1] = fmaf(a, xhat, s[1]);
            dw[i * VEC + k] = fmaf(t, xhat, dw[i * VEC + k]);
            db[i * VEC + k] += t;
          }
    }
    row_sums<2>(s, G, red[parity]);
    const float c1 = s[0] * inv_d, c2 = s[1] * inv_d;
    if (row < p.N) {
      T* o = static_cast<T*>(p.out) + row * p.s_out;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int e = (tid + i * G) * VEC;
        if (e < d) {
          Pack<T, VEC> y;
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float xhat = (to_f32(x[i].e[k]) - mean) * rstd, a = to_f32(dy[i].e[k]) * w[i * VEC + k];
            y.e[k] = from_f32<T>(rstd * (a - fmaf(xhat, c2, c1)));
          }
          *reinterpret_cast<Pack<T, VEC>*>(o + e) = y;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = next_x[i];
      dy[i] = next_dy[i];
    }
    mean = next_mean;
    rstd = next_rstd;
  }
  if (!p.part) return;
  float* part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * d;
  if (R == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const int e = (tid + i * G) * VEC + k;
        if (e < d) {
          part[e] = dw[i * VEC + k];
          part[d + e] = db[i * VEC + k];
        }
      }
    return;
  }
  const int width = G * NV * VEC;  // at least d
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const int e = (tid + i * G) * VEC + k;
      cols[g * width + e] = dw[i * VEC + k];
      cols[(R + g) * width + e] = db[i * VEC + k];
    }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * d; e += blockDim.x) {
    const float* c = cols + (e < d ? e : R * width + e - d);
    float sum = 0.f;
    for (int r = 0; r < R; ++r) sum += c[r * width];
    part[e] = sum;
  }
}

// Rows wider than kHeldWidth: a CTA a row, which is read again (from L2) for each sum.
template <typename T, int VEC>
__global__ void __launch_bounds__(kWideThreads) norm_wide_kernel(const NormParams p) {
  using P = Pack<T, VEC>;
  __shared__ float red[2][1][32];
  const float inv_d = 1.f / static_cast<float>(p.d);
  wait_for_previous();
  for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + row * p.s_x;
    T* o = static_cast<T*>(p.out) + row * p.s_out;
    float s[1] = {0.f};
    for (int e = threadIdx.x * VEC; e < p.d; e += kWideThreads * VEC) {
      const P v = *reinterpret_cast<const P*>(x + e);
#pragma unroll
      for (int k = 0; k < VEC; ++k) s[0] += to_f32(v.e[k]);
    }
    row_sums<1>(s, kWideThreads, red[0]);
    const float mean = s[0] * inv_d;
    s[0] = 0.f;
    for (int e = threadIdx.x * VEC; e < p.d; e += kWideThreads * VEC) {
      const P v = *reinterpret_cast<const P*>(x + e);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float c = to_f32(v.e[k]) - mean;
        s[0] = fmaf(c, c, s[0]);
      }
    }
    row_sums<1>(s, kWideThreads, red[1]);
    const float rstd = 1.f / sqrtf(s[0] * inv_d + p.eps);
    for (int e = threadIdx.x * VEC; e < p.d; e += kWideThreads * VEC) {
      P v = *reinterpret_cast<const P*>(x + e);
#pragma unroll
      for (int k = 0; k < VEC; ++k)
        v.e[k] = from_f32<T>(fmaf((to_f32(v.e[k]) - mean) * rstd, load_param(p.w, p.w_bf16, e + k),
                                  p.b ? load_param(p.b, p.w_bf16, e + k) : 0.f));
      *reinterpret_cast<P*>(o + e) = v;
    }
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kWideThreads) norm_grad_wide_kernel(const NormParams p) {
  using P = Pack<T, VEC>;
  __shared__ float red[2][2][32];
  const float inv_d = 1.f / static_cast<float>(p.d);
  wait_for_previous();
  int parity = 0;
  for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x, parity ^= 1) {
    const T* x = static_cast<const T*>(p.x) + row * p.s_x;
    const T* dy = static_cast<const T*>(p.dy) + row * p.s_dy;
    T* o = static_cast<T*>(p.out) + row * p.s_out;
    const float mean = p.mean[row], rstd = p.rstd[row];
    float s[2] = {0.f, 0.f};
    for (int e = threadIdx.x * VEC; e < p.d; e += kWideThreads * VEC) {
      const P u = *reinterpret_cast<const P*>(x + e), t = *reinterpret_cast<const P*>(dy + e);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float a = to_f32(t.e[k]) * load_param(p.w, p.w_bf16, e + k);
        s[0] += a;
        s[1] = fmaf(a, (to_f32(u.e[k]) - mean) * rstd, s[1]);
      }
    }
    row_sums<2>(s, kWideThreads, red[parity]);
    const float c1 = s[0] * inv_d, c2 = s[1] * inv_d;
    for (int e = threadIdx.x * VEC; e < p.d; e += kWideThreads * VEC) {
      const P u = *reinterpret_cast<const P*>(x + e), t = *reinterpret_cast<const P*>(dy + e);
      P y;
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float a = to_f32(t.e[k]) * load_param(p.w, p.w_bf16, e + k);
        y.e[k] = from_f32<T>(rstd * (a - fmaf((to_f32(u.e[k]) - mean) * rstd, c2, c1)));
      }
      *reinterpret_cast<P*>(o + e) = y;
    }
  }
}

// The sums of 256 columns (blockIdx.x) over the rows blockIdx.y, blockIdx.y + parts, ...
template <typename T>
__global__ void __launch_bounds__(kRowThreads) norm_columns_kernel(const NormParams p) {
  wait_for_previous();
  const int c = blockIdx.x * kRowThreads + threadIdx.x;
  if (c >= p.d) return;
  float dw = 0.f, db = 0.f;
#pragma unroll 4
  for (int64_t row = blockIdx.y; row < p.N; row += gridDim.y) {
    const float t = to_f32(static_cast<const T*>(p.dy)[row * p.s_dy + c]);
    dw = fmaf(t, (to_f32(static_cast<const T*>(p.x)[row * p.s_x + c]) - p.mean[row]) * p.rstd[row], dw);
    db += t;
  }
  float* part = p.part + static_cast<int64_t>(blockIdx.y) * 2 * p.d;
  part[c] = dw;
  part[p.d + c] = db;
}

// Adds the parts of 32 columns (blockIdx.x) of dw or db (blockIdx.y), in a fixed order.
constexpr int kReduceRows = 16;
__global__ void __launch_bounds__(32 * kReduceRows)
    norm_reduce_kernel(const float* part, int parts, int d, int bf16, void* dw, void* db) {
  __shared__ float sums[kReduceRows][33];
  void* out = blockIdx.y ? db : dw;
  if (!out) return;
  wait_for_previous();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;
  float s = 0.f;
  if (c < d)
#pragma unroll 4
    for (int i = ty; i < parts; i += kReduceRows) s += part[(static_cast<int64_t>(i) * 2 + blockIdx.y) * d + c];
  sums[ty][tx] = s;
  __syncthreads();
  if (ty || c >= d) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kReduceRows; ++i) s += sums[i][tx];
  if (bf16)
    static_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(s);
  else
    static_cast<float*>(out)[c] = s;
}

// Threads a row, rows a CTA and loads a thread: the fewest loads whose threads fit
// in a CTA; a row of few loads shares a CTA, and a warp, with others.
struct Shape {
  int G, R, nv;
};

Shape shape_of(int64_t loads, const int* nvs) {
  int nv = *nvs;
  while ((loads + nv - 1) / nv > kRowThreads) nv = *++nvs;
  const int64_t need = (loads + nv - 1) / nv;
  if (need > 32) return {static_cast<int>((need + 31) / 32 * 32), 1, nv};
  int G = 8;
  while (G < need) G *= 2;
  return {G, kRowThreads / G, nv};
}

bool by_vectors(const void* p, int64_t stride, int esz) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * esz % 16 == 0;
}

template <typename T, int VEC, int NV>
cudaError_t launch_shape(bool grad, const NormParams& p, const Shape& s, int ctas, cudaStream_t stream) {
  const size_t smem = grad && s.R > 1 ? static_cast<size_t>(2) * s.R * s.G * NV * VEC * 4 : 0;
  return launch_overlapped(grad ? norm_grad_kernel<T, VEC, NV> : norm_kernel<T, VEC, NV>, dim3(static_cast<unsigned>(ctas)),
                           s.G * s.R, smem, stream, 1, true, p);
}

template <typename T, int VEC>
cudaError_t launch_wide(bool grad, const NormParams& p, int max_ctas, int* parts, cudaStream_t stream) {
  const int64_t most = p.N < 304 ? p.N : 304;  // two CTAs of 1024 threads an SM
  cudaError_t e = launch_overlapped(grad ? norm_grad_wide_kernel<T, VEC> : norm_wide_kernel<T, VEC>,
                                    dim3(static_cast<unsigned>(most)), kWideThreads, 0, stream, 1, true, p);
  if (e != cudaSuccess || !p.part) return e;
  *parts = static_cast<int>(p.N < max_ctas ? p.N : max_ctas);
  return launch_overlapped(norm_columns_kernel<T>, dim3(static_cast<unsigned>((p.d + kRowThreads - 1) / kRowThreads), *parts),
                           kRowThreads, 0, stream, 1, true, p);
}

// *parts: the parts of dw and db that the launches write.
template <typename T>
int launch_typed(bool grad, NormParams p, int max_ctas, int* parts, cudaStream_t stream) {
  constexpr int kVec = 16 / static_cast<int>(sizeof(T));
  const bool vec = p.d % kVec == 0 && by_vectors(p.x, p.s_x, sizeof(T)) && by_vectors(p.out, p.s_out, sizeof(T)) &&
                   (!grad || by_vectors(p.dy, p.s_dy, sizeof(T)));
  cudaError_t e;
  if (p.d > kHeldWidth) {
    e = vec ? launch_wide<T, kVec>(grad, p, max_ctas, parts, stream) : launch_wide<T, 1>(grad, p, max_ctas, parts, stream);
  } else {
    static const int kVecLoads[] = {1, 2, 4, 8}, kLoads[] = {8, 32};
    constexpr int kMost = 32 / kVec;  // loads a thread of the widest row held
    const Shape s = vec ? shape_of(p.d / kVec, kVecLoads) : shape_of(p.d, kLoads);
    p.G = s.G;
    const int64_t want = (p.N + s.R - 1) / s.R;
    *parts = static_cast<int>(want < max_ctas ? want : max_ctas);
    if (!vec)
      e = s.nv == 8 ? launch_shape<T, 1, 8>(grad, p, s, *parts, stream) : launch_shape<T, 1, 32>(grad, p, s, *parts, stream);
    else if (s.nv == 1)
      e = launch_shape<T, kVec, 1>(grad, p, s, *parts, stream);
    else if (s.nv == 2)
      e = launch_shape<T, kVec, 2>(grad, p, s, *parts, stream);
    else
      e = s.nv == kMost ? launch_shape<T, kVec, kMost>(grad, p, s, *parts, stream) : launch_shape<T, kVec, 4>(grad, p, s, *parts, stream);
  }
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "layer norm launch: %s", cudaGetErrorString(e));
}

NormParams params_of(const NormArgs& a) {
  NormParams p = {};
  p.x = a.x;
  p.w = a.weight;
  p.mean = a.mean;
  p.rstd = a.rstd;
  p.N = a.N;
  p.s_x = a.s_x;
  p.d = static_cast<int>(a.d);
  p.w_bf16 = a.weight_bf16;
  return p;
}

}  // namespace

int launch_layer_norm(const NormArgs& a, cudaStream_t stream) {
  NormParams p = params_of(a);
  p.b = a.bias;
  p.out = a.out;
  p.s_out = a.s_out;
  p.eps = a.eps;
  int ctas;
  return a.is_bf16 ? launch_typed<__nv_bfloat16>(false, p, 152 * 8, &ctas, stream)
                   : launch_typed<float>(false, p, 152 * 8, &ctas, stream);
}

int launch_layer_norm_grad(const NormArgs& a, cudaStream_t stream) {
  NormParams p = params_of(a);
  p.dy = a.dout;
  p.s_dy = a.s_dout;
  p.out = a.dx;
  p.s_out = a.s_dx;
  p.part = a.dweight || a.dbias ? static_cast<float*>(a.workspace) : nullptr;
  int ctas = 0;
  if (a.N > 0) {
    const int most = norm_max_parts(a.d);
    const int st = a.is_bf16 ? launch_typed<__nv_bfloat16>(true, p, most, &ctas, stream) : launch_typed<float>(true, p, most, &ctas, stream);
    if (st != DLM_OK) return st;
  }
  if (!a.dweight && !a.dbias) return DLM_OK;
  const cudaError_t e =
      launch_overlapped(norm_reduce_kernel, dim3(static_cast<unsigned>((a.d + 31) / 32), 2), 32 * kReduceRows, 0, stream, 1,
                        true, static_cast<const float*>(a.workspace), ctas, p.d, a.weight_bf16, a.dweight, a.dbias);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "layer norm reduction launch: %s", cudaGetErrorString(e));
}

}  // namespace dlm
