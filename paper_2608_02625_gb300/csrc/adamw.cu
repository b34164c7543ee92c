// One AdamW step over many tensors, states in 32 bits or in 8.
//
//   g = grad c,  c = min(1, max_norm / (norm + 1e-6))   (1 without a norm)
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   p = p (1 - lr wd) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
//
// One pass: a warp takes 256 elements, eight a lane, loads everything that belongs to
// them, computes in fp32 and stores. HBM bounds it. 8-bit states are e4m3 codes of m and
// of sqrt(v) (whose range, 2^17 within a block with half a step of 2^-4, covers twice that in
// powers of two of v), in blocks of 256 elements with a scale of their own: the largest
// magnitude over 448. A block is a warp's 256 elements, so the old scale is one load and
// the new one a reduction over the warp. The step itself uses the new m and v before they are
// rounded to 8 bits. A sqrt(v) below the codes' range is held as the smallest code, not as 0:
// rounded to 0 it would leave m / eps for the next step. Products and sums of the states are
// rounded one by one (no fma), so what is rounded to 8 bits does not depend on how the
// compiler contracts it.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <cmath>
#include <cstdint>

#include "dlm_common.cuh"
#include "dlm_internal.h"

namespace dlm {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPerSm = 4;            // CTAs an SM (64 registers a thread)
constexpr int kBlock = kAdamwBlock;  // elements of a warp's turn, and of a scale
constexpr int kPer = kBlock / 32;    // elements a lane
constexpr float kTop = 448.f;        // the largest e4m3 value

enum Kind { kF32 = 0, kBF16 = 1, kMaster = 2 };  // of the weights; kMaster: fp32, and bf16 copies

struct Tensor {
  void* p;         // F32 or BF16 weights (kMaster: the copies)
  float* master;
  const void* g;
  void* m;         // F32, or codes
  void* v;
  float* ms;       // scales
  float* vs;
  int64_t n;
  int first;       // its first chunk
  int16_t kind;
  int8_t g_bf16, vectors;
};

template <int kTensors>
struct Table {
  Tensor t[kTensors];
  int count, chunks, chunk;  // tensors, chunks in all, elements a chunk (a multiple of 2048)
  float beta1, rest1, beta2, rest2, eps;
  double log_beta1, log_beta2, decay, max_norm;
  const float* lr;
  const int32_t* step;
  const float* norm;  // may be null
  int* err;
};

// What the step's scalars come to.
struct Step {
  float clip, keep, alpha, root;  // c, 1 - lr wd, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

template <typename Tab>
__device__ Step step_of(const Tab& tab) {
  Step s;
  int t = *tab.step;
  if (t < 1) {
    t = 1;
    if (blockIdx.x == 0) set_device_error(tab.err, DLM_DEVERR_LENGTH);
  }
  const float lr = *tab.lr;
  // 1 - beta^t = -expm1(t ln beta): t ln beta in fp64, the rest is good to some 1e-7 in fp32.
  const float one1 = -expm1f(static_cast<float>(t * tab.log_beta1)), one2 = -expm1f(static_cast<float>(t * tab.log_beta2));
  s.keep = static_cast<float>(1.0 - static_cast<double>(lr) * tab.decay);
  s.alpha = lr / one1;
  s.root = 1.f / sqrtf(one2);
  s.clip = 1.f;
  if (tab.norm) {
    const double c = tab.max_norm / (static_cast<double>(*tab.norm) + 1e-6);
    s.clip = c >= 1.0 ? 1.f : static_cast<float>(c);  // a NaN stays one
  }
  return s;
}

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

// ---------------------------------------------------------------- eight elements of a lane
//
// kVec: elements 8 lane .. 8 lane + 7 of the block, moved 8 to 32 bytes at a time; else
// elements lane, lane + 32, ..., one by one, n of the block's 256 present.

template <bool kVec>
__device__ __forceinline__ int place(int lane, int k) {
  return kVec ? kPer * lane + k : lane + 32 * k;
}

template <bool kVec>
__device__ __forceinline__ void load(const float* src, int lane, int n, float (&x)[kPer]) {
  if constexpr (kVec) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "l"(src + kPer * lane)
                 : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) x[k] = lane + 32 * k < n ? src[lane + 32 * k] : 0.f;
  }
}

template <bool kVec>
__device__ __forceinline__ void load(const __nv_bfloat16* src, int lane, int n, float (&x)[kPer]) {
  if constexpr (kVec) {
    const uint4 u = *reinterpret_cast<const uint4*>(src + kPer * lane);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(w[k] << 16);
      x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) x[k] = lane + 32 * k < n ? __bfloat162float(src[lane + 32 * k]) : 0.f;
  }
}

__device__ __forceinline__ float2 values_of(uint16_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3);
  return __half22float2(__half2(h));
}

// Codes as the values they stand for before their scale.
template <bool kVec>
__device__ __forceinline__ void load(const uint8_t* src, int lane, int n, float (&x)[kPer]) {
  uint32_t w[2] = {0, 0};
  if (kVec) {
    const uint2 u = *reinterpret_cast<const uint2*>(src + kPer * lane);
    w[0] = u.x;
    w[1] = u.y;
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) w[k >> 2] |= static_cast<uint32_t>(src[lane + 32 * k]) << (8 * (k & 3));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = values_of(static_cast<uint16_t>(w[k >> 1] >> (16 * (k & 1))));
    x[2 * k] = f.x;
    x[2 * k + 1] = f.y;
  }
}

template <bool kVec>
__device__ __forceinline__ void store(float* dst, int lane, int n, const float (&x)[kPer]) {
  if constexpr (kVec) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + kPer * lane), "f"(x[0]), "f"(x[1]),
                 "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) dst[lane + 32 * k] = x[k];
  }
}

template <bool kVec>
__device__ __forceinline__ void store(__nv_bfloat16* dst, int lane, int n, const float (&x)[kPer]) {
  if constexpr (kVec) {
    *reinterpret_cast<uint4*>(dst + kPer * lane) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                              pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) dst[lane + 32 * k] = __float2bfloat16_rn(x[k]);
  }
}

// The largest magnitude over the warp (a NaN's pattern is above an infinity's).
__device__ __forceinline__ float warp_top(const float (&x)[kPer]) {
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) top = max(top, __float_as_uint(x[k]) & 0x7FFFFFFFu);
  return __uint_as_float(__reduce_max_sync(0xffffffffu, top));
}

// Codes of x under the scale 1 / inv. kNotZero: x >= 0, and what is above 0 has a code above 0.
template <bool kVec, bool kNotZero>
__device__ __forceinline__ void store_codes(uint8_t* dst, int lane, int n, const float (&x)[kPer], float inv) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = make_float2(__fmul_rn(x[2 * k], inv), __fmul_rn(x[2 * k + 1], inv));
    uint32_t two = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
    if (kNotZero) {  // (a product above 0 is: 448 times the smallest scale is far above fp32's least)
      if (f.x > 0.f && (two & 0xFFu) == 0) two |= 1u;
      if (f.y > 0.f && (two & 0xFF00u) == 0) two |= 0x100u;
    }
    w[k >> 1] |= two << (16 * (k & 1));
  }
  if constexpr (kVec) {
    *reinterpret_cast<uint2*>(dst + kPer * lane) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) dst[lane + 32 * k] = static_cast<uint8_t>(w[k >> 2] >> (8 * (k & 3)));
  }
}

// One block of n elements (256 where kVec) at element `at` of a tensor.
template <bool kVec, bool kEight, int kKind, typename G>
__device__ __forceinline__ void block_step(const Tensor& t, int64_t at, int n, int lane, const Step& s, float beta1, float rest1,
                                           float beta2, float rest2, float eps) {
  float p[kPer], g[kPer], m[kPer], v[kPer];
  const int64_t b = at / kBlock;
  float ms = 0.f, vs = 0.f;
  load<kVec>(static_cast<const G*>(t.g) + at, lane, n, g);
  if (kEight) {
    ms = t.ms[b];
    vs = t.vs[b];
    load<kVec>(static_cast<const uint8_t*>(t.m) + at, lane, n, m);
    load<kVec>(static_cast<const uint8_t*>(t.v) + at, lane, n, v);
  } else {
    load<kVec>(static_cast<const float*>(t.m) + at, lane, n, m);
    load<kVec>(static_cast<const float*>(t.v) + at, lane, n, v);
  }
  if (kKind == kMaster)
    load<kVec>(t.master + at, lane, n, p);
  else if (kKind == kF32)
    load<kVec>(static_cast<const float*>(t.p) + at, lane, n, p);
  else
    load<kVec>(static_cast<const __nv_bfloat16*>(t.p) + at, lane, n, p);
  float r[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const float x = __fmul_rn(g[k], s.clip);
    if (kEight) {
      m[k] = __fmul_rn(m[k], ms);
      v[k] = __fmul_rn(v[k], vs);
      v[k] = __fmul_rn(v[k], v[k]);
    }
    m[k] = __fadd_rn(__fmul_rn(m[k], beta1), __fmul_rn(x, rest1));
    v[k] = __fadd_rn(__fmul_rn(v[k], beta2), __fmul_rn(__fmul_rn(x, x), rest2));
    r[k] = __fsqrt_rn(v[k]);
    p[k] = fmaf(p[k], s.keep, -s.alpha * __fdividef(m[k], fmaf(r[k], s.root, eps)));
  }
  if (kKind == kMaster) store<kVec>(t.master + at, lane, n, p);
  if (kKind == kF32)
    store<kVec>(static_cast<float*>(t.p) + at, lane, n, p);
  else
    store<kVec>(static_cast<__nv_bfloat16*>(t.p) + at, lane, n, p);
  if constexpr (!kEight) {
    store<kVec>(static_cast<float*>(t.m) + at, lane, n, m);
    store<kVec>(static_cast<float*>(t.v) + at, lane, n, v);
    return;
  }
  // Both scales in one go: even lanes m's, odd lanes sqrt(v)'s. Below fp32's normal range there
  // is none: everything is held as 0.
  const float top_m = warp_top(m), top_r = warp_top(r);
  float scale = __fmul_rn(lane & 1 ? top_r : top_m, 1.f / kTop);
  if (scale < 0x1p-126f) scale = 0.f;
  const float inv = scale == 0.f ? 0.f : __frcp_rn(scale);
  if (lane == 0) t.ms[b] = scale;
  if (lane == 1) t.vs[b] = scale;
  store_codes<kVec, false>(static_cast<uint8_t*>(t.m) + at, lane, n, m, __shfl_sync(0xffffffffu, inv, 0));
  store_codes<kVec, true>(static_cast<uint8_t*>(t.v) + at, lane, n, r, __shfl_sync(0xffffffffu, inv, 1));
}

template <bool kEight, int kKind, typename G>
__device__ void chunk_step(const Tensor& t, int64_t at, int64_t end, const Step& s, float beta1, float rest1, float beta2, float rest2,
                           float eps) {
  const int lane = threadIdx.x & 31;
  for (int64_t i = at + (threadIdx.x >> 5) * kBlock; i < end; i += kWarps * kBlock) {
    const int n = end - i < kBlock ? static_cast<int>(end - i) : kBlock;
    if (t.vectors && n == kBlock)
      block_step<true, kEight, kKind, G>(t, i, n, lane, s, beta1, rest1, beta2, rest2, eps);
    else
      block_step<false, kEight, kKind, G>(t, i, n, lane, s, beta1, rest1, beta2, rest2, eps);
  }
}

template <int kTensors, bool kEight>
__global__ void __launch_bounds__(kThreads, kPerSm) adamw_kernel(const __grid_constant__ Table<kTensors> tab) {
  __shared__ Step shared;
  wait_for_previous();
  if (threadIdx.x == 0) shared = step_of(tab);
  __syncthreads();
  const Step s = shared;
  for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
    const Tensor& t = find(tab, c);
    const int64_t at = static_cast<int64_t>(c - t.first) * tab.chunk;
    const int64_t end = t.n - at < tab.chunk ? t.n : at + tab.chunk;
#define DLM_STEP(kind, type) chunk_step<kEight, kind, type>(t, at, end, s, tab.beta1, tab.rest1, tab.beta2, tab.rest2, tab.eps)
    if (t.g_bf16) {
      if (t.kind == kF32)
        DLM_STEP(kF32, __nv_bfloat16);
      else if (t.kind == kBF16)
        DLM_STEP(kBF16, __nv_bfloat16);
      else
        DLM_STEP(kMaster, __nv_bfloat16);
    } else {
      if (t.kind == kF32)
        DLM_STEP(kF32, float);
      else if (t.kind == kBF16)
        DLM_STEP(kBF16, float);
      else
        DLM_STEP(kMaster, float);
    }
#undef DLM_STEP
  }
}

// ---------------------------------------------------------------- host side

bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }

template <int kTensors>
void fill(const AdamwArgs& a, int first, Table<kTensors>* tab) {
  tab->count = a.count - first < kTensors ? a.count - first : kTensors;
  // Chunks of 8192 elements, larger ones only where their number would pass an int.
  int64_t chunk = 4 * kThreads * kPer, chunks = 0;
  for (;; chunk *= 2) {
    chunks = 0;
    for (int i = 0; i < tab->count; ++i) chunks += (a.tensors[first + i].n + chunk - 1) / chunk;
    if (chunks <= (1 << 30) || chunk >= (1 << 29)) break;
  }
  // Few elements: a warp's turn each, over as many SMs as there are.
  if (chunks < 152) {
    chunk = kThreads * kPer;
    chunks = 0;
    for (int i = 0; i < tab->count; ++i) chunks += (a.tensors[first + i].n + chunk - 1) / chunk;
  }
  tab->chunk = static_cast<int>(chunk);
  tab->chunks = static_cast<int>(chunks);
  int at = 0;
  for (int i = 0; i < tab->count; ++i) {
    const AdamwTensor& t = a.tensors[first + i];
    const int kind = t.master ? kMaster : t.p_bf16 ? kBF16 : kF32, state = a.eight ? 8 : 32;
    const bool vectors = aligned(t.p, kind == kF32 ? 32 : 16) && aligned(t.master, 32) && aligned(t.g, t.g_bf16 ? 16 : 32) &&
                         aligned(t.m, state) && aligned(t.v, state);
    tab->t[i] = {t.p, t.master, t.g, t.m, t.v, t.ms, t.vs, t.n, at, static_cast<int16_t>(kind), static_cast<int8_t>(t.g_bf16),
                 static_cast<int8_t>(vectors)};
    at += static_cast<int>((t.n + chunk - 1) / chunk);
  }
}

template <int kTensors, bool kEight>
int launch_tables(const AdamwArgs& a, cudaStream_t stream) {
  const auto kernel = adamw_kernel<kTensors, kEight>;
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  Table<kTensors> tab;
  tab.beta1 = static_cast<float>(a.beta1);
  tab.rest1 = static_cast<float>(1.0 - a.beta1);
  tab.beta2 = static_cast<float>(a.beta2);
  tab.rest2 = static_cast<float>(1.0 - a.beta2);
  tab.eps = static_cast<float>(a.eps);
  tab.log_beta1 = std::log(a.beta1);
  tab.log_beta2 = std::log(a.beta2);
  tab.decay = a.weight_decay;
  tab.max_norm = a.max_norm;
  tab.lr = a.lr;
  tab.step = a.step;
  tab.norm = a.norm;
  tab.err = device_error_word();
  for (int first = 0; first < a.count; first += kTensors) {
    fill(a, first, &tab);
    const int64_t most = static_cast<int64_t>(sms) * kPerSm;
    const int ctas = static_cast<int>(tab.chunks < most ? tab.chunks : most);
    const cudaError_t e = launch_overlapped(kernel, dim3(static_cast<unsigned>(ctas)), kThreads, 0, stream, 1, true, tab);
    if (e != cudaSuccess) return fail(DLM_ERR_CUDA, "adamw launch: %s", cudaGetErrorString(e));
  }
  return DLM_OK;
}

template <int kTensors>
int launch_either(const AdamwArgs& a, cudaStream_t stream) {
  return a.eight ? launch_tables<kTensors, true>(a, stream) : launch_tables<kTensors, false>(a, stream);
}

}  // namespace

int launch_adamw(const AdamwArgs& a, cudaStream_t stream) {
  if (a.count <= 24) return launch_either<24>(a, stream);
  return launch_either<kAdamwTable>(a, stream);
}

}  // namespace dlm
