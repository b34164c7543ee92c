// One AdamW step over many tensors, states in 32 bits or in 8.
//
//   g = grad c,  c = min(1, max_norm / (norm + 1e-6))   (1 without a norm)
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   p = p (1 - lr wd) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
//
// One pass: a warp takes 256 elements, eight a lane, loads everything that belongs to
// them, computes in fp32 (two elements an instruction) and stores. HBM bounds it: 213 M weights with
// bf16 copies, bf16 gradients and 32-bit states 918-929 us (6.5 TB/s, 95 % of a copy), bf16 weights with
// 8-bit states 346 us (6.21 TB/s, 92 %; 341 with sums that are fused with a product, 333 with a square root, too,
// that flushes what is below the normal range and so leaves such a v's m to be divided by eps alone). 8-bit states are e4m3 codes of m and of sqrt(v) (whose range,
// 2^17 within a block with half a step of 2^-4 over most of it, is twice that in powers of two of v), in
// blocks of 256 elements with a scale of their own: the largest magnitude over 448. A block is a
// warp's 256 elements, so a scale is a reduction over the warp. The step itself uses the new m and v
// before they are rounded to 8 bits. A sqrt(v) below the codes' range is held as the smallest code, not
// as 0: rounded to 0 it would leave m / eps for the next step. Products and sums of the states are
// rounded one by one (no fma), so what is rounded to 8 bits does not depend on how the compiler
// contracts it.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "dlm_common.cuh"
#include "dlm_internal.h"

namespace dlm {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPerSm = 3;            // CTAs an SM: 80 registers a thread, two more of which 8-bit states spill (four of 64: 6 % slower)
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
  int64_t first;   // its first chunk
  int kind;
  int16_t g_bf16, vectors;
};

// The coefficients of m and v, and 1.
struct Betas {
  float beta1, rest1, beta2, rest2, one;
};

template <int kTensors>
struct Table {
  Tensor t[kTensors];
  int64_t chunks;
  int count, chunk;  // tensors, elements a chunk (a multiple of 2048)
  Betas betas;
  double log_beta1, log_beta2, decay, max_norm;
  float eps;
  const float* lr;
  const int32_t* step;
  const float* norm;  // may be null
  int* err;
};

// What the step's scalars come to.
struct Step {
  float clip, keep, alpha, root, eps;  // c, 1 - lr wd, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

template <bool kEight, typename Tab>
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
  // With 8-bit states no m is divided by less than what its v may have lost: g^2, its product, the v held and
  // theirs are rounded by up to 2^-150 each below the normal range, which is a root of up to 2^-74. So a v
  // that is 0 for that moves its weight by no more than the v itself would, and 0 / 0 is 0.
  s.eps = kEight ? fmaxf(tab.eps, 0x1p-74f * s.root) : tab.eps;
  s.clip = 1.f;
  if (tab.norm) {
    const double c = tab.max_norm / (static_cast<double>(*tab.norm) + 1e-6);
    s.clip = c >= 1.0 ? 1.f : static_cast<float>(c);  // a NaN stays one
  }
  return s;
}

template <typename Tab>
__device__ __forceinline__ const Tensor& find(const Tab& tab, int64_t chunk) {
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
// elements lane, lane + 32, ..., one by one, n of the block's 256 present. What is loaded stays as
// it lies in memory until it is computed with, so that a block can be on its way while the one
// before it is computed.

template <typename T>
struct Raw {
  uint32_t w[2 * sizeof(T)];  // eight of T
};

template <bool kVec, typename T>
__device__ __forceinline__ void load(const T* src, int lane, int n, Raw<T>* to) {
  if constexpr (kVec && sizeof(T) == 4) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(to->w[0]), "=r"(to->w[1]), "=r"(to->w[2]), "=r"(to->w[3]), "=r"(to->w[4]), "=r"(to->w[5]), "=r"(to->w[6]),
                   "=r"(to->w[7])
                 : "l"(src + kPer * lane)
                 : "memory");
  } else if constexpr (kVec && sizeof(T) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(src + kPer * lane);
    to->w[0] = u.x;
    to->w[1] = u.y;
    to->w[2] = u.z;
    to->w[3] = u.w;
  } else if constexpr (kVec) {
    const uint2 u = *reinterpret_cast<const uint2*>(src + kPer * lane);
    to->w[0] = u.x;
    to->w[1] = u.y;
  } else {
    constexpr int kIn = 4 / sizeof(T);  // of T in a word
#pragma unroll
    for (int k = 0; k < static_cast<int>(2 * sizeof(T)); ++k) to->w[k] = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) {
        uint32_t x;
        if constexpr (sizeof(T) == 4)
          x = __float_as_uint(src[lane + 32 * k]);
        else if constexpr (sizeof(T) == 2)
          x = reinterpret_cast<const unsigned short*>(src)[lane + 32 * k];
        else
          x = src[lane + 32 * k];
        to->w[k / kIn] |= x << (8 * sizeof(T) * (k % kIn));
      }
  }
}

// Elements 2 k and 2 k + 1.
__device__ __forceinline__ float2 pair_of(const Raw<float>& r, int k) {
  return make_float2(__uint_as_float(r.w[2 * k]), __uint_as_float(r.w[2 * k + 1]));
}
__device__ __forceinline__ float2 pair_of(const Raw<__nv_bfloat16>& r, int k) {
  return make_float2(__uint_as_float(r.w[k] << 16), __uint_as_float(r.w[k] & 0xFFFF0000u));
}
__device__ __forceinline__ float2 pair_of(const Raw<uint8_t>& r, int k) {  // codes: values before their scale
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(r.w[k >> 1] >> (16 * (k & 1))), __NV_E4M3);
  return __half22float2(__half2(h));
}

template <bool kVec>
__device__ __forceinline__ void store(float* dst, int lane, int n, const float2 (&x)[kPer / 2]) {
  if constexpr (kVec) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + kPer * lane), "f"(x[0].x), "f"(x[0].y),
                 "f"(x[1].x), "f"(x[1].y), "f"(x[2].x), "f"(x[2].y), "f"(x[3].x), "f"(x[3].y)
                 : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) dst[lane + 32 * k] = k & 1 ? x[k >> 1].y : x[k >> 1].x;
  }
}

template <bool kVec>
__device__ __forceinline__ void store(__nv_bfloat16* dst, int lane, int n, const float2 (&x)[kPer / 2]) {
  if constexpr (kVec) {
    *reinterpret_cast<uint4*>(dst + kPer * lane) =
        make_uint4(pack_bf16x2(x[0].x, x[0].y), pack_bf16x2(x[1].x, x[1].y), pack_bf16x2(x[2].x, x[2].y), pack_bf16x2(x[3].x, x[3].y));
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) dst[lane + 32 * k] = __float2bfloat16_rn(k & 1 ? x[k >> 1].y : x[k >> 1].x);
  }
}

// The largest of a and two magnitudes; a NaN stays one.
__device__ __forceinline__ float top_of(float a, float2 x) {
  float c;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(c) : "f"(a), "f"(fabsf(x.x)), "f"(fabsf(x.y)));
  return c;
}

// The largest magnitude over the warp (the pattern of a NaN is above an infinity's).
__device__ __forceinline__ float warp_top(const float2 (&x)[kPer / 2]) {
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < kPer / 2; ++k) top = top_of(top, x[k]);
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7FFFFFFFu));
}

// What is above 0 rounds to a code above 0: at least to the smallest code's value, 2^-9 (between half
// of that and that it rounds there anyway). x: before its scale; 2^100 of any x above 0 (a square root
// of fp32 numbers, 2^-75 or more) is above 448.
__device__ __forceinline__ float not_zero(float y, float x) { return fminf(fmaxf(y, 0x1p-9f), x * 0x1p100f); }

// Codes of x under the scale 1 / inv. kNotZero: x >= 0, and what is above 0 has a code above 0.
template <bool kVec, bool kNotZero>
__device__ __forceinline__ void store_codes(uint8_t* dst, int lane, int n, const float2 (&x)[kPer / 2], float inv) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < kPer / 2; ++k) {
    float2 f = fmul2(x[k], make_float2(inv, inv));
    if (kNotZero) f = make_float2(not_zero(f.x, x[k].x), not_zero(f.y, x[k].y));
    w[k >> 1] |= static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3)) << (16 * (k & 1));
  }
  if constexpr (kVec) {
    *reinterpret_cast<uint2*>(dst + kPer * lane) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (lane + 32 * k < n) dst[lane + 32 * k] = static_cast<uint8_t>(w[k >> 2] >> (8 * (k & 3)));
  }
}

// sqrt(x), off by 2^-23 relative at most (quotients by 2^-22), below fp32's normal range too: a v flushed to
// 0 there leaves m to be divided by eps alone.
__device__ __forceinline__ float sqrt_approx(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool kEight, int kKind, typename G>
struct Block {
  using State = typename std::conditional<kEight, uint8_t, float>::type;
  using Weight = typename std::conditional<kKind == kBF16, __nv_bfloat16, float>::type;  // what is read of them
  Raw<G> g;
  Raw<State> m, v;
  Raw<Weight> p;

  // Block at element `at` of a tensor, n elements of it (256 where kVec).
  template <bool kVec>
  __device__ __forceinline__ void fetch(const Tensor& t, int64_t at, int n, int lane) {
    load<kVec>(static_cast<const G*>(t.g) + at, lane, n, &g);
    load<kVec>(static_cast<const State*>(t.m) + at, lane, n, &m);
    load<kVec>(static_cast<const State*>(t.v) + at, lane, n, &v);
    load<kVec>(kKind == kMaster ? reinterpret_cast<const Weight*>(t.master) + at : static_cast<const Weight*>(t.p) + at, lane, n, &p);
  }

  // ms, vs: the states' scales, and the new ones (8-bit states).
  template <bool kVec>
  __device__ __forceinline__ void step(const Tensor& t, int64_t at, int n, int lane, const Step& s, const Betas& b, float* ms,
                                       float* vs) const {
    const auto both = [](float x) { return make_float2(x, x); };
    // A sum of products that stays one: add.rn.f32x2 is fused with a product before it all the same (30 % of
    // the states were then off by a last place from what the order of the formula gives), an fma by a 1 that
    // the compiler does not know is not.
    const auto sum = [&](float2 p, float2 q) { return ffma2(p, both(b.one), q); };
    float2 pn[kPer / 2], mn[kPer / 2], vn[kPer / 2], rn[kPer / 2];
#pragma unroll
    for (int k = 0; k < kPer / 2; ++k) {
      const float2 x = fmul2(pair_of(g, k), both(s.clip));
      float2 m0 = pair_of(m, k), v0 = pair_of(v, k);
      if (kEight) {
        m0 = fmul2(m0, both(*ms));
        v0 = fmul2(v0, both(*vs));
        v0 = fmul2(v0, v0);
      }
      mn[k] = sum(fmul2(m0, both(b.beta1)), fmul2(x, both(b.rest1)));
      vn[k] = sum(fmul2(v0, both(b.beta2)), fmul2(fmul2(x, x), both(b.rest2)));
      rn[k] = make_float2(sqrt_approx(vn[k].x), sqrt_approx(vn[k].y));
      const float2 d = ffma2(rn[k], both(s.root), both(s.eps));
      float2 change;
      if constexpr (kEight) {
        // The reciprocal serves the square root too, for a step of Newton's: off by some half a last place then
        // where eps is far below the corrected root, and, as the step is scaled by root r / (root r + eps),
        // by the approximation's own last place where eps is far above it.
        const float2 y = make_float2(rcp_approx(d.x), rcp_approx(d.y));
        change = fmul2(mn[k], y);
        rn[k] = ffma2(ffma2(fmul2(rn[k], both(-1.f)), rn[k], vn[k]), fmul2(y, both(0.5f * s.root)), rn[k]);
      } else {
        change = make_float2(__fdividef(mn[k].x, d.x), __fdividef(mn[k].y, d.y));
      }
      pn[k] = ffma2(pair_of(p, k), both(s.keep), fmul2(change, both(-s.alpha)));
    }
    if (kKind == kMaster) store<kVec>(t.master + at, lane, n, pn);
    if (kKind == kF32)
      store<kVec>(static_cast<float*>(t.p) + at, lane, n, pn);
    else
      store<kVec>(static_cast<__nv_bfloat16*>(t.p) + at, lane, n, pn);
    if constexpr (!kEight) {
      store<kVec>(static_cast<float*>(t.m) + at, lane, n, mn);
      store<kVec>(static_cast<float*>(t.v) + at, lane, n, vn);
    } else {
      // Both scales in one go: even lanes m's, odd lanes sqrt(v)'s. Below fp32's normal range there
      // is none: everything is held as 0.
      const float top_m = warp_top(mn), top_r = warp_top(rn);
      float scale = __fmul_rn(lane & 1 ? top_r : top_m, 1.f / kTop);
      if (scale < 0x1p-126f) scale = 0.f;
      const float inv = scale == 0.f ? 0.f : __frcp_rn(scale);
      *ms = __shfl_sync(0xffffffffu, scale, 0);
      *vs = __shfl_sync(0xffffffffu, scale, 1);
      store_codes<kVec, false>(static_cast<uint8_t*>(t.m) + at, lane, n, mn, __shfl_sync(0xffffffffu, inv, 0));
      store_codes<kVec, true>(static_cast<uint8_t*>(t.v) + at, lane, n, rn, __shfl_sync(0xffffffffu, inv, 1));
    }
  }
};

// A warp's share of a chunk, blocks that follow each other, with 8-bit states. Their scales are
// read and written as one piece, lane k those of m of block k, lane 16 + k those of v: with
// accesses of four bytes for each block, whose sectors eight warps share, 200 M bf16 weights took
// 405 us instead of 300. Two whole blocks at a time are fetched before the first is computed.
template <int kKind, typename G>
__device__ void share_step8(const Tensor& t, int64_t at, int64_t end, const Step& s, const Betas& b) {
  using B = Block<true, kKind, G>;
  const int lane = threadIdx.x & 31;
  const int64_t first = at / kBlock;
  const int blocks = static_cast<int>((end - at + kBlock - 1) / kBlock), mine = lane & 15;  // at most 16
  float* scales = (lane < 16 ? t.ms : t.vs) + first + mine;
  float scale = mine < blocks ? *scales : 0.f, fresh = 0.f;
  const auto step = [&](const B& block, auto vec, int k, int n) {
    float ms = __shfl_sync(0xffffffffu, scale, k), vs = __shfl_sync(0xffffffffu, scale, 16 + k);
    block.template step<decltype(vec)::value>(t, at + k * kBlock, n, lane, s, b, &ms, &vs);
    if (mine == k) fresh = lane < 16 ? ms : vs;
  };
  int k = 0;
  if (t.vectors) {
    const int whole = static_cast<int>((end - at) / kBlock);
    for (; k + 2 <= whole; k += 2) {
      B one, two;
      one.template fetch<true>(t, at + k * kBlock, kBlock, lane);
      two.template fetch<true>(t, at + (k + 1) * kBlock, kBlock, lane);
      step(one, std::true_type{}, k, kBlock);
      step(two, std::true_type{}, k + 1, kBlock);
    }
    for (; k < whole; ++k) {
      B one;
      one.template fetch<true>(t, at + k * kBlock, kBlock, lane);
      step(one, std::true_type{}, k, kBlock);
    }
  }
  for (; k < blocks; ++k) {
    const int64_t i = at + k * kBlock;
    const int n = end - i < kBlock ? static_cast<int>(end - i) : kBlock;
    B one;
    one.template fetch<false>(t, i, n, lane);
    step(one, std::false_type{}, k, n);
  }
  if (mine < blocks) *scales = fresh;
}

// A warp's blocks of a chunk, every eighth, with 32-bit states.
template <int kKind, typename G>
__device__ void chunk_step32(const Tensor& t, int64_t at, int64_t end, const Step& s, const Betas& b) {
  using B = Block<false, kKind, G>;
  constexpr int64_t kStride = kWarps * kBlock;
  const int lane = threadIdx.x & 31;
  int64_t i = at + (threadIdx.x >> 5) * kBlock;
  for (; t.vectors && i + kBlock <= end; i += kStride) {
    B one;
    one.template fetch<true>(t, i, kBlock, lane);
    one.template step<true>(t, i, kBlock, lane, s, b, nullptr, nullptr);
  }
  for (; i < end; i += kStride) {
    const int n = end - i < kBlock ? static_cast<int>(end - i) : kBlock;
    B one;
    one.template fetch<false>(t, i, n, lane);
    one.template step<false>(t, i, n, lane, s, b, nullptr, nullptr);
  }
}

template <bool kEight, int kKind, typename G>
__device__ void chunk_step(const Tensor& t, int64_t at, int64_t end, int chunk, const Step& s, const Betas& b) {
  if constexpr (kEight) {
    const int share = chunk / kWarps;
    const int64_t mine = at + (threadIdx.x >> 5) * share;
    if (mine < end) share_step8<kKind, G>(t, mine, mine + share < end ? mine + share : end, s, b);
  } else {
    chunk_step32<kKind, G>(t, at, end, s, b);
  }
}

template <int kTensors, bool kEight>
__global__ void __launch_bounds__(kThreads, kPerSm) adamw_kernel(const __grid_constant__ Table<kTensors> tab) {
  __shared__ Step shared;
  wait_for_previous();
  if (threadIdx.x == 0) shared = step_of<kEight>(tab);
  __syncthreads();
  const Step s = shared;
  for (int64_t c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
    const Tensor& t = find(tab, c);
    const int64_t at = (c - t.first) * tab.chunk;
    const int64_t end = t.n - at < tab.chunk ? t.n : at + tab.chunk;
#define DLM_STEP(kind, type) chunk_step<kEight, kind, type>(t, at, end, tab.chunk, s, tab.betas)
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
  // 16384 elements with 8-bit states, eight blocks a warp, whose scales are a sector of 32 bytes, and
  // 8192 with 32-bit ones; fewer where those leave places empty, down to a block a warp.
  const auto chunks_of = [&](int64_t chunk) {
    int64_t chunks = 0;
    for (int i = 0; i < tab->count; ++i) chunks += (a.tensors[first + i].n + chunk - 1) / chunk;
    return chunks;
  };
  constexpr int64_t kLeast = kWarps * kBlock;
  int64_t chunk = (a.eight ? 8 : 4) * kLeast, chunks = chunks_of(chunk);
  while (chunks < kPerSm * 152 && chunk > kLeast) chunks = chunks_of(chunk /= 2);
  tab->chunk = static_cast<int>(chunk);
  tab->chunks = chunks;
  int64_t at = 0;
  for (int i = 0; i < tab->count; ++i) {
    const AdamwTensor& t = a.tensors[first + i];
    const int kind = t.master ? kMaster : t.p_bf16 ? kBF16 : kF32, state = a.eight ? 8 : 32;
    const bool vectors = aligned(t.p, kind == kF32 ? 32 : 16) && aligned(t.master, 32) && aligned(t.g, t.g_bf16 ? 16 : 32) &&
                         aligned(t.m, state) && aligned(t.v, state);
    tab->t[i] = {t.p, t.master, t.g, t.m, t.v, t.ms, t.vs, t.n, at, kind, static_cast<int16_t>(t.g_bf16),
                 static_cast<int16_t>(vectors)};
    at += (t.n + chunk - 1) / chunk;
  }
}

template <int kTensors, bool kEight>
int launch_tables(const AdamwArgs& a, cudaStream_t stream) {
  const auto kernel = adamw_kernel<kTensors, kEight>;
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  Table<kTensors> tab;
  tab.betas = {static_cast<float>(a.beta1), static_cast<float>(1.0 - a.beta1), static_cast<float>(a.beta2),
               static_cast<float>(1.0 - a.beta2), 1.f};
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
