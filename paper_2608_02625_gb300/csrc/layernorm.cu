// Layer norm in front of the output projection, and its gradients.
//
//   mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps)
//   out  = xhat w + b              with xhat = (x - mean) rstd
//   dx   = rstd (a - (sum a + xhat sum a xhat) / d)      with a = dout w
//   dw   = sum over rows of dout xhat,   db = sum over rows of dout
//
// One pass over the rows: a row lives in the registers of a group of threads (a part
// of a warp, a warp, or several), which takes its two sums over the centred values
// (not from sums of x and x^2, which cancel where the mean is large). The groups of a
// persistent grid walk the rows, the rows to come on their way to shared memory, the
// weights there in fp32. In the gradient each thread also keeps the sums of its columns
// over the rows of its group; the CTAs' sums go to the caller's workspace and a second
// launch adds them in a fixed order, so the results do not depend on scheduling. All
// sums are fp32. Rows too wide for that are read once for each sum, their columns' sums
// by a launch of their own.
//
// What bounds it is HBM, then the issue slots: what a row costs whatever a thread holds
// (two sums over the group, the root and its reciprocal, the loop) was most of the
// instructions with 8 elements a thread, so a thread holds 32. 16384 x 2048 bf16, among
// other calls: 25.1 us, 5.3 TB/s (8 elements, a CTA a row: 41.8; 64 elements, a warp a
// row, too few warps: 37), the gradients 41.4 us, 4.9 TB/s (98 before; 55 % of the issue
// slots busy at 16 warps an SM, whose registers hold the columns' sums).
#include <cuda_bf16.h>

#include <cstdint>

#include "dlm_common.cuh"
#include "dlm_internal.h"

namespace dlm {
namespace {

constexpr int kRowThreads = 256;    // a CTA of the kernels that hold rows in registers
constexpr int kWideThreads = 1024;  // a CTA of those that read a row again
constexpr int kHeldWidth = 8192;    // widest row held: 32 elements a thread

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

__device__ __forceinline__ void group_barrier(int G) {
  if (G <= 32)
    __syncwarp();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(1 + static_cast<int>(threadIdx.x) / G), "r"(G) : "memory");
}

// The sums of v over the G threads of a row: a power of two, side by side. Whole warps
// call it. `red` is not written again before the group has passed another barrier.
template <int NS>
__device__ __forceinline__ void row_sums(float (&v)[NS], int G, float (*red)[32]) {
  const int top = G < 32 ? G : 32;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < top)
#pragma unroll
      for (int k = 0; k < NS; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (G <= 32) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = G >> 5;
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < NS; ++k) red[k][warp] = v[k];
  group_barrier(G);
#pragma unroll
  for (int k = 0; k < NS; ++k) v[k] = red[k][(warp & ~(warps - 1)) + (lane & (warps - 1))];
  for (int o = warps >> 1; o > 0; o >>= 1)
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
  int ring;         // bytes of the ring, and of what else lies there
  float eps;
};

// The rows to come lie in a ring in shared memory, fetched with cp.async, 16 bytes a copy.
//
// Vectors (VEC > 1: bases, strides and d multiples of 16 bytes): a thread reads back the
// vectors that it fetched itself, so no barrier is needed. Slot (stage, load, thread).
//
// Single elements (anything else): the group fetches the aligned blocks of 16 bytes around
// its row (never a byte outside a block of which the row has a part) and, behind a
// barrier, each thread takes the columns tid, tid + G, ... (An aligned four bytes for each element, fetched by
// the thread itself: 16384 x 1001 bf16 36 us, 70 in the gradient. A test of each column
// against d costs as many instructions as its arithmetic.)
__device__ __forceinline__ void fetch16(void* slot, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(slot)), "l"(src) : "memory");
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void fetch_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

// One tensor's part of a stage. `at`: the thread's first slot, or the group's row.
template <typename T, int VEC, int NV>
struct Row {
  // Loads whose columns all lie below d: of single elements the first half, for a row is
  // wider than half of what its threads hold (launch_typed).
  static constexpr int kSure = VEC == 1 && NV > 4 ? NV / 2 : 0;
  static __device__ __forceinline__ int offset(const T* src) {
    return VEC == 1 ? static_cast<int>(reinterpret_cast<uintptr_t>(src) & 15) : 0;
  }
  // Vectors past d, which no fetch writes: zeros, in every stage of the ring.
  static __device__ __forceinline__ void clear(uint8_t* ring, int bytes, int tid, int G, int d) {
    if (VEC == 1 || G * NV * VEC == d) return;
    for (int k = 0; k < bytes; k += 16 * NV * kRowThreads)
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((tid + i * G) * VEC >= d) *reinterpret_cast<uint4*>(ring + k + (i * kRowThreads + threadIdx.x) * 16) = make_uint4(0, 0, 0, 0);
  }
  static __device__ __forceinline__ void fetch(uint8_t* at, const T* src, int tid, int G, int d) {
    if constexpr (VEC > 1) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((tid + i * G) * VEC < d) fetch16(at + i * 16 * kRowThreads, src + (tid + i * G) * VEC);
    } else {
      const uint8_t* first = reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(src) & ~static_cast<uintptr_t>(15));
      const int blocks = (static_cast<int>(reinterpret_cast<uintptr_t>(src) & 15) + d * static_cast<int>(sizeof(T)) + 15) / 16;
      for (int q = tid; q < blocks; q += G) fetch16(at + 16 * q, first + 16 * q);
    }
  }
  // Load i's values; past d 0. off: the row's offset in its first block.
  static __device__ __forceinline__ void get(const uint8_t* at, int off, int i, int tid, int G, int d, float* v) {
    if constexpr (VEC == 8) {
      const uint4 u = *reinterpret_cast<const uint4*>(at + i * 16 * kRowThreads);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = __uint_as_float(w[k] << 16);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      }
    } else if constexpr (VEC == 4) {
      const float4 u = *reinterpret_cast<const float4*>(at + i * 16 * kRowThreads);
      v[0] = u.x;
      v[1] = u.y;
      v[2] = u.z;
      v[3] = u.w;
    } else {
      // What lies behind a row in shared memory (other rows, the weights) is read and dropped.
      const float x = to_f32(reinterpret_cast<const T*>(at + off)[tid + i * G]);
      v[0] = i < kSure || tid + i * G < d ? x : 0.f;
    }
  }
};

template <typename T, int VEC>
__device__ __forceinline__ void store(T* dst, const float* v) {
  if constexpr (VEC == 8) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                                pack_bf16x2(v[6], v[7]));
  } else if constexpr (VEC == 4) {
    *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    *dst = from_f32<T>(v[0]);
  }
}

// The parameters of vector i (of width / VEC) in shared memory: eight of them lie apart
// in two runs of four, so that neighbouring threads' 16-byte loads meet different banks.
template <int VEC>
__device__ __forceinline__ void load_params(const float* src, int i, int width, float* v) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int k = 0; k < VEC; k += 4) {
      const float4 u = *reinterpret_cast<const float4*>(src + (k ? width / 2 : 0) + i * 4);
      v[k] = u.x;
      v[k + 1] = u.y;
      v[k + 2] = u.z;
      v[k + 3] = u.w;
    }
  } else {
    v[0] = src[i];
  }
}
template <int VEC>
__device__ __forceinline__ int param_place(int e, int width) {
  return VEC == 8 ? (e & 4 ? width / 2 : 0) + (e >> 3) * 4 + (e & 3) : e;
}

// VEC: elements per load (16 bytes, or one where a base, a stride or d is not a multiple
// of that); NV: loads per thread, row and tensor. CTAs on an SM by the registers that the
// elements a thread holds take; the ring's depth by the shared memory of each, kShort: a row less.
template <int VEC, int NV, bool kGradient, bool kShort>
struct Held {
  static constexpr int kElems = VEC * NV;
  static constexpr int kTensors = kGradient ? 2 : 1;
  static constexpr int kStage = 16 * NV * kRowThreads * kTensors;  // bytes (vectors)
  static constexpr int kShared = (kGradient ? 192 : 144) * 1024;
  static constexpr int kCtas = VEC == 1 ? (kElems <= 8 ? 4 : 2)
                               : kElems <= 8 ? 4 : !kGradient && kStage <= 16384 ? 3 : kShared / 2 / kStage >= 2 ? 2 : 1;
  static constexpr int kRoom = kShared / kCtas / kStage;
  static constexpr int kDepth = VEC == 1 ? (NV <= 4 ? 6 : NV <= 8 ? 4 : 3) : kRoom > 6 ? 6 : kRoom - (kShort ? 1 : 0);
  static_assert(kDepth >= 2, "a ring of one row waits for every load");
};

// Bytes of a row's part of a stage (single elements): its length and up to 15 at either end.
__host__ __device__ inline int row_room(int d, int esz) { return (d * esz + 15) / 16 * 16 + 16; }

// The columns a group's threads hold, a multiple of what d needs.
__host__ __device__ inline int held_width(int G, int elems) { return G * elems; }

// The weight (and bias) in fp32 behind the ring, zeros past d.
template <int VEC>
__device__ __forceinline__ void stage_params(const NormParams& p, float* w, float* b, int width) {
  for (int e = threadIdx.x; e < width; e += kRowThreads) {
    const int at = param_place<VEC>(e, width);
    w[at] = e < p.d ? load_param(p.w, p.w_bf16, e) : 0.f;
    if (b) b[at] = e < p.d && p.b ? load_param(p.b, p.w_bf16, e) : 0.f;
  }
  __syncthreads();
}

template <typename T, int VEC, int NV, bool kShort>
__global__ void __launch_bounds__(kRowThreads, (Held<VEC, NV, false, kShort>::kCtas)) norm_kernel(const NormParams p) {
  using H = Held<VEC, NV, false, kShort>;
  using Src = Row<T, VEC, NV>;
  constexpr int kElems = H::kElems, kDepth = H::kDepth;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[2][1][32];
  const int G = p.G, R = kRowThreads / G, tid = threadIdx.x % G, d = p.d, width = held_width(G, kElems);
  const int stage_bytes = p.ring / kDepth;
  uint8_t* ring = smem + (VEC > 1 ? 16 * threadIdx.x : threadIdx.x / G * row_room(d, sizeof(T)));
  float* w = reinterpret_cast<float*>(smem + p.ring);
  float* b = w + width;
  const float inv_d = 1.f / static_cast<float>(d);
  const bool full = VEC > 1 && width == d;  // every element held is one of the row
  Src::clear(smem, p.ring, tid, G, d);
  wait_for_previous();
  const int64_t step = static_cast<int64_t>(gridDim.x) * R;
  int64_t row = static_cast<int64_t>(blockIdx.x) * R + threadIdx.x / G;
  // Whole warps stay together: the first row of a warp's groups says when it ends.
  int64_t warp_row = static_cast<int64_t>(blockIdx.x) * R + (threadIdx.x & ~31) / G;
  const T* src = static_cast<const T*>(p.x);
  const auto ask = [&](int64_t r, int stage) {
    if (r < p.N) Src::fetch(ring + stage * stage_bytes, src + r * p.s_x, tid, G, d);
    fetch_commit();
  };
#pragma unroll
  for (int k = 0; k < kDepth; ++k) ask(row + k * step, k);
  stage_params<VEC>(p, w, b, width);
  int stage = 0;
  for (; warp_row < p.N; warp_row += step, row += step) {
    fetch_wait<kDepth - 1>();
    if (VEC == 1) group_barrier(G);  // the whole row is there
    float x[kElems];
#pragma unroll
    for (int i = 0; i < NV; ++i) Src::get(ring + stage * stage_bytes, Src::offset(src + row * p.s_x), i, tid, G, d, x + i * VEC);
    float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kElems; j += 2) s2 = fadd2(s2, make_float2(x[j], x[j + 1]));
    float s[1] = {s2.x + s2.y};
    row_sums<1>(s, G, red[0]);
    if (VEC == 1) group_barrier(G);  // the row has been read
    ask(row + kDepth * step, stage);
    stage = stage + 1 == kDepth ? 0 : stage + 1;
    const float mean = s[0] * inv_d;
    const float2 m2 = make_float2(-mean, -mean);
    s2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kElems; j += 2) {
      const float2 c = fadd2(make_float2(x[j], x[j + 1]), m2);
      x[j] = c.x;
      x[j + 1] = c.y;
    }
    if (!full)
#pragma unroll
      for (int i = Src::kSure; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < VEC; ++k) x[i * VEC + k] = (tid + i * G) * VEC >= d ? 0.f : x[i * VEC + k];
#pragma unroll
    for (int j = 0; j < kElems; j += 2) s2 = ffma2(make_float2(x[j], x[j + 1]), make_float2(x[j], x[j + 1]), s2);
    s[0] = s2.x + s2.y;
    row_sums<1>(s, G, red[1]);
    const float rstd = 1.f / sqrtf(s[0] * inv_d + p.eps);
    if (row >= p.N) continue;
    T* o = static_cast<T*>(p.out) + row * p.s_out + tid * VEC;
    const float2 r2 = make_float2(rstd, rstd);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float wv[VEC], bv[VEC];
      load_params<VEC>(w, tid + i * G, width, wv);
      load_params<VEC>(b, tid + i * G, width, bv);
      if constexpr (VEC == 1) {
        wv[0] = fmaf(x[i] * rstd, wv[0], bv[0]);
      } else {
#pragma unroll
        for (int k = 0; k < VEC; k += 2) {
          const float2 y = ffma2(fmul2(make_float2(x[i * VEC + k], x[i * VEC + k + 1]), r2), make_float2(wv[k], wv[k + 1]),
                                 make_float2(bv[k], bv[k + 1]));
          wv[k] = y.x;
          wv[k + 1] = y.y;
        }
      }
      if (i < Src::kSure || full || (tid + i * G) * VEC < d) store<T, VEC>(o + i * G * VEC, wv);
    }
    if (tid == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
  fetch_wait<0>();
}

template <typename T, int VEC, int NV, bool kShort>
__global__ void __launch_bounds__(kRowThreads, (Held<VEC, NV, true, kShort>::kCtas)) norm_grad_kernel(const NormParams p) {
  using H = Held<VEC, NV, true, kShort>;
  using Src = Row<T, VEC, NV>;
  constexpr int kElems = H::kElems, kDepth = H::kDepth;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[2][2][32];
  const int G = p.G, R = kRowThreads / G, g = threadIdx.x / G, tid = threadIdx.x % G, d = p.d, width = held_width(G, kElems);
  const int stage_bytes = p.ring / kDepth;
  uint8_t* ring = smem + (VEC > 1 ? 16 * threadIdx.x : g * row_room(d, sizeof(T)));  // x, and dy half a stage on
  float* w = reinterpret_cast<float*>(smem + p.ring);
  const float inv_d = 1.f / static_cast<float>(d);
  const bool full = VEC > 1 && width == d;
  Src::clear(smem, p.ring, tid, G, d);
  wait_for_previous();
  const int64_t step = static_cast<int64_t>(gridDim.x) * R;
  int64_t row = static_cast<int64_t>(blockIdx.x) * R + g;
  int64_t warp_row = static_cast<int64_t>(blockIdx.x) * R + (threadIdx.x & ~31) / G;
  const T* src_x = static_cast<const T*>(p.x);
  const T* src_dy = static_cast<const T*>(p.dy);
  const auto ask = [&](int64_t r, int stage) {
    if (r < p.N) {
      Src::fetch(ring + stage * stage_bytes, src_x + r * p.s_x, tid, G, d);
      Src::fetch(ring + stage * stage_bytes + stage_bytes / 2, src_dy + r * p.s_dy, tid, G, d);
    }
    fetch_commit();
  };
#pragma unroll
  for (int k = 0; k < kDepth; ++k) ask(row + k * step, k);
  stage_params<VEC>(p, w, nullptr, width);
  float2 dw[kElems / 2], db[kElems / 2];
#pragma unroll
  for (int j = 0; j < kElems / 2; ++j) dw[j] = db[j] = make_float2(0.f, 0.f);
  float mean = row < p.N ? p.mean[row] : 0.f, rstd = row < p.N ? p.rstd[row] : 0.f;
  int parity = 0, stage = 0;
  for (; warp_row < p.N; warp_row += step, row += step, parity ^= 1) {
    const int64_t after = row + step;
    const float next_mean = after < p.N ? p.mean[after] : 0.f, next_rstd = after < p.N ? p.rstd[after] : 0.f;
    const float2 m2 = make_float2(-mean, -mean), r2 = make_float2(rstd, rstd);
    const int off_x = Src::offset(src_x + row * p.s_x), off_dy = Src::offset(src_dy + row * p.s_dy);
    // kPair elements at a time: a vector, or two loads of one element. Past d x, dy and w
    // are 0, and so is all that is added up.
    constexpr int kPair = VEC == 1 ? 2 : VEC;
    const auto get = [&](int j, float* x, float* dy, float* wv) {
      constexpr int kLoads = kPair / VEC;
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        const int i = j / VEC + l;
        Src::get(ring + stage * stage_bytes, off_x, i, tid, G, d, x + l);
        Src::get(ring + stage * stage_bytes + stage_bytes / 2, off_dy, i, tid, G, d, dy + l);
        load_params<VEC>(w, tid + i * G, width, wv + l);
      }
    };
    fetch_wait<kDepth - 1>();
    if (VEC == 1) group_barrier(G);
    float2 s0 = make_float2(0.f, 0.f), s1 = s0;
    if (row < p.N) {  // a group without a row adds nothing
#pragma unroll
      for (int j = 0; j < kElems; j += kPair) {
        float x[kPair], dy[kPair], wv[kPair];
        get(j, x, dy, wv);
#pragma unroll
        for (int k = 0; k < kPair; k += 2) {
          const float2 xhat = fmul2(fadd2(make_float2(x[k], x[k + 1]), m2), r2), t = make_float2(dy[k], dy[k + 1]);
          const float2 a = fmul2(t, make_float2(wv[k], wv[k + 1]));
          s0 = fadd2(s0, a);
          s1 = ffma2(a, xhat, s1);
          dw[(j + k) / 2] = ffma2(t, xhat, dw[(j + k) / 2]);
          db[(j + k) / 2] = fadd2(db[(j + k) / 2], t);
        }
      }
    }
    float s[2] = {s0.x + s0.y, s1.x + s1.y};
    row_sums<2>(s, G, red[parity]);
    if (row < p.N) {
      // dx = rstd (dout w - ((x - mean) (rstd c2) + c1)): no square of rstd, which overflows where
      // a row's deviations are below 1e-19.
      const float c1 = -(s[0] * inv_d), c2 = -(rstd * (s[1] * inv_d));
      const float2 n1 = make_float2(c1, c1), n2 = make_float2(c2, c2);
      T* o = static_cast<T*>(p.out) + row * p.s_out + tid * VEC;
#pragma unroll
      for (int j = 0; j < kElems; j += kPair) {
        float x[kPair], dy[kPair], wv[kPair];
        get(j, x, dy, wv);
#pragma unroll
        for (int k = 0; k < kPair; k += 2) {
          const float2 rest = ffma2(fadd2(make_float2(x[k], x[k + 1]), m2), n2, n1);
          const float2 y = fmul2(ffma2(make_float2(dy[k], dy[k + 1]), make_float2(wv[k], wv[k + 1]), rest), r2);
          x[k] = y.x;
          x[k + 1] = y.y;
        }
#pragma unroll
        for (int l = 0; l < kPair / VEC; ++l) {
          const int i = j / VEC + l;
          if (i < Src::kSure || full || (tid + i * G) * VEC < d) store<T, VEC>(o + i * G * VEC, x + l);
        }
      }
    }
    if (VEC == 1) group_barrier(G);
    ask(row + kDepth * step, stage);
    stage = stage + 1 == kDepth ? 0 : stage + 1;
    mean = next_mean;
    rstd = next_rstd;
  }
  fetch_wait<0>();
  if (!p.part) return;
  // The groups' sums of each column, dw's and then db's, joined through the ring's memory.
  float* part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * d;
  float* cols = reinterpret_cast<float*>(smem);
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kElems; ++j) {
      const float2 v = which ? db[j / 2] : dw[j / 2];
      cols[g * width + (tid + j / VEC * G) * VEC + j % VEC] = j & 1 ? v.y : v.x;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < d; e += kRowThreads) {
      float sum = 0.f;
      for (int r = 0; r < R; ++r) sum += cols[r * width + e];
      part[which * d + e] = sum;
    }
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

// Adds the parts of 8 columns (a sector; blockIdx.x) of dw or db (blockIdx.y) in a fixed
// order, 32 threads a column, each with its loads in flight at once. (32 columns and 1024
// threads a CTA: 7.5 us instead of 4.)
constexpr int kReduceThreads = 256;
__global__ void __launch_bounds__(kReduceThreads)
    norm_reduce_kernel(const float* part, int parts, int d, int bf16, void* dw, void* db) {
  __shared__ float sums[kReduceThreads / 32][8];
  void* out = blockIdx.y ? db : dw;
  if (!out) return;
  wait_for_previous();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 8 + (lane & 7);
  float s = 0.f;
  const float* src = part + static_cast<int64_t>(blockIdx.y) * d + c;
  for (int i = warp * 4 + (lane >> 3); i < parts; i += kReduceThreads) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int at = i + k * (kReduceThreads / 8);
      v[k] = c < d && at < parts ? src[static_cast<int64_t>(at) * 2 * d] : 0.f;
    }
    s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  }
  s += __shfl_xor_sync(0xffffffffu, s, 8);
  s += __shfl_xor_sync(0xffffffffu, s, 16);
  if (lane < 8) sums[warp][lane] = s;
  __syncthreads();
  if (threadIdx.x >= 8 || c >= d) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kReduceThreads / 32; ++i) s += sums[i][lane];
  if (bf16)
    static_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(s);
  else
    static_cast<float*>(out)[c] = s;
}

// Threads a row and loads a thread. Many rows: as many loads as a thread holds, so that few
// threads pay for each row, and several rows share a warp. Few rows: more threads each,
// while half of them still find a place at once, for the chain of loads and sums is what a
// call then waits for (512 x 2048 bf16: 3.6 us).
struct Shape {
  int G, nv;
};

Shape shape_of(int64_t N, int64_t loads, int most_nv, int sms) {
  int G = 8, nv = 1;
  while (static_cast<int64_t>(G) * nv < loads) {
    if (nv < most_nv)
      nv *= 2;
    else
      G *= 2;
  }
  while (nv > 1 && G < kRowThreads && N * G * 2 <= static_cast<int64_t>(sms) * 512) {
    G *= 2;
    nv /= 2;
  }
  return {G, nv};
}

bool by_vectors(const void* p, int64_t stride, int esz) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * esz % 16 == 0;
}

// Shared memory of a CTA: the ring, and the weights (and biases).
template <typename H, int VEC>
size_t held_bytes(bool grad, const NormParams& p, int esz) {
  const int R = kRowThreads / p.G, width = held_width(p.G, H::kElems);
  int ring = H::kDepth * (VEC > 1 ? H::kStage : R * row_room(p.d, esz) * H::kTensors);
  // The groups' columns' sums take the ring's place at the end.
  const int unit = H::kDepth * 32;
  if (grad && ring < R * width * 4) ring = (R * width * 4 + unit - 1) / unit * unit;
  return ring + static_cast<size_t>(width) * 4 * (grad ? 1 : 2);
}

// CTAs that find room on an SM beside each other (each takes 1 KB for the system, and what
// is declared in the kernel): the weights of wide rows leave it for fewer than the registers do.
template <typename H>
int held_ctas(size_t smem) {
  const int fit = static_cast<int>(228 * 1024 / (smem + 1024 + 512));
  return fit < 1 ? 1 : fit < H::kCtas ? fit : H::kCtas;
}

// One CTA for every place on the SMs, or fewer: each walks rows.
template <typename T, int VEC, int NV, bool kGradient, bool kShort>
cudaError_t launch_held(NormParams p, int sms, int* parts, cudaStream_t stream) {
  using H = Held<VEC, NV, kGradient, kShort>;
  const size_t smem = held_bytes<H, VEC>(kGradient, p, sizeof(T));
  if constexpr (!kShort && VEC == 8 && NV > 2) {
    // A row less in the ring where that leaves room for one more CTA (16384 x 2048 elements as
    // rows of 8192: 46.4 -> 36.8 us, the gradients 61.6 -> 57.4; fp32 rows gain nothing).
    using S = Held<VEC, NV, kGradient, true>;
    if (held_ctas<S>(held_bytes<S, VEC>(kGradient, p, sizeof(T))) > held_ctas<H>(smem))
      return launch_held<T, VEC, NV, kGradient, true>(p, sms, parts, stream);
  }
  const auto kernel = kGradient ? norm_grad_kernel<T, VEC, NV, kShort> : norm_kernel<T, VEC, NV, kShort>;
  const int R = kRowThreads / p.G;
  p.ring = static_cast<int>(smem) - held_width(p.G, H::kElems) * 4 * (kGradient ? 1 : 2);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  const int most = norm_max_parts(p.d);
  int places = sms * held_ctas<H>(smem);
  if (kGradient && places > most) places = most;
  const int64_t want = (p.N + R - 1) / R;
  *parts = static_cast<int>(want < places ? want : places);
  return launch_overlapped(kernel, dim3(static_cast<unsigned>(*parts)), kRowThreads, smem, stream, 1, true, p);
}

template <typename T, int VEC, int NV>
cudaError_t launch_shape(bool grad, const NormParams& p, int sms, int* parts, cudaStream_t stream) {
  return grad ? launch_held<T, VEC, NV, true, false>(p, sms, parts, stream) : launch_held<T, VEC, NV, false, false>(p, sms, parts, stream);
}

template <typename T, int VEC>
cudaError_t launch_wide(bool grad, const NormParams& p, int sms, int* parts, cudaStream_t stream) {
  const int64_t most = p.N < 2 * sms ? p.N : 2 * sms;
  cudaError_t e = launch_overlapped(grad ? norm_grad_wide_kernel<T, VEC> : norm_wide_kernel<T, VEC>,
                                    dim3(static_cast<unsigned>(most)), kWideThreads, 0, stream, 1, true, p);
  if (e != cudaSuccess || !p.part) return e;
  const int64_t room = norm_max_parts(p.d) < sms ? norm_max_parts(p.d) : sms;
  *parts = static_cast<int>(p.N < room ? p.N : room);
  return launch_overlapped(norm_columns_kernel<T>, dim3(static_cast<unsigned>((p.d + kRowThreads - 1) / kRowThreads), *parts),
                           kRowThreads, 0, stream, 1, true, p);
}

// *parts: the parts of dw and db that the launches write.
template <typename T>
int launch_typed(bool grad, NormParams p, int* parts, cudaStream_t stream) {
  constexpr int kVec = 16 / static_cast<int>(sizeof(T));
  const bool vec = p.d % kVec == 0 && by_vectors(p.x, p.s_x, sizeof(T)) && by_vectors(p.out, p.s_out, sizeof(T)) &&
                   (!grad || by_vectors(p.dy, p.s_dy, sizeof(T)));
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  cudaError_t e;
  if (p.d > kHeldWidth) {
    e = vec ? launch_wide<T, kVec>(grad, p, sms, parts, stream) : launch_wide<T, 1>(grad, p, sms, parts, stream);
  } else {
    Shape s = vec ? shape_of(p.N, p.d / kVec, 32 / kVec, sms) : shape_of(p.N, (p.d + 3) / 4 * 4, 32, sms);
    // Three quarters of the loads where they hold the row (16384 x 2048 elements as rows of
    // 2560 bf16: 37 -> 34 us, the gradients 59 -> 52; of 6144 42 -> 37, 59 -> 54), but not the
    // gradients of narrow fp32 rows, where two CTAs with two rows each in their rings do worse
    // than one with three (1536: 71 -> 76; 2560: 86 -> 76).
    if (vec && s.nv == 32 / kVec && s.G * (24 / kVec) >= p.d / kVec && (!grad || kVec == 8 || p.d > 2048)) s.nv = 24 / kVec;
    p.G = s.G;
    if (vec)
      e = s.nv == 1   ? launch_shape<T, kVec, 1>(grad, p, sms, parts, stream)
          : s.nv == 2 ? launch_shape<T, kVec, 2>(grad, p, sms, parts, stream)
          : s.nv == 24 / kVec ? launch_shape<T, kVec, 24 / kVec>(grad, p, sms, parts, stream)
          : s.nv == 4 ? launch_shape<T, kVec, 4>(grad, p, sms, parts, stream)
                      : launch_shape<T, kVec, 32 / kVec>(grad, p, sms, parts, stream);
    else
      e = s.nv <= 4    ? launch_shape<T, 1, 4>(grad, p, sms, parts, stream)
          : s.nv <= 8  ? launch_shape<T, 1, 8>(grad, p, sms, parts, stream)
          : s.nv <= 16 ? launch_shape<T, 1, 16>(grad, p, sms, parts, stream)
                       : launch_shape<T, 1, 32>(grad, p, sms, parts, stream);
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
  int parts;
  return a.is_bf16 ? launch_typed<__nv_bfloat16>(false, p, &parts, stream) : launch_typed<float>(false, p, &parts, stream);
}

int launch_layer_norm_grad(const NormArgs& a, cudaStream_t stream) {
  NormParams p = params_of(a);
  p.dy = a.dout;
  p.s_dy = a.s_dout;
  p.out = a.dx;
  p.s_out = a.s_dx;
  p.part = a.dweight || a.dbias ? static_cast<float*>(a.workspace) : nullptr;
  int parts = 0;
  if (a.N > 0) {
    const int st = a.is_bf16 ? launch_typed<__nv_bfloat16>(true, p, &parts, stream) : launch_typed<float>(true, p, &parts, stream);
    if (st != DLM_OK) return st;
  }
  if (!a.dweight && !a.dbias) return DLM_OK;
  const cudaError_t e =
      launch_overlapped(norm_reduce_kernel, dim3(static_cast<unsigned>((a.d + 7) / 8), 2), kReduceThreads, 0, stream, 1,
                        true, static_cast<const float*>(a.workspace), parts, p.d, a.weight_bf16, a.dweight, a.dbias);
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "layer norm reduction launch: %s", cudaGetErrorString(e));
}

}  // namespace dlm
