// Activations of a feed-forward block, x sigmoid(s):
//   SiLU         s = x
//   GELU (tanh)  s = 2 sqrt(2 / pi) (x + 0.044715 x^3)   (x (1 + tanh(s / 2)) / 2)
// sigmoid(s) = 1 / (1 + 2^(-s log2 e)) with the approximate exponential and reciprocal: off by
// 2^-20 + 2^-21 min(|s|, 90) relative at most (their own 2^-22 each; s log2 e is rounded, and GELU's s
// three times before, which the exponential turns into relative errors), 2^-14.4 at the far end, where the
// rounding to bf16 behind it is 2^-8.
#pragma once

#include <cuda_bf16.h>

#include "dlm_common.cuh"

namespace dlm {

constexpr float kGelu = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kGeluCube = 0.044715f;

__device__ __forceinline__ float sigmoid_approx(float s) {
  float r;  // 1 / inf = 0
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2_approx(s * -1.4426950408889634f)));
  return r;
}

// `act` is DLM_ACT_*, the same in every thread.
__device__ __forceinline__ float activate(int act, float x) {
  if (act == DLM_ACT_NONE) return x;
  return x * sigmoid_approx(act == DLM_ACT_SILU ? x : kGelu * x * fmaf(kGeluCube, x * x, 1.f));
}

// Value and derivative at x: sigmoid (1 + x (1 - sigmoid) ds/dx). Past |x| = 100 the derivative
// is 0 or 1 and is taken there, where nothing overflows (a NaN stays one).
__device__ __forceinline__ void activate_grad(int act, float x, float* value, float* slope) {
  if (act == DLM_ACT_NONE) {
    *value = x;
    *slope = 1.f;
    return;
  }
  float c;
  asm("{\n.reg .f32 t;\nmin.NaN.f32 t, %1, 0f42C80000;\nmax.NaN.f32 %0, t, 0fC2C80000;\n}" : "=f"(c) : "f"(x));
  const bool silu = act == DLM_ACT_SILU;
  const float p = sigmoid_approx(silu ? c : kGelu * c * fmaf(kGeluCube, c * c, 1.f));
  const float ds = silu ? 1.f : kGelu * fmaf(3.f * kGeluCube, c * c, 1.f);
  *value = x * p;
  *slope = p * fmaf(c * (1.f - p), ds, 1.f);
}

__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __uint_as_float(w[k] << 16);
    x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
  }
}
// Eight neighbouring columns of a row; wide: 16-byte aligned.
__device__ __forceinline__ uint4 load8_raw(const __nv_bfloat16* src, bool wide) {
  if (wide) return *reinterpret_cast<const uint4*>(src);
  const unsigned short* h = reinterpret_cast<const unsigned short*>(src);
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = h[2 * k] | static_cast<uint32_t>(h[2 * k + 1]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* dst, bool wide, const float (&x)[8]) {
  if (wide) {
    *reinterpret_cast<uint4*>(dst) =
        make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) dst[k] = __float2bfloat16_rn(x[k]);
  }
}

}  // namespace dlm
