// The activations of products whose rows lie one expert's behind the other's (ROWS in the grouped GEMM's kernels), applied to the fp32 sums before their one rounding.
#pragma once
#include "common.h"

namespace moe {
namespace {

// Phi(-y) = erfc(y / sqrt 2) / 2 = 2^-(P(y) + 1) for y >= 0, with a polynomial of degree 9 and P(0) = 0, fitted to equal ripple in P over [0, 13.2], where bf16's
// smallest normal number is reached: 2.1e-5 of Phi(-y) throughout, so that GeLU is exact to 1/160 of a bf16 rounding also where it is small itself (to 5e-5 with the
// fp32 evaluation).  One exponential, no division.
constexpr float kPhi[9] = {1.151095026e+00f, 4.586445080e-01f, 5.404893616e-02f, -8.699391121e-03f, 1.027744177e-03f, -8.451740843e-05f, 4.530642880e-06f, -1.413703882e-07f, 1.939663995e-09f};
constexpr float kPhiEnd = 13.2f;
__device__ __forceinline__ float normal_tail(float y) {             // Phi(-y), 0 <= y <= kPhiEnd
  float p = kPhi[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) p = fmaf(p, y, kPhi[i]);
  return __builtin_amdgcn_exp2f(fmaf(-p, y, -1.0f));
}

// bf16 results.  ReLU keeps a NaN; SiLU by the hardware's exponential and reciprocal, 1e-6.
template <int ACT> __device__ __forceinline__ float rows_act(float v) {
  if (ACT == MOE_ACT_RELU) return v < 0.f ? 0.f : v;
  if (ACT == MOE_ACT_GELU) {                                        // v Phi(v) = max(v, 0) - |v| Phi(-|v|); a NaN stays one
    const float y = fminf(fabsf(v), kPhiEnd);
    return fmaf(-y, normal_tail(y), v < 0.f ? 0.f : v);
  }
  if (ACT == MOE_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.0f + __expf(-v));
  return v;
}
// The derivative: phi(v) = exp2(-v^2 / (2 ln 2)) / sqrt(2 pi); 7e-6 for GeLU.
template <int ACT> __device__ __forceinline__ float rows_act_grad(float v) {
  if (ACT == MOE_ACT_RELU) return v > 0.f ? 1.f : 0.f;
  if (ACT == MOE_ACT_GELU) {
    const float t = normal_tail(fminf(fabsf(v), kPhiEnd));
    return fmaf(v, __builtin_amdgcn_exp2f(-0.72134752f * v * v) * 0.39894228f, v < 0.f ? t : 1.f - t);
  }
  if (ACT == MOE_ACT_SILU) {
    const float sg = __builtin_amdgcn_rcpf(1.0f + __expf(-v));
    return sg * fmaf(v, 1.f - sg, 1.f);
  }
  return 1.f;
}

// fp32 results: erf, exp and divisions to fp32's own accuracy.
template <int ACT> __device__ __forceinline__ float rows_act32(float v) {
  if (ACT == MOE_ACT_RELU) return v < 0.f ? 0.f : v;
  if (ACT == MOE_ACT_GELU) return v * (0.5f * erfcf(v * -0.70710678118654752440f));
  if (ACT == MOE_ACT_SILU) return v / (1.0f + expf(-v));
  return v;
}
template <int ACT> __device__ __forceinline__ float rows_act_grad32(float v) {
  if (ACT == MOE_ACT_RELU) return v > 0.f ? 1.f : 0.f;
  if (ACT == MOE_ACT_GELU) return fmaf(v, expf(-0.5f * v * v) * 0.39894228040143267794f, 0.5f * erfcf(v * -0.70710678118654752440f));
  if (ACT == MOE_ACT_SILU) {
    const float sg = 1.f / (1.f + expf(-v));
    return sg * (1.f + v * (1.f - sg));
  }
  return 1.f;
}

template <typename ET, int ACT> __device__ __forceinline__ float rows_act_as(float v) {
  if constexpr (sizeof(ET) == 2) return rows_act<ACT>(v);
  else return rows_act32<ACT>(v);
}
template <typename ET, int ACT> __device__ __forceinline__ float rows_act_grad_as(float v) {
  if constexpr (sizeof(ET) == 2) return rows_act_grad<ACT>(v);
  else return rows_act_grad32<ACT>(v);
}

}  // namespace
}  // namespace moe
