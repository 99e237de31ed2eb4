// The activations of products whose rows lie one expert's behind the other's (ROWS in the grouped GEMM's kernels), applied to the fp32 sums before their one rounding.
#pragma once
#include "common.h"

namespace moe {
namespace {

// Phi(-y) = erfc(y / sqrt 2) / 2 = 2^-(P(y) + 1) for y >= 0, with a polynomial of degree 9 and P(0) = 0, fitted to equal ripple in P over [0, 13.2], where v Phi(v) reaches
// the smallest normal number: 2.1e-5 of Phi(-y) in exact arithmetic, 5e-5 (1/78 of a bf16 rounding) with the fp32 evaluation, so that GeLU is exact to that also where it is small itself.  Up to 13.5,
// where its derivative is past that number and Phi(-y) 1/180 of it, 2e-4.  One exponential, no division.  The hardware's exponential gives zero instead of results below 2^-126, and
// Phi(-12.95) is there already: the exponent is raised by 10 and taken out again in the product with y.  From 13.47 on it is zero all the same.
constexpr float kPhi[9] = {1.151095026e+00f, 4.586445080e-01f, 5.404893616e-02f, -8.699391121e-03f, 1.027744177e-03f, -8.451740843e-05f, 4.530642880e-06f, -1.413703882e-07f, 1.939663995e-09f};
constexpr float kPhiEnd = 14.0f, kPhiUnit = 0x1p-10f;
__device__ __forceinline__ float normal_tail(float y) {             // Phi(-y) / kPhiUnit, 0 <= y <= kPhiEnd
  float p = kPhi[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) p = fmaf(p, y, kPhi[i]);
  return __builtin_amdgcn_exp2f(fmaf(-p, y, 9.0f));
}

// sigma(v) / kSigmaUnit by the hardware's exponential and reciprocal, likewise raised: v sigma(v) is a normal number down to v = -91.9, sigma(v) to -87.3, and 1 + exp(-v) is finite to -88.7.
constexpr float kSigmaUnit = 0x1p-8f;
__device__ __forceinline__ float sigma(float v) { return __builtin_amdgcn_rcpf(kSigmaUnit + __builtin_amdgcn_exp2f(fmaf(v, -1.44269504f, -8.0f))); }

// bf16 results.  ReLU keeps a NaN; SiLU to 2e-6 and the rounding of its exponential's argument, |v| 2^-23.
template <int ACT> __device__ __forceinline__ float rows_act(float v) {
  if (ACT == MOE_ACT_RELU) return v < 0.f ? 0.f : v;
  if (ACT == MOE_ACT_GELU) {                                        // v Phi(v) = max(v, 0) - |v| Phi(-|v|); a NaN stays one
    const float y = fminf(fabsf(v), kPhiEnd);
    return fmaf(-y * kPhiUnit, normal_tail(y), v < 0.f ? 0.f : v);
  }
  if (ACT == MOE_ACT_SILU) return v * kSigmaUnit * sigma(v);
  return v;
}
// The derivative.  GeLU: Phi(v) + v phi(v), phi(v) = exp2(-v^2 / (2 ln 2)) / sqrt(2 pi): each to the exponentials' accuracy of itself, together 7e-6 at most.
template <int ACT> __device__ __forceinline__ float rows_act_grad(float v) {
  if (ACT == MOE_ACT_RELU) return v > 0.f ? 1.f : 0.f;
  if (ACT == MOE_ACT_GELU) {
    const float t = normal_tail(fminf(fabsf(v), kPhiEnd));
    const float dens = __builtin_amdgcn_exp2f(fmaf(-0.72134752f * v, v, 10.0f));
    return fmaf(v * (kPhiUnit * 0.39894228f), dens, v < 0.f ? t * kPhiUnit : fmaf(-t, kPhiUnit, 1.f));
  }
  if (ACT == MOE_ACT_SILU) {
    const float s = sigma(v);
    return s * fmaf(v * kSigmaUnit, fmaf(-s, kSigmaUnit, 1.f), kSigmaUnit);
  }
  return 1.f;
}

// fp32 results: erfc, exp and divisions, whose arguments' roundings grow with v^2 and |v|: 16 + v^2 + 2 |v| roundings of fp32 at most for GeLU and its derivative's parts, 16 + 2 |v| for SiLU.  Below -64, where
// 1 + exp(-v) is exp(-v), SiLU takes exp(v) as exp(v + 32) exp(-32), so that it ends where its results do (-91.9) and not where exp(-v) does (-88.7).
constexpr float kExpMinus32 = 1.2664165549e-14f;
template <int ACT> __device__ __forceinline__ float rows_act32(float v) {
  if (ACT == MOE_ACT_RELU) return v < 0.f ? 0.f : v;
  if (ACT == MOE_ACT_GELU) return v * (0.5f * erfcf(v * -0.70710678118654752440f));
  if (ACT == MOE_ACT_SILU) return v < -64.f ? v * kExpMinus32 * expf(v + 32.f) : v / (1.0f + expf(-v));
  return v;
}
template <int ACT> __device__ __forceinline__ float rows_act_grad32(float v) {
  if (ACT == MOE_ACT_RELU) return v > 0.f ? 1.f : 0.f;
  if (ACT == MOE_ACT_GELU) return fmaf(v, expf(-0.5f * v * v) * 0.39894228040143267794f, 0.5f * erfcf(v * -0.70710678118654752440f));
  if (ACT == MOE_ACT_SILU) {
    if (v < -64.f) return fmaf(v, kExpMinus32, kExpMinus32) * expf(v + 32.f);
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
