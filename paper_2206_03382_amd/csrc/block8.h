// The 8-bit block format: e4m3 values in blocks of 128 along the axis that a product sums over, each with one power of two 2^e, kept as the
// byte e + 127.  The matrix cores take such a byte with an operand and apply it for nothing; multiplying by it is exact, so it costs no
// accuracy but up to one bit of the block's range.  e is the smallest with amax <= 448 * 2^e (448: the largest e4m3 value), and at least -126, so
// that 2^-e is a normal fp32 number too.  A block that holds an infinity or NaN has the byte 255 and only NaNs.
//
// Layout: rows of values are zero-padded to whole blocks (row_bytes8), rows of exponents to a multiple of four bytes with 127 (row_scales8): a
// product loads the exponents of four blocks as one word and never looks at the row's end.
#pragma once
#include "common.h"

namespace moe {

constexpr int kBlock8 = 128;
constexpr uint32_t kScaleOne = 127, kScaleNaN = 255;

static inline __host__ __device__ int64_t row_bytes8(int64_t K) { return ceil_div(K, kBlock8) * kBlock8; }
static inline __host__ __device__ int64_t row_scales8(int64_t K) { return ceil_div(ceil_div(K, kBlock8), 4) * 4; }

// The exponent byte of a block from the bits of its largest magnitude.  Compared as integers NaN > inf > finite, so a maximum over the bits
// of |v| keeps a NaN that a floating maximum would lose.
__device__ __forceinline__ uint32_t scale_of_amax(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kScaleNaN;
  const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);   // 448 = 1.75 * 2^8
  return e < 1 ? 1u : (uint32_t)e;
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) {     // 2^-e; the finite ones are at most 247
  return __uint_as_float(byte == kScaleNaN ? 0x7fc00000u : (254u - byte) << 23);
}

// four values times m = inverse_scale(their block's exponent) -> four e4m3 bytes, round to nearest even
__device__ __forceinline__ uint32_t pack8x4(float a, float b, float c, float d, float m) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * m, b * m, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c * m, d * m, w, true);
  return (uint32_t)w;
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// maximum over a row of 16 lanes, in all of them: quads, then their mirror images
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  auto with = [&](uint32_t o) { v = v > o ? v : o; };
  with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));      // quad_perm 1,0,3,2
  with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));      // quad_perm 2,3,0,1
  with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));     // row_half_mirror
  with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));     // row_mirror
  return v;
}

// ReLU that keeps a NaN, which apply_act's (max(v, 0), of the layer in the storage types) does not.
__device__ __forceinline__ float relu_or_nan(float v) { return v <= 0.f ? 0.f : v; }
__device__ __forceinline__ float act_full(float v, int act) { return act == MOE_ACT_RELU ? relu_or_nan(v) : apply_act(v, act); }

// The activations of results in 8 bits.  gelu(v) = v Phi(v) with Phi(-y) = 2^-P(y) / 2, P of degree 7 fitted to -log2 erfc(y / sqrt 2) on [0, 8] for the least largest error, 4.5e-5: 3e-5 of
// Phi there, where half a step of the format is 6e-2 (and below 1e-14 beyond).  One exponential, no division; the erf form costs as much as a K-step of the products.  SiLU's exponential and reciprocal are the hardware's, good to 2^-21 or so.
constexpr float kPhi8C1 = 1.15079675f, kPhi8C2 = 4.59715568e-01f, kPhi8C3 = 5.27749787e-02f, kPhi8C4 = -7.98642309e-03f, kPhi8C5 = 8.14003300e-04f,
                kPhi8C6 = -4.87606510e-05f, kPhi8C7 = 1.28089860e-06f;
template <int ACT> __device__ __forceinline__ float act8(float v) {
  if (ACT == MOE_ACT_RELU) return relu_or_nan(v);
  if (ACT == MOE_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.0f + __expf(-v));
  if (ACT == MOE_ACT_GELU) {
    const float y = fabsf(v);
    float s = fmaf(kPhi8C7, y, kPhi8C6);
    s = fmaf(s, y, kPhi8C5);
    s = fmaf(s, y, kPhi8C4);
    s = fmaf(s, y, kPhi8C3);
    s = fmaf(s, y, kPhi8C2);
    s = fmaf(s, y, kPhi8C1);
    const float tail = 0.5f * __builtin_amdgcn_exp2f(-(s * y));     // Phi(-|v|)
    return v * (v < 0.f ? tail : 1.0f - tail);
  }
  return v;
}

// ---- launchers (norm.hip, quantize8.hip, matmul8.hip, few_tokens.hip); arguments are already validated ---------------------
hipError_t launch_rms_norm(const void* x, const void* residual, const void* weight, float eps, int dtype, int64_t T, int64_t M, void* h,
                           void* y, void* q, uint8_t* scales, hipStream_t s);
size_t rms_norm_backward_workspace_bytes(int64_t T, int64_t M);
hipError_t launch_rms_norm_backward(const void* dy, const void* dh, const void* h, const void* weight, float eps, int dtype, int64_t T,
                                    int64_t M, float* ws, void* dx, void* dweight, hipStream_t s);
// fills [E]: gets min(counts[e], R), not below 0.  zeros [E, R, zero_width] in dtype: rows past the counts get zeros.
hipError_t launch_quantize8(const void* src, int dtype, const int32_t* counts, int64_t E, int64_t R, int64_t K, bool blocks, void* q,
                            uint8_t* scales, void* qt, uint8_t* scales_t, hipStream_t s, int32_t* fills = nullptr, void* zeros = nullptr,
                            int64_t zero_width = 0);
hipError_t launch_dequantize8(const void* q, const uint8_t* scales, bool blocks, int64_t E, int64_t R, int64_t K, int dtype, void* out,
                              hipStream_t s);

// out[e] (rows_e x N) = act(A[e] (rows_e x K) * B[e]^T + bias[e]), B [E, N, K]; A and B in the 8-bit format with blocks along K.
struct Matmul8 {
  const void* A;
  const uint8_t* A_scales;        // [E, C, row_scales8(K)], or of the gathered matrix [gather_rows, ..]
  const void* B;
  const uint8_t* B_scales;        // [E, N, ..], or [E, ceil(N / 128), ..] with b_blocks
  int b_blocks;
  const void* bias;               // [E, N] in bias_dtype, or null
  int act;                        // MOE_ACT_*, < 0: none
  const int32_t* counts;          // live rows per expert, or null
  const int32_t* k_counts;        // live length of the sum per expert (values beyond it up to the block's end are zero), or null
  const int32_t* gather;          // row c of expert e is row gather[e, c] of one matrix
  int64_t gather_rows;
  int64_t E, C, K, N, rows_hint;  // rows_hint: as launch_grouped_gemm's
  int dtype;                      // of out and bias
  void* out;                      // [E, C, N], or null:
  void* out8;                     // [E, C, row_bytes8(N)] and its exponents instead
  uint8_t* out8_scales;
};
hipError_t launch_matmul8(const Matmul8& p, hipStream_t s);

struct FewTokens {
  const void *x, *Wg, *W1, *b1, *W2, *b2;
  const float* gate_bias;
  const uint8_t *s1, *s2;         // 8-bit weights [E, N, row_bytes8(K)] (blocks of 128 x 128), or null: [E, K, N] in dtype
  int32_t *idx, *loc, *counts;    // the gate's decisions: outputs
  float *gate_w, *logits;
  int64_t T, M, H, E, C;
  int k, act, dtype, normalize;
  bool planned, alone;            // set by launch_few_tokens, as are the next two
  int expert_bits, token_bits, slice_bits, up_bits, down_bits;
  double* logit_parts;            // few_logit_bytes: [slices, T, E]
  int32_t* plan;                  // [min(E, T k), kFewPlan]
  void* hidden;                   // [T k, H]
  float* partial;                 // few_partial_bytes: [parts, T k, H or M]
  int32_t* arrived;               // few_arrivals_bytes(M)
  void* out;
};
constexpr int kFewPlan = 2 + MOE_FEW_MAX_TOKENS;
size_t few_arrivals_bytes(int64_t M);
size_t few_logit_bytes(int64_t T, int64_t M, int64_t E);
size_t few_partial_bytes(int64_t T, int64_t M, int64_t H, int64_t E, int k);
hipError_t launch_few_tokens(const FewTokens& p, hipStream_t s);

}  // namespace moe
