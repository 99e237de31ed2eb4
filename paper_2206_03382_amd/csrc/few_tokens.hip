// The experts' feed-forward layer and the combine for a few tokens.
#include "block8.h"

namespace moe {
namespace {

// W[k, n] of expert e
template <typename ET>
__device__ __forceinline__ float weight_at(const void* W, const uint8_t* sc, int64_t e, int64_t k, int64_t n, int64_t K, int64_t N) {
  if (!sc) return load_as_f32((const ET*)W + (e * K + k) * N + n);
  const uint32_t b = sc[(e * ceil_div(N, kBlock8) + n / kBlock8) * row_scales8(K) + k / kBlock8];
  const int v = ((const uint8_t*)W)[(e * N + n) * row_bytes8(K) + k];
  return __builtin_amdgcn_cvt_f32_fp8(v, 0) * (b == kScaleNaN ? __uint_as_float(0x7fc00000u) : b == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(b << 23));
}

// hidden[t, j, :] of kept choices: 64 columns to a block, a quarter of the sum to a wave
template <typename ET>
__global__ __launch_bounds__(256) void few_up_kernel(const FewTokens p) {
  __shared__ float part[4][64];
  const int pair = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = pair / p.k, e = p.idx[pair], n = (int64_t)blockIdx.x * 64 + lane;
  if (p.loc[pair] >= p.C) return;
  float s = 0.f;
  if (n < p.H)
    for (int64_t k = wave; k < p.M; k += 4) s += load_as_f32((const ET*)p.x + t * p.M + k) * weight_at<ET>(p.W1, p.s1, e, k, n, p.M, p.H);
  part[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || n >= p.H) return;
  s = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
  if (p.b1) s += load_as_f32((const ET*)p.b1 + e * p.H + n);
  store_from_f32((ET*)p.hidden + (int64_t)pair * p.H + n, apply_act(s, p.act));
}

template <typename ET>
__global__ __launch_bounds__(256) void few_down_kernel(const FewTokens p) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = blockIdx.y, n = (int64_t)blockIdx.x * 64 + lane;
  float sum = 0.f;
  for (int j = 0; j < p.k; ++j) {
    const int64_t pair = t * p.k + j, e = p.idx[pair];
    if (p.loc[pair] >= p.C) continue;
    float s = 0.f;
    if (n < p.M)
      for (int64_t k = wave; k < p.H; k += 4) s += load_as_f32((const ET*)p.hidden + pair * p.H + k) * weight_at<ET>(p.W2, p.s2, e, k, n, p.H, p.M);
    part[wave][lane] = s;
    __syncthreads();
    s = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
    if (p.b2 && n < p.M) s += load_as_f32((const ET*)p.b2 + e * p.M + n);
    sum += p.gate_w[pair] * s;
    __syncthreads();
  }
  if (wave == 0 && n < p.M) store_from_f32((ET*)p.out + t * p.M + n, sum);
}

}  // namespace

hipError_t launch_few_tokens(const FewTokens& p, hipStream_t s) {
  const dim3 up((unsigned)ceil_div(p.H, 64), (unsigned)(p.T * p.k)), down((unsigned)ceil_div(p.M, 64), (unsigned)p.T);
  if (p.dtype == MOE_F32) few_up_kernel<float><<<up, dim3(256), 0, s>>>(p);
  else few_up_kernel<uint16_t><<<up, dim3(256), 0, s>>>(p);
  if (hipError_t err = hipGetLastError()) return err;
  if (p.dtype == MOE_F32) few_down_kernel<float><<<down, dim3(256), 0, s>>>(p);
  else few_down_kernel<uint16_t><<<down, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace moe
