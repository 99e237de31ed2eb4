// The grouped GEMM's launches for experts' slabs: which of its kernels a product runs on (rules: ffn_rules.h).
#include "ffn_device.h"

namespace moe {
namespace {

// Branch-free activations for the bf16 epilogue.  gelu(v) = v Phi(v) with Phi(-y) = erfc(y / sqrt 2) / 2 for y = |v|:
// e = 2^-P(y) with a degree-5 polynomial P fitted to -log2 erfc(y / sqrt 2) (weighted least squares on [0, 9] with P(0) = 0;
// |gelu error| < 6e-7 everywhere, three orders below bf16 resolution), then Phi = 1 - e/2 for
// v >= 0 and e/2 for v < 0.  One exponential, no division.
constexpr float kGeluC1 = 1.151000500e+00f, kGeluC2 = 4.595958591e-01f, kGeluC3 = 5.214662850e-02f,
                kGeluC4 = -7.198722102e-03f, kGeluC5 = 4.881033092e-04f;
__device__ __forceinline__ float fast_gelu(float v) {
  const float y = fabsf(v);
  float p = fmaf(kGeluC5, y, kGeluC4);
  p = fmaf(p, y, kGeluC3);
  p = fmaf(p, y, kGeluC2);
  p = fmaf(p, y, kGeluC1);
  const float e = __builtin_amdgcn_exp2f(-(p * y));
  const float d = copysignf(fmaf(-0.5f, e, 0.5f), v);              // Phi(v) - 1/2
  return v * (0.5f + d);
}

// gelu'(v) = Phi(v) + v phi(v) with the same Phi and phi(v) = exp2(-v^2 / (2 ln 2)) / sqrt(2 pi): two exponentials,
// |error| < 3e-6.
constexpr float kHalfLog2e = 0.72134752f, kInvSqrt2Pi = 0.39894228f;
__device__ __forceinline__ float fast_gelu_grad(float v) {
  const float y = fabsf(v);
  float p = fmaf(kGeluC5, y, kGeluC4);
  p = fmaf(p, y, kGeluC3);
  p = fmaf(p, y, kGeluC2);
  p = fmaf(p, y, kGeluC1);
  const float e = __builtin_amdgcn_exp2f(-(p * y));
  const float d = copysignf(fmaf(-0.5f, e, 0.5f), v);              // Phi(v) - 1/2
  const float dens = __builtin_amdgcn_exp2f(-kHalfLog2e * v * v) * kInvSqrt2Pi;
  return fmaf(v, dens, 0.5f + d);
}

// act'(p) for the epilogue that turns dH into dP (bf16 results: relative error far below the output resolution)
template <int ACT> __device__ __forceinline__ float epilogue_act_grad(float p) {
  if (ACT == MOE_ACT_RELU) return p > 0.f ? 1.f : 0.f;
  if (ACT == MOE_ACT_GELU) return fast_gelu_grad(p);
  const float sg = __builtin_amdgcn_rcpf(1.0f + __expf(-p));        // SiLU
  return sg * fmaf(p, 1.f - sg, 1.f);
}

template <int ACT> __device__ __forceinline__ float epilogue_act(float v) {
  if (ACT == MOE_ACT_RELU) return fmaxf(v, 0.f);
  if (ACT == MOE_ACT_GELU) return fast_gelu(v);
  if (ACT == MOE_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.0f + __expf(-v));
  return v;
}

// The activations of bf16 results.  The fit behind epilogue_act is good to 6e-7, which is below a bf16 rounding except where GeLU
// itself is small: at -4 it is off by 0.4 %, twice that rounding, and the erf form by 0.02 %.  Widths the large tile does not
// take have always had the erf form (and true divisions) and keep it, whichever tile they run on; widths it takes keep the fit.
template <int ACT> __device__ __forceinline__ float tile_act(float v) {
  if constexpr (ACT >= kFullAct) return apply_act(v, ACT - kFullAct);
  else return epilogue_act<ACT>(v);
}
template <int ACT> __device__ __forceinline__ float tile_act_grad(float p) {
  if constexpr (ACT >= kFullAct) return apply_act_grad(p, ACT - kFullAct);
  else return epilogue_act_grad<ACT>(p);
}

}  // namespace
}  // namespace moe

#include "ffn_large.h"

namespace moe {

// `half`: on the half tile; `total`: rows of all experts that exist, at most.
static hipError_t launch_large_nn(const void* A, const void* B, const void* bias, int act, const int32_t* counts,
                                  int64_t E, int64_t C, int64_t K, int64_t N, void* out, hipStream_t s, bool half, int64_t total,
                                  int64_t rows_hint, const int32_t* gather, int64_t gather_rows, void* pre_out) {
  const int64_t bm = half ? BM / 2 : BM;
  const int MT = (int)ceil_div(C, bm), NT = (int)(N / BN);
  const bool cut = !half && !far_rows(gather_rows, K) && cuts_last_round(E, C, mean_or(rows_hint, C), counts, NT);
  const int64_t blocks = tile_grid(NT, live_row_tiles(E, C, total, bm), true, cut);
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kThreads);
#define MOE_LAUNCH_GEMM_AT(ACT, DUAL, FAR, CUT)                                                                       \
  grouped_gemm_mfma_kernel<ACT, kNN, false, DUAL, false, FAR, CUT><<<grid, block, 0, s>>>(                                 \
      (const uint16_t*)A, (const uint16_t*)B, (const uint16_t*)bias, counts, gather, (int)gather_rows, (int)E, C,     \
      (int)K, (int)N, MT, NT, (uint16_t*)out, nullptr, nullptr, nullptr, nullptr,                                       \
      (uint16_t*)pre_out)
#define MOE_LAUNCH_GEMM(ACT, DUAL)                                                                                    \
  do {                                                                                                                \
    if (half)                                                                                                         \
      grouped_gemm_half_kernel<ACT><<<grid, block, 0, s>>>((const uint16_t*)A, (const uint16_t*)B, (const uint16_t*)bias, \
                                                           counts, gather, (int)gather_rows, (int)E, C, (int)K, (int)N, MT, NT, (uint16_t*)out); \
    else if (far_rows(gather_rows, K)) MOE_LAUNCH_GEMM_AT(ACT, DUAL, true, false);                                     \
    else if (cut) MOE_LAUNCH_GEMM_AT(ACT, DUAL, false, true);                                                         \
    else MOE_LAUNCH_GEMM_AT(ACT, DUAL, false, false);                                                                 \
  } while (0)
  if (pre_out && act >= 0) {
    switch (act) {
      case MOE_ACT_RELU: MOE_LAUNCH_GEMM(MOE_ACT_RELU, true); break;
      case MOE_ACT_GELU: MOE_LAUNCH_GEMM(MOE_ACT_GELU, true); break;
      default: MOE_LAUNCH_GEMM(MOE_ACT_SILU, true); break;
    }
  } else {
    switch (act) {
      case MOE_ACT_RELU: MOE_LAUNCH_GEMM(MOE_ACT_RELU, false); break;
      case MOE_ACT_GELU: MOE_LAUNCH_GEMM(MOE_ACT_GELU, false); break;
      case MOE_ACT_SILU: MOE_LAUNCH_GEMM(MOE_ACT_SILU, false); break;
      default: MOE_LAUNCH_GEMM(-1, false); break;
    }
  }
#undef MOE_LAUNCH_GEMM
#undef MOE_LAUNCH_GEMM_AT
  return hipGetLastError();
}

// out[e] = A[e] (rows_e x K) * Bt[e]^T, Bt [E, N, K]; with `pre` [E, C, N] the result is multiplied by act'(pre), or,
// with act < 0, has `pre` added (pre == out accumulates in place).
static hipError_t launch_large_nt(const void* A, const void* Bt, const int32_t* counts, int64_t E, int64_t C,
                                  int64_t K, int64_t N, void* out, const void* pre, int act, hipStream_t s, int64_t total, int64_t rows_hint) {
  const int MT = (int)ceil_div(C, BM), NT = (int)(N / BN);
  const bool cut = cuts_last_round(E, C, mean_or(rows_hint, C), counts, NT);
  const int64_t blocks = tile_grid(NT, live_row_tiles(E, C, total, BM), true, cut);
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kThreads);
#define MOE_LAUNCH_GEMM_AT(ACT, GRAD, CUT)                                                                            \
  grouped_gemm_mfma_kernel<ACT, kNT, GRAD, false, false, false, CUT><<<grid, block, 0, s>>>(                          \
      (const uint16_t*)A, (const uint16_t*)Bt, nullptr, counts, nullptr, 0, (int)E, C, (int)K, (int)N, MT, NT,        \
      (uint16_t*)out, nullptr, nullptr, nullptr, (const uint16_t*)pre, nullptr)
#define MOE_LAUNCH_GEMM(ACT, GRAD)                                                                                    \
  do {                                                                                                                \
    if (cut) MOE_LAUNCH_GEMM_AT(ACT, GRAD, true);                                                                     \
    else MOE_LAUNCH_GEMM_AT(ACT, GRAD, false);                                                                        \
  } while (0)
  if (!pre) MOE_LAUNCH_GEMM(-1, false);
  else if (act < 0) MOE_LAUNCH_GEMM(-1, true);                      // out = product + pre
  else switch (act) {
    case MOE_ACT_RELU: MOE_LAUNCH_GEMM(MOE_ACT_RELU, true); break;
    case MOE_ACT_GELU: MOE_LAUNCH_GEMM(MOE_ACT_GELU, true); break;
    default: MOE_LAUNCH_GEMM(MOE_ACT_SILU, true); break;
  }
#undef MOE_LAUNCH_GEMM
#undef MOE_LAUNCH_GEMM_AT
  return hipGetLastError();
}

// out[e] (R x N) = At[e]^T * B[e] over the first min(kfill[e], C) of the C slots; At [E, C, R], B [E, C, N], R and N
// multiples of 256.  a_tail [E, 64, R] and b_tail [E, 64, N] are scratch for the zero-padded last K-step.
// With `gather` [E, C] (slot -> row, as the dispatch builds it) At is one matrix [gather_rows, R] and slot c of expert e
// is its row gather[e, c].
static hipError_t launch_large_tn(const void* At, const void* B, const int32_t* kfill, int64_t E, int64_t C, int64_t R,
                                  int64_t N, void* a_tail, void* b_tail, void* out, hipStream_t s, const int32_t* gather,
                                  int64_t gather_rows) {
  const TailRows ta = {(const uint4*)At, (uint4*)a_tail, gather, gather_rows, (int)(R / 8)}, tb = {(const uint4*)B, (uint4*)b_tail, nullptr, 0, (int)(N / 8)};
  tail_rows_kernel<false><<<dim3(BK / 4, (unsigned)E, 2), dim3(256), 0, s>>>(ta, tb, kfill, C);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const int MT = (int)(R / BM), NT = (int)(N / BN);
  const int64_t blocks = tile_grid(NT, E * MT);
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kThreads);
#define MOE_LAUNCH_GATHERED(FAR)                                                                                        \
  grouped_gemm_mfma_kernel<-1, kTN, false, false, true, FAR><<<grid, block, 0, s>>>(                                    \
      (const uint16_t*)At, (const uint16_t*)B, nullptr, nullptr, gather, (int)gather_rows, (int)E, R, (int)C, (int)N, MT, NT, \
      (uint16_t*)out, kfill, (const uint16_t*)a_tail, (const uint16_t*)b_tail, nullptr, nullptr)
  if (gather && far_rows(gather_rows, R)) MOE_LAUNCH_GATHERED(true);
  else if (gather) MOE_LAUNCH_GATHERED(false);
#undef MOE_LAUNCH_GATHERED
  else
    grouped_gemm_mfma_kernel<-1, kTN, false><<<grid, block, 0, s>>>(
        (const uint16_t*)At, (const uint16_t*)B, nullptr, nullptr, nullptr, 0, (int)E, R, (int)C, (int)N, MT, NT,
        (uint16_t*)out, kfill, (const uint16_t*)a_tail, (const uint16_t*)b_tail, nullptr, nullptr);
  return hipGetLastError();
}

bool grouped_gemm_gathers_on_large_tile(int64_t E, int64_t C, int64_t K, int64_t N, int64_t gather_rows) {
  return large_tile_supports(E, C, K, N, gather_rows) && !far_rows(gather_rows, K);
}

// Rows that exist in all, at most.  Only a caller that counts has a hint that is also a promise.
static int64_t total_rows(const int32_t* counts, int64_t E, int64_t C, int64_t rows_hint) {
  return E * (counts && rows_hint > 0 && rows_hint < C ? rows_hint : C);
}

hipError_t launch_grouped_gemm(const void* A, const void* B, const void* bias, int act, int dtype, const int32_t* counts,
                               int64_t E, int64_t C, int64_t K, int64_t N, void* out, hipStream_t s, int64_t rows_hint,
                               void* pre_out, const int32_t* gather, int64_t gather_rows) {
  if (act < 0) pre_out = nullptr;                                   // nothing to tell apart
  const Tile tile = dtype == MOE_BF16 ? tile_of(kNN, E, C, K, N, rows_hint, gather ? gather_rows : 0, pre_out != nullptr) : Tile::k64;
  const int64_t total = total_rows(counts, E, C, rows_hint);
  if (tile == Tile::k256 || tile == Tile::kHalf)
    return launch_large_nn(A, B, bias, act, counts, E, C, K, N, out, s, tile == Tile::kHalf, total, rows_hint, gather, gather_rows, pre_out);
  if (dtype == MOE_BF16 && act > MOE_ACT_RELU && !large_tile_supports(E, C, K, N, 0)) act += kFullAct;
  const TileArgs p = {A, B, bias, counts, gather, gather_rows, C, K, (int)N, (int)E, 0, 0, 0, out, nullptr, nullptr, pre_out, act, 0};
  return launch_small<kNN>(dtype, tile, p, total, s);
}

// out[e] = A[e] (rows_e x K) * Bt[e]^T, Bt [E, N, K]; with `pre` [E, C, N] the result is multiplied by act'(pre), or,
// with act < 0, has `pre` added (pre == out accumulates in place).
hipError_t launch_grouped_gemm_nt(const void* A, const void* Bt, int dtype, const int32_t* counts, int64_t E, int64_t C,
                                  int64_t K, int64_t N, void* out, const void* pre, int act, hipStream_t s, int64_t rows_hint) {
  const Tile tile = dtype == MOE_BF16 ? tile_of(kNT, E, C, K, N, rows_hint, 0, false) : Tile::k64;
  const int64_t total = total_rows(counts, E, C, rows_hint);
  if (tile == Tile::k256) return launch_large_nt(A, Bt, counts, E, C, K, N, out, pre, act, s, total, rows_hint);
  if (dtype == MOE_BF16 && act > MOE_ACT_RELU && !large_tile_supports_backward(E, C, K, N)) act += kFullAct;
  const TileArgs p = {A, Bt, nullptr, counts, nullptr, 0, C, K, (int)N, (int)E, 0, 0, 0, out, nullptr, pre, nullptr, pre ? act : -1, 0};
  return launch_small<kNT>(dtype, tile, p, total, s);
}

size_t grouped_gemm_tn_tail_bytes(int64_t E, int64_t W) { return (size_t)E * BK * W * 2; }

// out[e] (R x N) = At[e]^T * B[e] over the first min(kfill[e], C) of the C slots; At [E, C, R], B [E, C, N].  a_tail and
// b_tail: scratch of grouped_gemm_tn_tail_bytes(E, R) and (E, N).  With `gather` [E, C] At is one matrix [gather_rows, R] and
// slot c of expert e is its row gather[e, c].
hipError_t launch_grouped_gemm_tn(const void* At, const void* B, int dtype, const int32_t* kfill, int64_t E, int64_t C, int64_t R,
                                  int64_t N, void* a_tail, void* b_tail, void* out, hipStream_t s, int64_t rows_hint,
                                  const int32_t* gather, int64_t gather_rows) {
  const Tile tile = dtype == MOE_BF16 ? tile_of(kTN, E, R, C, N, rows_hint, gather_rows, false) : Tile::k64;
  if (tile == Tile::k256) return launch_large_tn(At, B, kfill, E, C, R, N, a_tail, b_tail, out, s, gather, gather_rows);
  const TileArgs p = {At, B, nullptr, nullptr, gather, gather_rows, R, C, (int)N, (int)E, 0, 0, 0, out, kfill, nullptr, nullptr, -1, 0};
  return launch_small<kTN>(dtype, tile, p, E * R, s);
}

// The reduction of a kTN product with one small result, cut into slices whose sums leave as fp32: see common.h.
template <typename ET, int BM, int BN, int WR, int WC>
static hipError_t launch_slices(TileArgs p, hipStream_t s) {
  p.MT = (int)ceil_div(p.C, BM);
  p.NT = (int)ceil_div(p.N, BN);
  const int64_t blocks = tile_grid(p.NT, (int64_t)p.E * p.MT);
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
  grouped_gemm_tile_kernel<ET, kTN, BM, BN, WR, WC, 2, false, true><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

// Columns of a slice's tile: no more than the results have, as far as a matrix instruction is not narrower still.  (fp32, 65536
// tokens, M = 2048, dWg of 8 experts: 163 us with 64, 106 with 32.)
static int slices_width(int dtype, int64_t N) { return N <= 32 ? 32 : (N <= 64 || dtype == MOE_F32 ? 64 : 128); }
static int slices_height(int dtype, int64_t N) { return dtype == MOE_F32 && N > 32 ? 64 : 128; }

// Enough slices for about four blocks per compute unit, but no more than 64 (their sums are written and read again) and no more
// than one to 256 k; a slice is a whole number of K-steps.
GemmSlices gemm_slices(int dtype, int64_t K, int64_t R, int64_t N) {
  const int64_t tiles = ceil_div(R, slices_height(dtype, N)) * ceil_div(N, slices_width(dtype, N));
  int64_t n = ceil_div(1024, tiles);
  n = n < 64 ? n : 64;
  n = n < ceil_div(K, 256) ? n : ceil_div(K, 256);
  GemmSlices g;
  g.length = ceil_div(ceil_div(K, n), 64) * 64;
  g.count = ceil_div(K, g.length);
  return g;
}

hipError_t launch_gemm_tn_slices(const void* At, const void* B, int dtype, int64_t K, int64_t R, int64_t N, float* out, hipStream_t s) {
  const GemmSlices g = gemm_slices(dtype, K, R, N);
  TileArgs p = {At, B, nullptr, nullptr, nullptr, 0, R, g.length, (int)N, (int)g.count, 0, 0, 0, out, nullptr, nullptr, nullptr, -1, K};
  if (dtype == MOE_F32) return N <= 32 ? launch_slices<float, 128, 32, 4, 1>(p, s) : launch_slices<float, 64, 64, 2, 2>(p, s);
  switch (slices_width(dtype, N)) {
    case 32: return launch_slices<uint16_t, 128, 32, 4, 1>(p, s);
    case 64: return launch_slices<uint16_t, 128, 64, 2, 2>(p, s);
    default: return launch_slices<uint16_t, 128, 128, 2, 2>(p, s);
  }
}

}  // namespace moe
