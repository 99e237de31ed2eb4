// Matrix products of experts' rows that lie one behind the other, as a router that drops nothing leaves them (and, with one expert, of any rows):
//   y[r] = act(x[src r] W[e] + b[e]) + residual[r],   dx[r] = d[r] W[e]^T (* act'(x_pre[r])),   dW[e] = sum_r x[src r]^T d[r].
// The kernels are those of the experts' slabs (ffn_large.h, ffn_ring.h, ffn_tile.h) with ROWS: a block finds its tile in the offsets on the device, so that
// the host needs nothing but a bound of the rows.  2 R K N operations against one read of x, W and one write of y: bound by the matrix cores, at few rows by W.
#include "ffn_device.h"
#include "rows.h"
#include "rows_act.h"
#include "rows_rules.h"

namespace moe {
namespace {

// What the slabs' epilogues are written with; ROWS does not come by them.
template <int ACT> __device__ __forceinline__ float epilogue_act(float v) { return rows_act<ACT>(v); }
template <int ACT> __device__ __forceinline__ float epilogue_act_grad(float v) { return rows_act_grad<ACT>(v); }
template <int ACT> __device__ __forceinline__ float tile_act(float v) { return rows_act<ACT>(v); }
template <int ACT> __device__ __forceinline__ float tile_act_grad(float v) { return rows_act_grad<ACT>(v); }

}  // namespace
}  // namespace moe

#include "ffn_large.h"

namespace moe {

#include "rows_thin.h"
#include "rows_fp32.h"
#include "rows_outer.h"
#include "rows_short.h"

namespace {

// The products on tiles below the large one.
template <int MODE> hipError_t launch_small_rows(int dtype, const RowsPlan& plan, const TileArgs& t, int64_t total, hipStream_t s) {
  if constexpr (MODE != kTN) {
    if (plan.kernel == RowsKernel::kShort) return launch_short<MODE>(t, total, s);
    if (plan.kernel == RowsKernel::kFp32Split) return launch_tile<float, MODE, kSplitTile, kSplitTile, 2, false, kSplitParts, true>(t, total, s);
  }
  if (dtype == MOE_F32) return launch_rows_fp32<MODE>(t, total, s);
  return launch_small<MODE, true>(dtype, plan.tile, t, total, s);
}
bool is_large(const RowsPlan& plan) { return plan.kernel == RowsKernel::kTile && plan.tile == Tile::k256; }

}  // namespace

size_t rows_product_bytes(int dtype, int64_t R, int64_t K, int64_t N) {
  if (dtype != MOE_BF16) return 0;
  const ThinPlan plan = thin_plan(false, 1, R, K, N);
  return plan.parts > 1 ? (size_t)plan.parts * R * N * 4 : 0;
}

hipError_t launch_rows_product(const RowsProduct& p, void* ws, hipStream_t s) {
  const bool dual = p.pre && p.act >= 0;
  const TileArgs t = {p.A, p.W, p.bias, p.offsets, p.gather, p.gather_rows, p.R, p.K, (int)p.N, (int)p.E, 0, 0, 0, p.out, nullptr, p.residual, p.pre, p.act, 0};
  const RowsPlan plan = product_plan(p.dtype == MOE_BF16, p.offsets != nullptr, p.E, p.R, p.K, p.N, p.gather ? p.gather_rows : 0, p.act >= 0, p.residual || p.pre);
  if (plan.kernel == RowsKernel::kThin) return launch_thin(t, plan, (float*)ws, s);
  if (!is_large(plan)) return launch_small_rows<kNN>(p.dtype, plan, t, p.R, s);
  const int MT = (int)ceil_div(p.R, BM), NT = (int)(p.N / BN);
  const int64_t blocks = tile_grid(NT, live_row_tiles(p.E, p.R, p.R, BM), true, false);
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
#define MOE_LAUNCH_ROWS(ACT, DUAL)                                                                                                                          \
  grouped_gemm_mfma_kernel<ACT, kNN, false, DUAL, false, false, false, true><<<dim3((unsigned)blocks), dim3(kThreads), 0, s>>>(                              \
      (const uint16_t*)p.A, (const uint16_t*)p.W, (const uint16_t*)p.bias, p.offsets, p.gather, (int)p.gather_rows, (int)p.E, p.R, (int)p.K, (int)p.N, MT, NT, \
      (uint16_t*)p.out, nullptr, nullptr, nullptr, (const uint16_t*)p.residual, (uint16_t*)p.pre)
#define MOE_LAUNCH_ROWS_ACT(ACT)            \
  do {                                      \
    if (dual) MOE_LAUNCH_ROWS(ACT, true);   \
    else MOE_LAUNCH_ROWS(ACT, false);       \
  } while (0)
  switch (p.act) {
    case MOE_ACT_RELU: MOE_LAUNCH_ROWS_ACT(MOE_ACT_RELU); break;
    case MOE_ACT_GELU: MOE_LAUNCH_ROWS_ACT(MOE_ACT_GELU); break;
    case MOE_ACT_SILU: MOE_LAUNCH_ROWS_ACT(MOE_ACT_SILU); break;
    default:
      if (p.pre) MOE_LAUNCH_ROWS(-1, true);
      else MOE_LAUNCH_ROWS(-1, false);
  }
#undef MOE_LAUNCH_ROWS_ACT
#undef MOE_LAUNCH_ROWS
  return hipGetLastError();
}

hipError_t launch_rows_product_nt(const void* d, const void* W, const void* x_pre, int x_act, int dtype, const int32_t* offsets, int64_t R, int64_t E, int64_t K,
                                  int64_t N, void* dx, hipStream_t s) {
  if (x_act < 0) x_pre = nullptr;
  const TileArgs t = {d, W, nullptr, offsets, nullptr, 0, R, N, (int)K, (int)E, 0, 0, 0, dx, nullptr, x_pre, nullptr, x_pre ? x_act : -1, 0};
  const RowsPlan plan = product_nt_plan(dtype == MOE_BF16, E, R, K, N, x_pre != nullptr);
  if (!is_large(plan)) return launch_small_rows<kNT>(dtype, plan, t, R, s);
  const int MT = (int)ceil_div(R, BM), NT = (int)(K / BN);
  const int64_t blocks = tile_grid(NT, live_row_tiles(E, R, R, BM), true, false);
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
#define MOE_LAUNCH_ROWS(ACT, GRAD)                                                                                                                 \
  grouped_gemm_mfma_kernel<ACT, kNT, GRAD, false, false, false, false, true><<<dim3((unsigned)blocks), dim3(kThreads), 0, s>>>(                     \
      (const uint16_t*)d, (const uint16_t*)W, nullptr, offsets, nullptr, 0, (int)E, R, (int)N, (int)K, MT, NT, (uint16_t*)dx, nullptr, nullptr, nullptr, \
      (const uint16_t*)x_pre, nullptr)
  if (!x_pre) MOE_LAUNCH_ROWS(-1, false);
  else switch (x_act) {
    case MOE_ACT_RELU: MOE_LAUNCH_ROWS(MOE_ACT_RELU, true); break;
    case MOE_ACT_GELU: MOE_LAUNCH_ROWS(MOE_ACT_GELU, true); break;
    default: MOE_LAUNCH_ROWS(MOE_ACT_SILU, true); break;
  }
#undef MOE_LAUNCH_ROWS
  return hipGetLastError();
}

// Sums of the blocks that share a tile; or the large tile's last K-step of 64 rows, which comes from side buffers of both operands.  Enough whether rows are gathered or not.
size_t rows_weight_grad_bytes(int dtype, int64_t R, int64_t E, int64_t K, int64_t N) {
  const RowsPlan in_place = weight_grad_plan(dtype == MOE_BF16, E, R, K, N, 0);
  if (in_place.parts > 1) return (size_t)in_place.parts * E * K * N * 4;
  if (!is_large(in_place) && !is_large(weight_grad_plan(dtype == MOE_BF16, E, R, K, N, 1))) return 0;
  return grouped_gemm_tn_tail_bytes(E, K) + grouped_gemm_tn_tail_bytes(E, N);
}

hipError_t launch_rows_weight_grad(const void* A, const int32_t* gather, int64_t gather_rows, const void* d, int dtype, const int32_t* offsets, int64_t R, int64_t E,
                                   int64_t K, int64_t N, void* ws, void* dW, hipStream_t s) {
  const RowsPlan plan = weight_grad_plan(dtype == MOE_BF16, E, R, K, N, gather ? gather_rows : 0);
  TileArgs t = {A, d, nullptr, nullptr, gather, gather_rows, K, R, (int)N, (int)E, 0, 0, 0, dW, offsets, nullptr, nullptr, -1, 0};
  if (plan.parts > 1) {
    t.parts = plan.parts;
    t.part_sums = (float*)ws;
    if (hipError_t err = launch_small_rows<kTN>(dtype, plan, t, E * K, s)) return err;
    return join_parts(t, dtype, s);
  }
  if (plan.kernel == RowsKernel::kOuter) return launch_outer(t, E * K, s);
  if (!is_large(plan)) return launch_small_rows<kTN>(dtype, plan, t, E * K, s);
  uint16_t* a_tail = (uint16_t*)ws;
  uint16_t* b_tail = a_tail + grouped_gemm_tn_tail_bytes(E, K) / 2;
  const TailRows ta = {(const uint4*)A, (uint4*)a_tail, gather, gather_rows, (int)(K / 8)}, tb = {(const uint4*)d, (uint4*)b_tail, nullptr, 0, (int)(N / 8)};
  tail_rows_kernel<true><<<dim3(BK / 4, (unsigned)E, 2), dim3(256), 0, s>>>(ta, tb, offsets, R);
  if (hipError_t err = hipGetLastError()) return err;
  const int MT = (int)(K / BM), NT = (int)(N / BN);
  const int64_t blocks = tile_grid(NT, E * MT);
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
#define MOE_LAUNCH_ROWS(GATHERED)                                                                                                                  \
  grouped_gemm_mfma_kernel<-1, kTN, false, false, GATHERED, false, false, true><<<dim3((unsigned)blocks), dim3(kThreads), 0, s>>>(                  \
      (const uint16_t*)A, (const uint16_t*)d, nullptr, nullptr, gather, (int)gather_rows, (int)E, K, (int)R, (int)N, MT, NT, (uint16_t*)dW, offsets, \
      a_tail, b_tail, nullptr, nullptr)
  if (gather) MOE_LAUNCH_ROWS(true);
  else MOE_LAUNCH_ROWS(false);
#undef MOE_LAUNCH_ROWS
  return hipGetLastError();
}

}  // namespace moe
