// C ABI of the operators on experts' rows that lie one behind the other, of the dense product with its epilogue, and of dropout: argument validation, workspace
// layout, sequencing.
#include <cmath>
#include <initializer_list>

#include "api_checks.h"
#include "ffn_rules.h"
#include "rows.h"

namespace moe {
namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxRowWidth = (int64_t)1 << 20;

bool all_aligned(std::initializer_list<const void*> ps, size_t a) {
  for (const void* p : ps)
    if (p && !aligned(p, a)) return false;
  return true;
}

// whether a result would go onto an input, or onto another result
bool clash(std::initializer_list<const void*> results, std::initializer_list<const void*> inputs) {
  for (const void* const* r = results.begin(); r != results.end(); ++r) {
    if (!*r) continue;
    for (const void* const* o = r + 1; o != results.end(); ++o)
      if (*o == *r) return true;
    for (const void* p : inputs)
      if (p == *r) return true;
  }
  return false;
}

bool any_act(int act) { return act == MOE_ACT_NONE || act_ok(act); }
inline int status_of(hipError_t err) { return err == hipSuccess ? MOE_OK : MOE_HIP_ERROR; }

// R rows of E experts through weights K x N; every tile of every form of the product fits a grid
int product_status(int64_t R, int64_t E, int64_t K, int64_t N) {
  if (R < 1 || E < 1) return MOE_INVALID_ARG;
  if (int st = row_shape_status(K)) return st;
  if (int st = row_shape_status(N)) return st;
  if (R >= kMaxRows || E > kMaxExperts || K > kMaxRowWidth || N > kMaxRowWidth || K * N >= ((int64_t)1 << 31)) return MOE_UNSUPPORTED;
  const int64_t wide = K > N ? K : N;
  if ((ceil_div(R, 64) + E) * ceil_div(wide, 64) >= kMaxBlocks / 2 || E * ceil_div(K, 64) * ceil_div(N, 64) >= kMaxBlocks / 2) return MOE_UNSUPPORTED;
  return MOE_OK;
}

struct BackwardWorkspace {
  size_t dp, sums, tails, total;
};

BackwardWorkspace backward_layout(int64_t R, int64_t E, int64_t K, int64_t N, int act, int dtype) {
  BackwardWorkspace w;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return at; };
  w.dp = take(act >= 0 ? (size_t)R * N * esize(dtype) : 0);
  w.sums = take(rows_act_backward_bytes(R, E, N));
  w.tails = take(rows_weight_grad_bytes(dtype, R, E, K, N));
  w.total = off > 0 ? off : 256;                                    // never the size that means a refusal
  return w;
}

// the probability as a number of 2^-16 and the factor of what is kept
bool dropout_of(double p, const uint64_t* seed, Dropout& d) {
  if (!(p >= 0.0 && p <= 1.0)) return false;
  d.seed = seed;
  d.below = (uint32_t)nearbyint(p * 65536.0);
  d.scale = d.below < 65536u ? (float)(65536.0 / (double)(65536u - d.below)) : 0.f;
  return d.below == 0 || seed;
}

int backward(const void* dy, const void* x, const int32_t* gather, int64_t x_rows, const void* W, const void* pre, int act, const void* x_pre, int x_act, int dtype,
             const int32_t* offsets, int64_t R, int64_t E, int64_t K, int64_t N, char* ws, void* dx, void* dW, void* db, hipStream_t s) {
  const BackwardWorkspace w = backward_layout(R, E, K, N, act, dtype);
  void* dp = act >= 0 ? ws + w.dp : nullptr;
  if (act >= 0 || db)
    if (launch_rows_act_backward(dy, pre, act, dtype, offsets, R, E, N, ws + w.sums, dp, db, s) != hipSuccess) return MOE_HIP_ERROR;
  const void* d = act >= 0 ? dp : dy;
  if (dx && launch_rows_product_nt(d, W, x_pre, x_act, dtype, offsets, R, E, K, N, dx, s) != hipSuccess) return MOE_HIP_ERROR;
  if (dW && launch_rows_weight_grad(x, gather, x_rows, d, dtype, offsets, R, E, K, N, ws + w.tails, dW, s) != hipSuccess) return MOE_HIP_ERROR;
  return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

int moe_ragged_rows(const int32_t* idx, const int32_t* loc, const int32_t* counts, int64_t T, int64_t E, int k, int64_t C, int32_t* offsets, int32_t* row_src,
                    int32_t* row_of, void* stream) {
  if (!idx || !loc || !counts || !offsets || !row_src || !row_of || T < 1 || E < 1 || k < 1 || k > E || C < 0) return MOE_INVALID_ARG;
  if (E > kMaxExperts || T * k >= kMaxRows || T >= kMaxRows) return MOE_UNSUPPORTED;
  if (!all_aligned({idx, loc, counts, offsets, row_src, row_of}, 4)) return MOE_UNSUPPORTED;
  if (clash({offsets, row_src, row_of}, {idx, loc, counts})) return MOE_INVALID_ARG;             // blocks write offsets while others add up the counts
  return status_of(launch_ragged_rows(idx, loc, counts, T, E, k, C, offsets, row_src, row_of, (hipStream_t)stream));
}

int moe_ragged_matmul(const void* A, const int32_t* gather, int64_t A_rows, const void* W, const void* bias, int act, int dtype, const int32_t* offsets, int64_t R,
                      int64_t E, int64_t K, int64_t N, void* pre, void* out, void* stream) {
  if (!A || !W || !offsets || !out || !dtype_ok(dtype) || !any_act(act) || (gather && A_rows < 1) || clash({out, pre}, {A, gather, W, bias, offsets}))
    return MOE_INVALID_ARG;
  if (int st = product_status(R, E, K, N)) return st;
  if ((gather && A_rows >= kMaxRows) || !all_aligned({A, W, bias, pre, out}, 16) || !all_aligned({gather, offsets}, 4)) return MOE_UNSUPPORTED;
  const RowsProduct p = {A, W, bias, nullptr, offsets, gather, A_rows, R, E, K, N, act, dtype, out, pre};
  return status_of(launch_rows_product(p, nullptr, (hipStream_t)stream));
}

size_t moe_ragged_matmul_backward_workspace_bytes(int64_t R, int64_t E, int64_t K, int64_t N, int act, int dtype) {
  if (!any_act(act) || !dtype_ok(dtype) || product_status(R, E, K, N) != MOE_OK) return 0;
  return backward_layout(R, E, K, N, act, dtype).total;
}

int moe_ragged_matmul_backward(const void* dy, const void* x, const int32_t* gather, int64_t x_rows, const void* W, const void* pre, int act, const void* x_pre, int x_act,
                               int dtype, const int32_t* offsets, int64_t R, int64_t E, int64_t K, int64_t N, void* ws, size_t ws_bytes, void* dx, void* dW, void* db,
                               void* stream) {
  if (!dy || !offsets || !dtype_ok(dtype) || !any_act(act) || !any_act(x_act) || (act >= 0) != (pre != nullptr) || (x_act >= 0) != (x_pre != nullptr) || (!dx && !dW && !db) ||
      (dx && !W) || (dW && !x) || (gather && x_rows < 1) || !ws || (x_pre && !dx) || clash({dx, dW, db}, {dy, x, gather, W, pre, x_pre, offsets, ws}))
    return MOE_INVALID_ARG;
  if (int st = product_status(R, E, K, N)) return st;
  if ((gather && x_rows >= kMaxRows) || !all_aligned({dy, x, W, pre, x_pre, dx, dW, db}, 16) || !all_aligned({gather, offsets}, 4) || !aligned(ws, 256)) return MOE_UNSUPPORTED;
  if (ws_bytes < backward_layout(R, E, K, N, act, dtype).total) return MOE_WORKSPACE_TOO_SMALL;
  if (clash({ws}, {dy, x, gather, W, pre, x_pre, offsets})) return MOE_INVALID_ARG;
  return backward(dy, x, gather, x_rows, W, pre, act, x_pre, x_act, dtype, offsets, R, E, K, N, (char*)ws, dx, dW, db, (hipStream_t)stream);
}

size_t moe_linear_workspace_bytes(int64_t T, int64_t K, int64_t N, int dtype) {
  return dtype_ok(dtype) && product_status(T, 1, K, N) == MOE_OK ? rows_product_bytes(dtype, T, K, N) : 0;
}

int moe_linear(const void* x, const void* W, const void* bias, int act, const void* residual, int dtype, int64_t T, int64_t K, int64_t N, void* ws, size_t ws_bytes,
               void* pre, void* out, void* stream) {
  if (!x || !W || !out || !dtype_ok(dtype) || !any_act(act) || clash({out, pre}, {x, W, bias}) || (pre && pre == residual)) return MOE_INVALID_ARG;
  if (int st = product_status(T, 1, K, N)) return st;
  const size_t need = rows_product_bytes(dtype, T, K, N);
  if (need > 0 && !ws) return MOE_INVALID_ARG;
  if (!all_aligned({x, W, bias, residual, pre, out}, 16) || !all_aligned({ws}, 256)) return MOE_UNSUPPORTED;
  if (need > ws_bytes) return MOE_WORKSPACE_TOO_SMALL;
  if (need > 0 && clash({ws}, {x, W, bias, residual, pre, out})) return MOE_INVALID_ARG;
  const RowsProduct p = {x, W, bias, residual, nullptr, nullptr, 0, T, 1, K, N, act, dtype, out, pre};
  return status_of(launch_rows_product(p, ws, (hipStream_t)stream));
}

size_t moe_linear_backward_workspace_bytes(int64_t T, int64_t K, int64_t N, int act, int dtype) {
  return moe_ragged_matmul_backward_workspace_bytes(T, 1, K, N, act, dtype);
}

int moe_linear_backward(const void* dy, const void* x, const void* W, const void* pre, int act, int dtype, int64_t T, int64_t K, int64_t N, void* ws, size_t ws_bytes,
                        void* dx, void* dW, void* db, void* stream) {
  if (!dy || !dtype_ok(dtype) || !any_act(act) || (act >= 0) != (pre != nullptr) || (!dx && !dW && !db) || (dx && !W) || (dW && !x) || !ws ||
      clash({dx, dW, db}, {dy, x, W, pre, ws}))
    return MOE_INVALID_ARG;
  if (int st = product_status(T, 1, K, N)) return st;
  if (!all_aligned({dy, x, W, pre, dx, dW, db}, 16) || !aligned(ws, 256)) return MOE_UNSUPPORTED;
  if (ws_bytes < backward_layout(T, 1, K, N, act, dtype).total) return MOE_WORKSPACE_TOO_SMALL;
  if (clash({ws}, {dy, x, W, pre})) return MOE_INVALID_ARG;
  return backward(dy, x, nullptr, 0, W, pre, act, nullptr, -1, dtype, nullptr, T, 1, K, N, (char*)ws, dx, dW, db, (hipStream_t)stream);
}

int moe_dropout(const void* x, const void* residual, double p, const uint64_t* seed, int dtype, int64_t n, void* out, void* stream) {
  Dropout d;
  if (!x || !out || !dtype_ok(dtype) || n < 1 || !dropout_of(p, seed, d) || clash({out}, {seed})) return MOE_INVALID_ARG;
  if (n % 8 != 0 || n >= ((int64_t)1 << 40) || !all_aligned({x, residual, out}, 16) || !all_aligned({seed}, 8)) return MOE_UNSUPPORTED;
  return status_of(launch_dropout(x, residual, d, dtype, n, out, (hipStream_t)stream));
}

static int combine_status(int64_t T, int64_t M, int k, int64_t R) {
  if (T < 1 || k < 1 || R < 1) return MOE_INVALID_ARG;
  if (int st = row_shape_status(M)) return st;
  if (k > kMaxExperts || T >= kMaxRows || T * k >= kMaxRows || R >= kMaxRows || M > kMaxRowWidth || T * ceil_div(M, 512) >= kMaxRows) return MOE_UNSUPPORTED;
  return MOE_OK;
}

int moe_ragged_combine(const void* Y, int64_t R, const int32_t* row_of, const float* gate_w, const void* residual, double p, const uint64_t* seed, int dtype, int64_t T,
                       int64_t M, int k, void* out, void* stream) {
  Dropout d;
  if (!Y || !row_of || !out || !dtype_ok(dtype) || !dropout_of(p, seed, d) || clash({out}, {Y, row_of, gate_w, seed})) return MOE_INVALID_ARG;
  if (int st = combine_status(T, M, k, R)) return st;
  if (!all_aligned({Y, residual, out}, 16) || !all_aligned({seed}, 8) || !all_aligned({row_of, gate_w}, 4)) return MOE_UNSUPPORTED;
  return status_of(launch_ragged_combine(Y, R, row_of, gate_w, residual, d, dtype, T, M, k, out, (hipStream_t)stream));
}

int moe_ragged_combine_backward(const void* d_out, const void* Y, int64_t R, const int32_t* row_of, const float* gate_w, double p, const uint64_t* seed, int dtype,
                                int64_t T, int64_t M, int k, void* dY, float* dgate_w, void* stream) {
  Dropout d;
  if (!d_out || !Y || !row_of || !dY || !dgate_w || !dtype_ok(dtype) || !dropout_of(p, seed, d) || clash({dY, dgate_w}, {d_out, Y, row_of, gate_w, seed})) return MOE_INVALID_ARG;
  if (int st = combine_status(T, M, k, R)) return st;
  if (!all_aligned({d_out, Y, dY}, 16) || !all_aligned({seed}, 8) || !all_aligned({row_of, gate_w, dgate_w}, 4)) return MOE_UNSUPPORTED;
  return status_of(launch_ragged_combine_backward(d_out, Y, R, row_of, gate_w, d, dtype, T, M, k, dY, dgate_w, (hipStream_t)stream));
}

}  // extern "C"
