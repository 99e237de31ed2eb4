// Operators on experts' rows that lie one behind the other (no slabs, no capacity): launchers, arguments already validated.
// offsets [E + 1] (device): expert e's rows are offsets[e] up to offsets[e + 1] of R; null: one expert, all R rows.
#pragma once
#include "common.h"

namespace moe {

// out[r] = act(A[gather[r]] W[e] + bias[e]) + residual[r], before the activation to `pre` as well; any of gather, bias, residual, pre may be null.
struct RowsProduct {
  const void *A, *W, *bias, *residual;
  const int32_t *offsets, *gather;
  int64_t gather_rows, R, E, K, N;
  int act, dtype;
  void *out, *pre;
};
// ws: rows_product_bytes where there are no offsets, else none
size_t rows_product_bytes(int dtype, int64_t R, int64_t K, int64_t N);
hipError_t launch_rows_product(const RowsProduct& p, void* ws, hipStream_t s);
// dx[r] = d[r] W[e]^T, times act'(x_pre[r]) if that is given; d [R,N], W [E,K,N], dx [R,K]
hipError_t launch_rows_product_nt(const void* d, const void* W, const void* x_pre, int x_act, int dtype, const int32_t* offsets, int64_t R, int64_t E, int64_t K,
                                  int64_t N, void* dx, hipStream_t s);
// dW[e] = sum over its rows of A[gather[r]]^T d[r]; ws: rows_weight_grad_bytes
size_t rows_weight_grad_bytes(int dtype, int64_t R, int64_t E, int64_t K, int64_t N);
hipError_t launch_rows_weight_grad(const void* A, const int32_t* gather, int64_t gather_rows, const void* d, int dtype, const int32_t* offsets, int64_t R, int64_t E,
                                   int64_t K, int64_t N, void* ws, void* dW, hipStream_t s);

// dp[r] = dy[r] * act'(pre[r]) (act >= 0; else dp is dy and not written) and db[e] = the sum over its rows of dp; either may be null.
// ws: rows_act_backward_bytes
size_t rows_act_backward_bytes(int64_t R, int64_t E, int64_t N);
hipError_t launch_rows_act_backward(const void* dy, const void* pre, int act, int dtype, const int32_t* offsets, int64_t R, int64_t E, int64_t N, void* ws, void* dp,
                                    void* db, hipStream_t s);

hipError_t launch_ragged_rows(const int32_t* idx, const int32_t* loc, const int32_t* counts, int64_t T, int64_t E, int k, int64_t C, int32_t* offsets, int32_t* row_src,
                              int32_t* row_of, hipStream_t s);

// What is dropped: elements whose 16 bits are below `below`; the others are multiplied by `scale`.  below = 0: nothing.
struct Dropout {
  const uint64_t* seed;
  uint32_t below;
  float scale;
};
hipError_t launch_dropout(const void* x, const void* residual, const Dropout& d, int dtype, int64_t n, void* out, hipStream_t s);
hipError_t launch_ragged_combine(const void* Y, int64_t R, const int32_t* row_of, const float* gate_w, const void* residual, const Dropout& d, int dtype, int64_t T,
                                 int64_t M, int k, void* out, hipStream_t s);
hipError_t launch_ragged_combine_backward(const void* d_out, const void* Y, int64_t R, const int32_t* row_of, const float* gate_w, const Dropout& d, int dtype, int64_t T,
                                          int64_t M, int k, void* dY, float* dgate_w, hipStream_t s);

}  // namespace moe
