// C ABI of the norm, the 8-bit matrices and the layers on them, and the layer for a few tokens: argument validation, workspace
// layout, stage sequencing.
#include <initializer_list>

#include "api_checks.h"
#include "block8.h"

namespace moe {
namespace {

constexpr int64_t kNormMaxWidth = 16384, kNormMaxRows = (int64_t)1 << 22;
constexpr int64_t kFewMaxWidth = (int64_t)1 << 22;
constexpr int64_t kMaxGrid = (int64_t)1 << 24;                      // blocks of 256 threads in a grid dimension

int norm_shape_status(int64_t T, int64_t M) {
  if (T < 1) return MOE_INVALID_ARG;
  if (int st = row_shape_status(M)) return st;
  return M > kNormMaxWidth || T >= kNormMaxRows ? MOE_UNSUPPORTED : MOE_OK;
}

// E matrices [R, K] whose rows, or columns, are kept in 8 bits
int matrix8_status(int64_t E, int64_t R, int64_t K) {
  if (E < 1 || E > 65535 || R < 1 || R > kMaxDim) return MOE_INVALID_ARG;
  if (int st = row_shape_status(K)) return st;
  return ceil_div(R, kBlock8) * ceil_div(K, kBlock8) >= kMaxGrid ? MOE_UNSUPPORTED : MOE_OK;
}

// a product's weights [E, N, K]: an expert's fit 32-bit offsets.  K is padded to whole blocks and may be anything.
int weights8_status(int64_t K, int64_t N) {
  if (K < 1 || K > kMaxDim) return MOE_INVALID_ARG;
  if (int st = row_shape_status(N)) return st;
  return N * row_bytes8(K) >= (int64_t)1 << 32 ? MOE_UNSUPPORTED : MOE_OK;
}

bool all_aligned16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (p && !aligned(p, 16)) return false;
  return true;
}

struct Layer8Workspace {
  size_t logits, idx, loc, gate_w, counts, slot_src, gate_ws, hidden, hidden_scales, Y, total;
};

Layer8Workspace layer8_layout(int64_t T, int64_t M, int64_t H, int64_t E, int k, int64_t C, int dtype) {
  Layer8Workspace w;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return at; };
  w.logits = take((size_t)T * E * 4);
  w.idx = take((size_t)T * k * 4);
  w.loc = take((size_t)T * k * 4);
  w.gate_w = take((size_t)T * k * 4);
  w.counts = take((size_t)E * 4);
  w.slot_src = take((size_t)E * C * 4);
  w.gate_ws = take(moe_gate_route_workspace_bytes(T, M, E, k, dtype));
  w.hidden = take((size_t)E * C * row_bytes8(H));
  w.hidden_scales = take((size_t)E * C * row_scales8(H));
  w.Y = take((size_t)E * C * M * esize(dtype));
  w.total = off;
  return w;
}

struct FewWorkspace {
  size_t logits, idx, loc, gate_w, counts, logit_parts, plan, hidden, partial, arrived, total;
};

FewWorkspace few_layout(int64_t T, int64_t M, int64_t H, int64_t E, int k, int dtype) {
  FewWorkspace w;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return at; };
  w.logits = take((size_t)T * E * 4);
  w.idx = take((size_t)T * k * 4);
  w.loc = take((size_t)T * k * 4);
  w.gate_w = take((size_t)T * k * 4);
  w.counts = take((size_t)E * 4);
  w.logit_parts = take(few_logit_bytes(T, M, E));
  w.plan = take((size_t)(E < T * k ? E : T * k) * kFewPlan * 4);
  w.hidden = take((size_t)T * k * H * esize(dtype));
  w.partial = take(few_partial_bytes(T, M, H, E, k));
  w.arrived = take(few_arrivals_bytes(M));
  w.total = off;
  return w;
}

// a layer of few tokens: offsets inside a step of a weight matrix, and inside an expert's 8-bit weights, fit 32 bits
int few_shape_status(int64_t M, int64_t H, bool weights8) {
  if (M > kFewMaxWidth || H > kFewMaxWidth) return MOE_UNSUPPORTED;
  if (!weights8) return MOE_OK;
  if (int st = weights8_status(M, H)) return st;
  return weights8_status(H, M);
}

int layer_shape_status(int64_t T, int64_t M, int64_t H, int64_t E, int k, int dtype) {
  if (!dtype_ok(dtype)) return MOE_INVALID_ARG;
  if (int st = gate_shape_status(T, E, k)) return st;
  if (int st = row_shape_status(M)) return st;
  return row_shape_status(H);
}

// A projection's training pass: what the forward keeps (x transposed, W as it is), behind it what one call needs for itself (forward: x, W transposed; backward: dy in both
// forms), and at the end the fills that the forward saw.
struct Linear8State {
  size_t xt, xt_scales, W, W_scales, x, x_scales, Wt, Wt_scales, dy, dy_scales, dyt, dyt_scales, fills, total;
};

Linear8State linear8_layout(int64_t E, int64_t C, int64_t K, int64_t N) {
  Linear8State w;
  size_t off = 0;
  auto rows = [&](size_t& q, size_t& scales, int64_t R, int64_t width, bool blocks) {
    q = off;
    off = align_up(off + (size_t)E * R * row_bytes8(width), 256);
    scales = off;
    off = align_up(off + (size_t)E * (blocks ? ceil_div(R, kBlock8) : R) * row_scales8(width), 256);
  };
  rows(w.xt, w.xt_scales, K, C, false);
  rows(w.W, w.W_scales, K, N, true);
  const size_t kept = off;
  rows(w.x, w.x_scales, C, K, false);
  rows(w.Wt, w.Wt_scales, N, K, true);
  w.fills = off;
  off = kept;
  rows(w.dy, w.dy_scales, C, N, false);
  rows(w.dyt, w.dyt_scales, N, C, false);
  w.fills = off > w.fills ? off : w.fills;
  w.total = w.fills + (size_t)E * 4;
  return w;
}

int linear8_status(int64_t E, int64_t C, int64_t K, int64_t N) {
  for (int st : {matrix8_status(E, C, K), matrix8_status(E, K, N), matrix8_status(E, C, N), weights8_status(K, N), weights8_status(N, K), weights8_status(C, N)})
    if (st) return st;
  return MOE_OK;
}

// The two products of the experts' layer; the first one's rows are gathered from x8 if slot_src is given.
// Two roundings between its sums, both of them choices: the activations to 8 bits, without which the second product could not be one of 8-bit matrices, and Y to the storage type, which is
// what the caller of moe_expert_ffn8 gets and what the combine reads: in fp32 it would be twice as much of what bounds that (32768 tokens, top-8, 4096 wide: 2.1 GB, 400 us, in
// bf16).  The layer is 2.5e-3 from the exact result with them, where one rounding to bf16 is 1.7e-3.
hipError_t run_ffn8(const void* x8, const uint8_t* xs, const int32_t* slot_src, int64_t T, const void* W1, const uint8_t* s1, const void* b1,
                    const void* W2, const uint8_t* s2, const void* b2, int act, int dtype, const int32_t* counts, int64_t E, int64_t C,
                    int64_t M, int64_t H, int64_t rows_hint, void* hidden, uint8_t* hidden_scales, void* Y, hipStream_t s) {
  const Matmul8 up = {x8, xs, W1, s1, 1, b1, act, counts, nullptr, slot_src, T, E, C, M, H, rows_hint, dtype, nullptr, hidden, hidden_scales};
  if (hipError_t err = launch_matmul8(up, s)) return err;
  const Matmul8 down = {hidden, hidden_scales, W2, s2, 1, b2, -1, counts, nullptr, nullptr, 0, E, C, H, M, rows_hint, dtype, Y, nullptr, nullptr};
  return launch_matmul8(down, s);
}

inline int status_of(hipError_t err) { return err == hipSuccess ? MOE_OK : MOE_HIP_ERROR; }

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" {

int moe_rms_norm(const void* x, const void* residual, const void* weight, double eps, int dtype, int64_t T, int64_t M, void* h, void* y,
                 void* q, uint8_t* q_scales, void* stream) {
  if (!x || !dtype_ok(dtype) || !((float)eps > 0.f) || (!y && !q) || (!q) != (!q_scales) || (residual && !h)) return MOE_INVALID_ARG;
  if (int st = norm_shape_status(T, M)) return st;
  if (!all_aligned16({x, residual, weight, h, y, q})) return MOE_UNSUPPORTED;
  return status_of(launch_rms_norm(x, residual, weight, (float)eps, dtype, T, M, h, y, q, q_scales, (hipStream_t)stream));
}

size_t moe_rms_norm_backward_workspace_bytes(int64_t T, int64_t M) {
  return norm_shape_status(T, M) == MOE_OK ? rms_norm_backward_workspace_bytes(T, M) : 0;
}

int moe_rms_norm_backward(const void* dy, const void* dh, const void* h, const void* weight, double eps, int dtype, int64_t T, int64_t M,
                          void* ws, size_t ws_bytes, void* dx, void* dweight, void* stream) {
  if (!dy || !h || !dx || !dtype_ok(dtype) || !((float)eps > 0.f) || (dweight && !ws)) return MOE_INVALID_ARG;
  if (int st = norm_shape_status(T, M)) return st;
  if (!all_aligned16({dy, dh, h, weight, dx}) || (dweight && !aligned(ws, 256))) return MOE_UNSUPPORTED;
  if (dweight && ws_bytes < rms_norm_backward_workspace_bytes(T, M)) return MOE_WORKSPACE_TOO_SMALL;
  return status_of(launch_rms_norm_backward(dy, dh, h, weight, (float)eps, dtype, T, M, (float*)ws, dx, dweight, (hipStream_t)stream));
}

int64_t moe_row_bytes8(int64_t K) { return K < 1 || K > kMaxDim ? -1 : row_bytes8(K); }
int64_t moe_row_scales8(int64_t K) { return K < 1 || K > kMaxDim ? -1 : row_scales8(K); }

int moe_quantize8(const void* src, int dtype, const int32_t* counts, int64_t E, int64_t R, int64_t K, int scale_mode, void* q, uint8_t* scales,
                  void* qt, uint8_t* scales_t, void* stream) {
  if (!src || !dtype_ok(dtype) || (scale_mode != MOE_SCALE_ROWS && scale_mode != MOE_SCALE_BLOCKS) || (!q && !qt) || (!q) != (!scales) ||
      (!qt) != (!scales_t))
    return MOE_INVALID_ARG;
  if (int st = matrix8_status(E, R, K)) return st;
  if (!all_aligned16({src, q, qt})) return MOE_UNSUPPORTED;
  return status_of(launch_quantize8(src, dtype, counts, E, R, K, scale_mode == MOE_SCALE_BLOCKS, q, scales, qt, scales_t, (hipStream_t)stream));
}

int moe_dequantize8(const void* q, const uint8_t* scales, int scale_mode, int64_t E, int64_t R, int64_t K, int dtype, void* out, void* stream) {
  if (!q || !scales || !out || !dtype_ok(dtype) || (scale_mode != MOE_SCALE_ROWS && scale_mode != MOE_SCALE_BLOCKS)) return MOE_INVALID_ARG;
  if (int st = matrix8_status(E, R, K)) return st;
  if (ceil_div(E * R * ceil_div(K, 16), 256) >= kMaxGrid || !all_aligned16({q, out})) return MOE_UNSUPPORTED;
  return status_of(launch_dequantize8(q, scales, scale_mode == MOE_SCALE_BLOCKS, E, R, K, dtype, out, (hipStream_t)stream));
}

int moe_matmul8(const void* A, const uint8_t* A_scales, const void* B, const uint8_t* B_scales, int B_scale_mode, const void* bias, int act,
                int dtype, const int32_t* counts, const int32_t* k_counts, const int32_t* gather, int64_t gather_rows, int64_t E, int64_t C,
                int64_t K, int64_t N, void* out, void* out8, uint8_t* out8_scales, void* stream) {
  if (!A || !A_scales || !B || !B_scales || !dtype_ok(dtype) || (act != MOE_ACT_NONE && !act_ok(act)) || E < 1 || E > 65535 || C < 1 || C > kMaxDim ||
      (B_scale_mode != MOE_SCALE_ROWS && B_scale_mode != MOE_SCALE_BLOCKS) || (!out) == (!out8) || (!out8) != (!out8_scales) ||
      (gather && (gather_rows < 1 || gather_rows > kMaxDim)))
    return MOE_INVALID_ARG;
  if (int st = weights8_status(K, N)) return st;
  if (!all_aligned16({A, B, out, out8}) || !aligned(A_scales, 4) || !aligned(B_scales, 4) || (bias && !aligned(bias, 16))) return MOE_UNSUPPORTED;
  const Matmul8 p = {A, A_scales, B, B_scales, B_scale_mode == MOE_SCALE_BLOCKS, bias, act, counts, k_counts, gather, gather_rows, E, C, K, N, 0, dtype,
                     out, out8, out8_scales};
  return status_of(launch_matmul8(p, (hipStream_t)stream));
}

int moe_expert_ffn8(const void* x8, const uint8_t* x_scales, const int32_t* slot_src, int64_t T, const void* W1, const uint8_t* s1, const void* b1,
                    const void* W2, const uint8_t* s2, const void* b2, int act, int dtype, const int32_t* counts, int64_t E, int64_t C, int64_t M,
                    int64_t H, void* hidden8, uint8_t* hidden_scales, void* Y, void* stream) {
  if (!x8 || !x_scales || !W1 || !s1 || !W2 || !s2 || !hidden8 || !hidden_scales || !Y || !dtype_ok(dtype) || !act_ok(act) || E < 1 || E > 65535 ||
      C < 1 || C > kMaxDim || (slot_src && (T < 1 || T > kMaxDim)))
    return MOE_INVALID_ARG;
  if (int st = weights8_status(M, H)) return st;
  if (int st = weights8_status(H, M)) return st;
  if (!all_aligned16({x8, W1, b1, W2, b2, hidden8, Y}) || !aligned(x_scales, 4) || !aligned(s1, 4) || !aligned(s2, 4) || !aligned(hidden_scales, 4))
    return MOE_UNSUPPORTED;
  return status_of(run_ffn8(x8, x_scales, slot_src, T, W1, s1, b1, W2, s2, b2, act, dtype, counts, E, C, M, H, 0, hidden8, hidden_scales, Y,
                            (hipStream_t)stream));
}

size_t moe_expert_linear8_state_bytes(int64_t E, int64_t C, int64_t K, int64_t N) {
  return linear8_status(E, C, K, N) == MOE_OK ? linear8_layout(E, C, K, N).total : 0;
}

int moe_expert_linear8_train(const void* x, const void* W, int dtype, const int32_t* counts, int64_t E, int64_t C, int64_t K, int64_t N, void* y, void* state,
                             size_t state_bytes, void* stream) {
  if (!x || !W || !y || !state || !dtype_ok(dtype)) return MOE_INVALID_ARG;
  if (int st = linear8_status(E, C, K, N)) return st;
  if (!all_aligned16({x, W, y}) || !aligned(state, 256)) return MOE_UNSUPPORTED;
  const Linear8State w = linear8_layout(E, C, K, N);
  if (state_bytes < w.total) return MOE_WORKSPACE_TOO_SMALL;
  uint8_t* b = (uint8_t*)state;
  const hipStream_t s = (hipStream_t)stream;
  if (launch_quantize8(x, dtype, counts, E, C, K, false, b + w.x, b + w.x_scales, b + w.xt, b + w.xt_scales, s, counts ? (int32_t*)(b + w.fills) : nullptr,
                       counts ? y : nullptr, N) != hipSuccess ||
      launch_quantize8(W, dtype, nullptr, E, K, N, true, b + w.W, b + w.W_scales, b + w.Wt, b + w.Wt_scales, s) != hipSuccess)
    return MOE_HIP_ERROR;
  const Matmul8 p = {b + w.x, b + w.x_scales, b + w.Wt, b + w.Wt_scales, 1, nullptr, MOE_ACT_NONE, counts, nullptr, nullptr, 0, E, C, K, N, 0, dtype, y, nullptr, nullptr};
  return status_of(launch_matmul8(p, s));
}

int moe_expert_linear8_backward(const void* dy, int dtype, const int32_t* counts, int64_t E, int64_t C, int64_t K, int64_t N, void* state, size_t state_bytes,
                                void* dx, void* dW, void* stream) {
  if (!dy || !state || (!dx && !dW) || !dtype_ok(dtype)) return MOE_INVALID_ARG;
  if (int st = linear8_status(E, C, K, N)) return st;
  if (!all_aligned16({dy, dx, dW}) || !aligned(state, 256)) return MOE_UNSUPPORTED;
  const Linear8State w = linear8_layout(E, C, K, N);
  if (state_bytes < w.total) return MOE_WORKSPACE_TOO_SMALL;
  uint8_t* b = (uint8_t*)state;
  const hipStream_t s = (hipStream_t)stream;
  // The forward's fills, not what the caller's counts hold by now: of the transposed x only their blocks were written.  (Without counts the products need no loads of them: 1 % of 8 experts
  // x 4096 rows, 2048 x 2048.)
  if (counts) counts = (const int32_t*)(b + w.fills);
  if (launch_quantize8(dy, dtype, counts, E, C, N, false, dx ? b + w.dy : nullptr, dx ? b + w.dy_scales : nullptr, dW ? b + w.dyt : nullptr,
                       dW ? b + w.dyt_scales : nullptr, s, nullptr, counts ? dx : nullptr, K) != hipSuccess)
    return MOE_HIP_ERROR;
  const Matmul8 px = {b + w.dy, b + w.dy_scales, b + w.W, b + w.W_scales, 1, nullptr, MOE_ACT_NONE, counts, nullptr, nullptr, 0, E, C, N, K, 0, dtype, dx, nullptr, nullptr};
  if (dx && launch_matmul8(px, s) != hipSuccess) return MOE_HIP_ERROR;
  const Matmul8 pw = {b + w.xt, b + w.xt_scales, b + w.dyt, b + w.dyt_scales, 0, nullptr, MOE_ACT_NONE, nullptr, counts, nullptr, 0, E, K, C, N, 0, dtype, dW, nullptr, nullptr};
  return dW ? status_of(launch_matmul8(pw, s)) : MOE_OK;
}

size_t moe_layer8_workspace_bytes(int64_t T, int64_t M, int64_t H, int64_t E, int k, int64_t C, int dtype) {
  if (layer_shape_status(T, M, H, E, k, dtype) != MOE_OK || weights8_status(M, H) != MOE_OK || weights8_status(H, M) != MOE_OK || C < 1 || C > kMaxDim)
    return 0;
  return layer8_layout(T, M, H, E, k, C, dtype).total;
}

int moe_layer_forward8(const void* x, const void* x8, const uint8_t* x_scales, const void* Wg, const float* gate_bias, const void* W1,
                       const uint8_t* s1, const void* b1, const void* W2, const uint8_t* s2, const void* b2, int64_t T, int64_t M, int64_t H,
                       int64_t E, int k, double f, int normalize, int act, int dtype, void* out, int32_t* idx, int32_t* loc, float* gate_w,
                       int32_t* counts, float* logits, void* ws, size_t ws_bytes, void* stream) {
  if (!x || !x8 || !x_scales || !Wg || !W1 || !s1 || !W2 || !s2 || !out || !ws || !act_ok(act) || !(f > 0.0)) return MOE_INVALID_ARG;
  if (int st = layer_shape_status(T, M, H, E, k, dtype)) return st;
  if (int st = weights8_status(M, H)) return st;
  if (int st = weights8_status(H, M)) return st;
  const int64_t C = moe_capacity(T, E, k, f);
  if (C < 1 || C > kMaxDim) return MOE_INVALID_ARG;
  if (!all_aligned16({x, x8, W1, b1, W2, b2, out, logits}) || !aligned(ws, 256) || !aligned(x_scales, 4) || !aligned(s1, 4) || !aligned(s2, 4))
    return MOE_UNSUPPORTED;
  const Layer8Workspace w = layer8_layout(T, M, H, E, k, C, dtype);
  if (ws_bytes < w.total) return MOE_WORKSPACE_TOO_SMALL;
  char* base = (char*)ws;
  idx = idx ? idx : (int32_t*)(base + w.idx);
  loc = loc ? loc : (int32_t*)(base + w.loc);
  gate_w = gate_w ? gate_w : (float*)(base + w.gate_w);
  counts = counts ? counts : (int32_t*)(base + w.counts);
  logits = logits ? logits : (float*)(base + w.logits);
  int32_t* slot_src = (int32_t*)(base + w.slot_src);
  if (int st = moe_gate_route(x, Wg, gate_bias, dtype, T, M, E, k, C, normalize, logits, idx, gate_w, loc, counts, slot_src, base + w.gate_ws,
                              moe_gate_route_workspace_bytes(T, M, E, k, dtype), stream))
    return st;
  if (run_ffn8(x8, x_scales, slot_src, T, W1, s1, b1, W2, s2, b2, act, dtype, counts, E, C, M, H, ceil_div(T * k, E), base + w.hidden,
               (uint8_t*)(base + w.hidden_scales), base + w.Y, (hipStream_t)stream) != hipSuccess)
    return MOE_HIP_ERROR;
  return status_of(launch_decode(base + w.Y, dtype, idx, loc, gate_w, T, M, E, k, C, out, (hipStream_t)stream));
}

size_t moe_layer_few_workspace_bytes(int64_t T, int64_t M, int64_t H, int64_t E, int k, int dtype) {
  if (T > MOE_FEW_MAX_TOKENS || layer_shape_status(T, M, H, E, k, dtype) != MOE_OK || few_shape_status(M, H, false) != MOE_OK) return 0;
  return few_layout(T, M, H, E, k, dtype).total;
}

int moe_layer_forward_few(const void* x, const void* Wg, const float* gate_bias, const void* W1, const uint8_t* s1, const void* b1, const void* W2,
                          const uint8_t* s2, const void* b2, int64_t T, int64_t M, int64_t H, int64_t E, int k, double f, int normalize, int act,
                          int dtype, void* out, int32_t* idx, int32_t* loc, float* gate_w, int32_t* counts, float* logits, void* ws,
                          size_t ws_bytes, void* stream) {
  if (!x || !Wg || !W1 || !W2 || !out || !ws || (!s1) != (!s2) || !act_ok(act) || !(f > 0.0)) return MOE_INVALID_ARG;
  if (int st = layer_shape_status(T, M, H, E, k, dtype)) return st;
  if (T > MOE_FEW_MAX_TOKENS) return MOE_UNSUPPORTED;
  if (int st = few_shape_status(M, H, s1 != nullptr)) return st;
  const int64_t C = moe_capacity(T, E, k, f);
  if (C < 1 || C > kMaxDim) return MOE_INVALID_ARG;
  if (!all_aligned16({x, W1, b1, W2, b2, out, logits}) || !aligned(ws, 256)) return MOE_UNSUPPORTED;
  const FewWorkspace w = few_layout(T, M, H, E, k, dtype);
  if (ws_bytes < w.total) return MOE_WORKSPACE_TOO_SMALL;
  char* base = (char*)ws;
  idx = idx ? idx : (int32_t*)(base + w.idx);
  loc = loc ? loc : (int32_t*)(base + w.loc);
  gate_w = gate_w ? gate_w : (float*)(base + w.gate_w);
  counts = counts ? counts : (int32_t*)(base + w.counts);
  logits = logits ? logits : (float*)(base + w.logits);
  const FewTokens p = {x, Wg, W1, b1, W2, b2, gate_bias, s1, s2, idx, loc, counts, gate_w, logits, T, M, H, E, C, k, act, dtype, normalize, false, false, 0, 0, 0, 0, 0,
                       (double*)(base + w.logit_parts), (int32_t*)(base + w.plan), base + w.hidden, (float*)(base + w.partial),
                       (int32_t*)(base + w.arrived), out};
  return status_of(launch_few_tokens(p, (hipStream_t)stream));
}

}  // extern "C"
