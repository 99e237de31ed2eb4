// What the entry points check their arguments with (api.hip, api8.hip).
#pragma once
#include "common.h"

namespace moe {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool dtype_ok(int d) { return d == MOE_F32 || d == MOE_BF16; }
inline bool act_ok(int a) { return a == MOE_ACT_RELU || a == MOE_ACT_GELU || a == MOE_ACT_SILU; }
inline size_t esize(int d) { return d == MOE_F32 ? 4 : 2; }
constexpr int64_t kMaxDim = (int64_t)1 << 30;

inline int gate_shape_status(int64_t T, int64_t E, int k) {
  if (T < 1 || E < 1 || k < 1 || k > E || T > kMaxDim) return MOE_INVALID_ARG;
  if (E > 512 || (int64_t)k * E > 16384) return MOE_UNSUPPORTED;
  return MOE_OK;
}

inline int row_shape_status(int64_t M) {
  if (M < 1 || M > kMaxDim) return MOE_INVALID_ARG;
  if (M % 8 != 0) return MOE_UNSUPPORTED;
  return MOE_OK;
}

}  // namespace moe
