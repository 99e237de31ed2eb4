// RMS norm with the residual's addition, its 8-bit output, and its gradient.
//   h = x + residual;  y = h * r * w,  r = 1 / sqrt(mean(h^2) + eps);  the row's statistics and y from the fp32 sum, before h is rounded.
//   backward, g = dy * w:  dx = r * (g - h * r^2 * mean(g * h)) + dh;  dw = sum over the rows of dy * h * r.
// One pass: a row stays in the registers of 64, 256 or 1024 lanes between the reduction and its use.  HBM bound: every input is read once with
// 16-byte loads and every output written once.  131072 x 4096 in bf16 with a residual, h and y: 774 us = 5.6 TB/s (a copy 5.2); 32768 x 4096 backward with the residual's gradient
// 203 us = 5.3 TB/s; 16 x 4096 with the 8-bit output as well 4 us, a launch and a row's latency.
#include "block8.h"

namespace moe {
namespace {

// Sum over the LANES lanes of a row (whole waves), in all of them, in a fixed order.  `part`: LDS of a value per wave, of this row's waves.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* part) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  if (LANES == 64) return v;
  const int lane = threadIdx.x & 63, wave = (threadIdx.x % LANES) >> 6;
  if (lane == 0) part[wave] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < LANES / 64; ++i) s += part[i];
  return s;
}

template <typename ET> __device__ __forceinline__ uint4 load16(const ET* p) { return load_stream(reinterpret_cast<const uint4*>(p)); }

// LANES lanes to a row, VPL pieces of 16 bytes to a lane: piece i of lane l is piece l + i * LANES of the row.
template <typename ET, int LANES, int VPL>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_norm_kernel(const ET* __restrict__ x, const ET* __restrict__ residual,
                                                                             const ET* __restrict__ weight, float eps, int64_t T, int M,
                                                                             ET* __restrict__ h, ET* __restrict__ y, uint8_t* __restrict__ q,
                                                                             uint8_t* __restrict__ scales, int row8, int rows_scales) {
  constexpr int N = Vec16<ET>::N, BLOCK = LANES < 256 ? 256 : LANES;
  __shared__ float part[BLOCK / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * (BLOCK / LANES) + threadIdx.x / LANES;
  if (LANES < BLOCK && row >= T) return;                            // whole waves, and no barrier where a block has several rows
  const int pieces = M / N;
  const int64_t at = row * M;
  uint4 raw[VPL], res[VPL];
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int p = lane + i * LANES;
    raw[i] = res[i] = make_uint4(0, 0, 0, 0);
    if (p < pieces) {
      raw[i] = load16(x + at + p * N);
      if (residual) res[i] = load16(residual + at + p * N);
    }
  }
  float v[VPL][N], sum = 0.f;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    Vec16<ET>::unpack(raw[i], v[i]);
    if (residual) {
      float r[N];
      Vec16<ET>::unpack(res[i], r);
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] += r[j];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) sum += v[i][j] * v[i][j];
  }
  if (h) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int p = lane + i * LANES;
      if (p < pieces) *reinterpret_cast<uint4*>(h + at + p * N) = Vec16<ET>::pack(v[i]);
    }
  }
  const float r = rsqrtf(row_sum<LANES>(sum, part) / (float)M + eps);
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int p = lane + i * LANES;
    if (weight && p < pieces) {
      float w[N];
      Vec16<ET>::unpack(*reinterpret_cast<const uint4*>(weight + p * N), w);
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] *= r * w[j];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] *= r;                     // pieces past the row's end stay zero
    }
    if (y && p < pieces) *reinterpret_cast<uint4*>(y + at + p * N) = Vec16<ET>::pack(v[i]);
  }
  if (!q) return;
  // a block of 128 values is 16 lanes' pieces in bf16, 32 lanes' in fp32
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int p = lane + i * LANES;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) top = max(top, magnitude_bits(v[i][j]));
    top = max16(top);
    if (N == 4) top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    const uint32_t scale = scale_of_amax(top);
    const float inverse = inverse_scale(scale);
    if (p * N < row8) {
      uint8_t* to = q + row * row8 + p * N;
      const uint32_t lo = pack8x4(v[i][0], v[i][1], v[i][2], v[i][3], inverse);
      if constexpr (N == 8) *reinterpret_cast<uint2*>(to) = make_uint2(lo, pack8x4(v[i][4], v[i][5], v[i][6], v[i][7], inverse));
      else *reinterpret_cast<uint32_t*>(to) = lo;
      if (p * N % kBlock8 == 0) scales[row * rows_scales + p * N / kBlock8] = (uint8_t)scale;
    }
  }
  const int past = row8 / kBlock8 + lane;
  if (past < rows_scales) scales[row * rows_scales + past] = (uint8_t)kScaleOne;
}

// Rows are dealt to the row slots of the grid; a slot's lanes keep the sums of dw over its rows in registers, and partial [slots, M] holds them in the
// end.  Sums over the slots follow in a second launch: no atomics, so the result is the same in every run.
template <typename ET, int LANES, int VPL>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rms_norm_backward_kernel(const ET* __restrict__ dy, const ET* __restrict__ dh,
                                                                                      const ET* __restrict__ h, const ET* __restrict__ weight,
                                                                                      float eps, int64_t T, int M, ET* __restrict__ dx,
                                                                                      float* __restrict__ partial) {
  constexpr int N = Vec16<ET>::N, BLOCK = LANES < 256 ? 256 : LANES;
  __shared__ float part[2][2][BLOCK / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t slot = (int64_t)blockIdx.x * (BLOCK / LANES) + threadIdx.x / LANES, slots = (int64_t)gridDim.x * (BLOCK / LANES);
  const int pieces = M / N;
  float dw[VPL][N] = {};
  int turn = 0;                                                     // the LDS of the reductions, in turn: one barrier a row is enough
  for (int64_t row = slot; row < T; row += slots, turn ^= 1) {
    const int64_t at = row * M;
    uint4 rh[VPL], rdy[VPL], rdh[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int p = lane + i * LANES;
      rh[i] = rdy[i] = rdh[i] = make_uint4(0, 0, 0, 0);
      if (p < pieces) {
        rh[i] = load16(h + at + p * N);
        rdy[i] = load16(dy + at + p * N);
        if (dh) rdh[i] = load16(dh + at + p * N);
      }
    }
    float squares = 0.f, dots = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int p = lane + i * LANES;
      float a[N], b[N], w[N];
      Vec16<ET>::unpack(rh[i], a);
      Vec16<ET>::unpack(rdy[i], b);
      if (weight && p < pieces) Vec16<ET>::unpack(*reinterpret_cast<const uint4*>(weight + p * N), w);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        squares += a[j] * a[j];
        dots += (weight && p < pieces ? b[j] * w[j] : b[j]) * a[j];
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      squares += __shfl_xor(squares, d);
      dots += __shfl_xor(dots, d);
    }
    if (LANES > 64) {
      const int wave = (threadIdx.x % LANES) >> 6;
      if ((threadIdx.x & 63) == 0) {
        part[turn][0][wave] = squares;
        part[turn][1][wave] = dots;
      }
      __syncthreads();
      squares = dots = 0.f;
#pragma unroll
      for (int i = 0; i < LANES / 64; ++i) {
        squares += part[turn][0][i];
        dots += part[turn][1][i];
      }
    }
    const float r = rsqrtf(squares / (float)M + eps), c = r * (r * (dots / (float)M));       // r * r may be no fp32 number
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int p = lane + i * LANES;
      float a[N], b[N], w[N], o[N];
      Vec16<ET>::unpack(rh[i], a);
      Vec16<ET>::unpack(rdy[i], b);
      Vec16<ET>::unpack(rdh[i], o);
      if (weight && p < pieces) Vec16<ET>::unpack(*reinterpret_cast<const uint4*>(weight + p * N), w);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        o[j] += r * ((weight && p < pieces ? b[j] * w[j] : b[j]) - a[j] * c);
        dw[i][j] += b[j] * (a[j] * r);
      }
      if (p < pieces) *reinterpret_cast<uint4*>(dx + at + p * N) = Vec16<ET>::pack(o);
    }
  }
  if (!partial) return;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int p = lane + i * LANES;
    if (p >= pieces) continue;
#pragma unroll
    for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(partial + slot * M + p * N + j) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
  }
}

// dw[c] = sum over the slots of partial[slot, c]: 32 columns to a block, 32 groups of slots.
template <typename ET>
__global__ __launch_bounds__(1024) void weight_sum_kernel(const float* __restrict__ partial, int slots, int M, ET* __restrict__ dw) {
  __shared__ float sums[32][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < M) {
#pragma unroll 4
    for (int i = g; i < slots; i += 32) s += partial[(int64_t)i * M + col];
  }
  sums[g][c] = s;
  __syncthreads();
  if (g == 0 && col < M) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][c];
    store_from_f32(dw + col, s);
  }
}

// Lanes to a row of so many 16-byte pieces.  A wave alone needs no barrier; more lanes have a shorter row, which is all the time that few rows take.
// us with 64 and with 256 lanes, bf16 with a residual: widths of 512 (64 pieces) 16 rows 2.9, 3.0, 4096 4.7, 7.0, 65536 49, 72; 1024 16 rows 3.6, 3.0, 4096 7.7, 9.4, 65536 110, 107;
// 2048 16 rows 4.9, 3.0, 4096 14.0, 15.8, 65536 221, 202.
inline int forward_lanes(int64_t pieces, int64_t T) {
  if (pieces <= 64 || (pieces <= 128 && T >= 2048)) return 64;
  return pieces <= 1024 ? 256 : 1024;
}
// Backward, where rows of fewer lanes are in more slots, whose sums for dw are written and read again: widths of 512 4096 rows 19.7, 12.0, 16384 27.8, 34.9, 65536 54, 121;
// 1024 4096 rows 26.6, 14.4, 16384 38, 41, 65536 92, 134; 2048 4096 rows 35, 21, 65536 190, 168.
inline int backward_lanes(int64_t pieces, int64_t T) {
  if (pieces <= 128 && T >= 16384) return 64;
  return pieces <= 1024 ? 256 : 1024;
}
constexpr int64_t kBackwardSlots = 1024;                            // of 256 lanes: four blocks to a unit

inline int64_t backward_slots(int64_t pieces, int64_t T) {
  const int lanes = backward_lanes(pieces, T);
  const int64_t per_block = lanes < 256 ? 256 / lanes : 1;
  const int64_t most = kBackwardSlots * 256 / lanes;
  return ceil_div(T < most ? T : most, per_block) * per_block;
}

}  // namespace

#define MOE_NORM_FORMS(CALL, ET)                                       \
  do {                                                                 \
    const int64_t vpl = ceil_div(pieces, lanes);                       \
    if (lanes == 64) {                                                 \
      if (vpl <= 1) CALL(ET, 64, 1);                                   \
      else CALL(ET, 64, 2);                                            \
    } else if (lanes == 256) {                                         \
      if (vpl <= 1) CALL(ET, 256, 1);                                  \
      else if (vpl <= 2) CALL(ET, 256, 2);                             \
      else CALL(ET, 256, 4);                                           \
    } else {                                                           \
      if (vpl <= 2) CALL(ET, 1024, 2);                                 \
      else CALL(ET, 1024, sizeof(ET) == 4 ? 4 : 2); /* rows of bf16: at most 2048 pieces */ \
    }                                                                  \
  } while (0)

hipError_t launch_rms_norm(const void* x, const void* residual, const void* weight, float eps, int dtype, int64_t T, int64_t M, void* h,
                           void* y, void* q, uint8_t* scales, hipStream_t s) {
  const int n = dtype == MOE_F32 ? 4 : 8;
  const int64_t row8 = row_bytes8(M), pieces = ceil_div(q ? row8 : M, n);
  const int lanes = forward_lanes(pieces, T);
  const dim3 block(lanes < 256 ? 256 : lanes), grid((unsigned)ceil_div(T, block.x / lanes));
#define MOE_NORM(ET, L, V)                                                                                                            \
  rms_norm_kernel<ET, L, V><<<grid, block, 0, s>>>((const ET*)x, (const ET*)residual, (const ET*)weight, eps, T, (int)M, (ET*)h, (ET*)y, \
                                                   (uint8_t*)q, scales, (int)row8, (int)row_scales8(M))
  if (dtype == MOE_F32) MOE_NORM_FORMS(MOE_NORM, float);
  else MOE_NORM_FORMS(MOE_NORM, uint16_t);
#undef MOE_NORM
  return hipGetLastError();
}

size_t rms_norm_backward_workspace_bytes(int64_t T, int64_t M) {
  const int64_t a = backward_slots(ceil_div(M, 8), T), b = backward_slots(ceil_div(M, 4), T);
  return (size_t)(a > b ? a : b) * M * sizeof(float);
}

hipError_t launch_rms_norm_backward(const void* dy, const void* dh, const void* h, const void* weight, float eps, int dtype, int64_t T,
                                    int64_t M, float* ws, void* dx, void* dweight, hipStream_t s) {
  const int64_t pieces = M / (dtype == MOE_F32 ? 4 : 8);
  const int lanes = backward_lanes(pieces, T);
  const int64_t slots = backward_slots(pieces, T);
  const dim3 block(lanes < 256 ? 256 : lanes), grid((unsigned)(slots * lanes / block.x));
  float* partial = dweight ? ws : nullptr;
#define MOE_NORM_BACKWARD(ET, L, V) \
  rms_norm_backward_kernel<ET, L, V><<<grid, block, 0, s>>>((const ET*)dy, (const ET*)dh, (const ET*)h, (const ET*)weight, eps, T, (int)M, (ET*)dx, partial)
  if (dtype == MOE_F32) MOE_NORM_FORMS(MOE_NORM_BACKWARD, float);
  else MOE_NORM_FORMS(MOE_NORM_BACKWARD, uint16_t);
#undef MOE_NORM_BACKWARD
  if (hipError_t err = hipGetLastError()) return err;
  if (!dweight) return hipSuccess;
  const dim3 columns((unsigned)ceil_div(M, 32));
  if (dtype == MOE_F32) weight_sum_kernel<float><<<columns, dim3(1024), 0, s>>>(ws, (int)slots, (int)M, (float*)dweight);
  else weight_sum_kernel<uint16_t><<<columns, dim3(1024), 0, s>>>(ws, (int)slots, (int)M, (uint16_t*)dweight);
  return hipGetLastError();
}
#undef MOE_NORM_FORMS

}  // namespace moe
