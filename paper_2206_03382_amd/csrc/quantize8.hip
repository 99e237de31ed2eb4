// Matrices to the 8-bit block format (block8.h) and back.  A block of threads takes a tile of 128 x 128 values, which holds whole blocks of the format
// along both axes, so one read gives the rows' form, the transposed one, or both.  HBM bound: src once, a byte a value and output.
#include "block8.h"

namespace moe {
namespace {

template <typename ET> __device__ __forceinline__ void load8(const ET* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float (&v)[8]) { Vec16<uint16_t>::unpack(load_stream(reinterpret_cast<const uint4*>(p)), v); }
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  float a[4], b[4];
  const uint4 ra = load_stream(reinterpret_cast<const uint4*>(p)), rb = load_stream(reinterpret_cast<const uint4*>(p) + 1);
  Vec16<float>::unpack(ra, a);
  Vec16<float>::unpack(rb, b);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = a[j];
    v[4 + j] = b[j];
  }
}

// Thread t of 256 has the 8 rows from 8 (t / 16) and the 8 columns from 8 (t % 16): 16 lanes read a row's 128 values, and a thread's 8 x 8 values are
// 8-byte pieces of both forms.  The transposed form goes through LDS (16 KB, 8-byte pieces, the pair of piece p of column c at p/2 ^ c/8 % 8: lanes of a
// wave write to different banks) and out in rows of 128 bytes.
// BLOCKS: one exponent for the tile; else one for each row and column of it.  Rows past an expert's fill count as zero: the transposed form has
// zeros there up to the end of its block; tiles that lie past it altogether are left alone.
template <typename ET, bool BLOCKS>
__global__ __launch_bounds__(256) void quantize8_kernel(const ET* __restrict__ src, const int32_t* __restrict__ counts, int64_t R, int64_t K,
                                                        uint8_t* __restrict__ q, uint8_t* __restrict__ scales, uint8_t* __restrict__ qt,
                                                        uint8_t* __restrict__ scales_t, int64_t row8, int64_t row_sc, int64_t col8, int64_t col_sc) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[kBlock8 * kBlock8];
  __shared__ uint32_t tops[4][kBlock8];
  const int64_t e = blockIdx.y, tiles_k = ceil_div(K, kBlock8), rb = blockIdx.x / tiles_k, kb = blockIdx.x % tiles_k;
  int64_t rows = R;
  if (counts) {
    const int64_t c = counts[e];
    rows = c < R ? (c > 0 ? c : 0) : R;
  }
  if (rb * kBlock8 >= rows) return;
  const int t = threadIdx.x, rg = t >> 4, cg = t & 15, wave = t >> 6;
  const int64_t r0 = rb * kBlock8 + rg * 8, c0 = kb * kBlock8 + cg * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    if (r0 + i < rows && c0 < K) load8(src + (e * R + r0 + i) * K + c0, v[i]);
  }
  uint32_t row_scale[8], col_scale[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude_bits(v[i][j]));
    row_scale[i] = max16(top);
  }
  if (BLOCKS) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, row_scale[i]);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if ((t & 63) == 0) tops[wave][0] = top;
    __syncthreads();
    const uint32_t sc = scale_of_amax(max(max(tops[0][0], tops[1][0]), max(tops[2][0], tops[3][0])));
#pragma unroll
    for (int i = 0; i < 8; ++i) row_scale[i] = col_scale[i] = sc;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) row_scale[i] = scale_of_amax(row_scale[i]);
    if (qt) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(v[i][j]));
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        if ((t & 63) < 16) tops[wave][cg * 8 + j] = top;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = cg * 8 + j;
        col_scale[j] = scale_of_amax(max(max(tops[0][c], tops[1][c]), max(tops[2][c], tops[3][c])));
      }
    }
  }
  const bool last_k = kb == tiles_k - 1, last_r = (rb + 1) * kBlock8 >= R;
  if (q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = r0 + i;
      if (r >= rows) break;
      uint2 w;
      w.x = pack8x4(v[i][0], v[i][1], v[i][2], v[i][3], row_scale[i]);
      w.y = pack8x4(v[i][4], v[i][5], v[i][6], v[i][7], row_scale[i]);
      *reinterpret_cast<uint2*>(q + (e * R + r) * row8 + c0) = w;
    }
    // exponents: of the thread's rows, or of the tile; the last tile of a row pads it
    uint8_t* to = scales + (BLOCKS ? (e * ceil_div(R, kBlock8) + rb) : e * R + r0) * row_sc;
    const int own = BLOCKS ? (t == 0) : (cg == 0 ? (int)(rows - r0 < 8 ? rows - r0 : 8) : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= own) break;
      to[i * row_sc + kb] = (uint8_t)row_scale[i];
      if (last_k) for (int64_t p = kb + 1; p < row_sc; ++p) to[i * row_sc + p] = (uint8_t)kScaleOne;
    }
  }
  if (!qt) return;
  {
    uint8_t* to = scales_t + (BLOCKS ? (e * ceil_div(K, kBlock8) + kb) : e * K + c0) * col_sc;
    const int own = BLOCKS ? (t == 0) : (rg == 0 && c0 < K ? 8 : 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= own) break;
      to[j * col_sc + rb] = (uint8_t)col_scale[j];
      if (last_r) for (int64_t p = rb + 1; p < col_sc; ++p) to[j * col_sc + p] = (uint8_t)kScaleOne;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint2 w;
    w.x = pack8x4(v[0][j], v[1][j], v[2][j], v[3][j], col_scale[j]);
    w.y = pack8x4(v[4][j], v[5][j], v[6][j], v[7][j], col_scale[j]);
    *reinterpret_cast<uint2*>(tile + (cg * 8 + j) * kBlock8 + (((rg >> 1) ^ (cg & 7)) << 4) + (rg & 1) * 8) = w;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = i * 32 + (t >> 3), p = t & 7;
    const int64_t col = kb * kBlock8 + c;
    if (col < K) *reinterpret_cast<uint4*>(qt + (e * K + col) * col8 + rb * kBlock8 + p * 16) = *reinterpret_cast<const uint4*>(tile + c * kBlock8 + ((p ^ ((c >> 3) & 7)) << 4));
  }
}

// 16 values a lane; bf16 holds every value of the format.
template <typename ET>
__global__ __launch_bounds__(256) void dequantize8_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scales, int blocks, int64_t R,
                                                          int64_t K, int64_t total, int64_t per_row, int64_t row8, int64_t row_sc, ET* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const int64_t row = i / per_row, c = (i - row * per_row) * 16;
  const uint4 w = load_stream(reinterpret_cast<const uint4*>(q + row * row8 + c));
  int64_t srow = row;
  if (blocks) {
    const int64_t e = row / R;
    srow = e * ceil_div(R, kBlock8) + (row - e * R) / kBlock8;
  }
  const uint32_t b = scales[srow * row_sc + c / kBlock8];
  const float m = b == kScaleNaN ? __uint_as_float(0x7fc00000u) : (b == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(b << 23));
  const uint32_t words[4] = {w.x, w.y, w.z, w.w};
  float v[16];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[4 * j] = __builtin_amdgcn_cvt_f32_fp8((int)words[j], 0) * m;
    v[4 * j + 1] = __builtin_amdgcn_cvt_f32_fp8((int)words[j], 1) * m;
    v[4 * j + 2] = __builtin_amdgcn_cvt_f32_fp8((int)words[j], 2) * m;
    v[4 * j + 3] = __builtin_amdgcn_cvt_f32_fp8((int)words[j], 3) * m;
  }
  constexpr int N = Vec16<ET>::N;
#pragma unroll
  for (int j = 0; j < 16; j += N) {
    if (c + j >= K) break;                                          // K is a multiple of 8
    float f[N];
#pragma unroll
    for (int n = 0; n < N; ++n) f[n] = v[j + n];
    *reinterpret_cast<uint4*>(out + row * K + c + j) = Vec16<ET>::pack(f);
  }
}

}  // namespace

hipError_t launch_quantize8(const void* src, int dtype, const int32_t* counts, int64_t E, int64_t R, int64_t K, bool blocks, void* q,
                            uint8_t* scales, void* qt, uint8_t* scales_t, hipStream_t s) {
  const dim3 grid((unsigned)(ceil_div(K, kBlock8) * ceil_div(R, kBlock8)), (unsigned)E);
#define MOE_QUANTIZE(ET, B)                                                                                                           \
  quantize8_kernel<ET, B><<<grid, dim3(256), 0, s>>>((const ET*)src, counts, R, K, (uint8_t*)q, scales, (uint8_t*)qt, scales_t, row_bytes8(K), \
                                                     row_scales8(K), row_bytes8(R), row_scales8(R))
  if (dtype == MOE_F32) { if (blocks) MOE_QUANTIZE(float, true); else MOE_QUANTIZE(float, false); }
  else { if (blocks) MOE_QUANTIZE(uint16_t, true); else MOE_QUANTIZE(uint16_t, false); }
#undef MOE_QUANTIZE
  return hipGetLastError();
}

hipError_t launch_dequantize8(const void* q, const uint8_t* scales, bool blocks, int64_t E, int64_t R, int64_t K, int dtype, void* out,
                              hipStream_t s) {
  const int64_t per_row = ceil_div(K, 16), total = E * R * per_row;
  const dim3 grid((unsigned)ceil_div(total, 256));
  if (dtype == MOE_F32)
    dequantize8_kernel<float><<<grid, dim3(256), 0, s>>>((const uint8_t*)q, scales, blocks, R, K, total, per_row, row_bytes8(K), row_scales8(K), (float*)out);
  else
    dequantize8_kernel<uint16_t><<<grid, dim3(256), 0, s>>>((const uint8_t*)q, scales, blocks, R, K, total, per_row, row_bytes8(K), row_scales8(K), (uint16_t*)out);
  return hipGetLastError();
}

}  // namespace moe
