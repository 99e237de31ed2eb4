// Matrices to the 8-bit block format (block8.h) and back.  A block of threads takes a tile of 128 x 128 values, which holds whole blocks of the format
// along both axes, so one read gives the rows' form, the transposed one, or both.  HBM bound: src once, a byte a value and output.  8 experts x 4096 x 2048 in bf16 to both forms
// 48 us = 5.6 TB/s, 8 x 2048 x 2048 with an exponent for 128 x 128 values 25 us = 5.4.
#include "block8.h"

namespace moe {
namespace {

__device__ __forceinline__ int live_rows(int64_t e, int R, const int32_t* counts) {
  if (!counts) return R;
  const int c = counts[e];
  return c < R ? (c > 0 ? c : 0) : R;
}

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
// zeros there up to the end of its block; tiles that lie past it altogether are left alone.  fills: gets the experts' live rows.  zeros: a matrix of R rows of zero_pieces 16 bytes for each expert that gets zeros in those rows.
template <typename ET, bool BLOCKS>
__global__ __launch_bounds__(256, 4) void quantize8_kernel(const ET* __restrict__ src, const int32_t* __restrict__ counts, int R, int K, int tiles_k,
                                                        uint8_t* __restrict__ q, uint8_t* __restrict__ scales, uint8_t* __restrict__ qt,
                                                        uint8_t* __restrict__ scales_t, int row8, int row_sc, int col8, int col_sc, int32_t* __restrict__ fills,
                                                        uint4* __restrict__ zeros, int zero_pieces) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[kBlock8 * kBlock8];
  __shared__ uint32_t tops[16][kBlock8];
  __shared__ uint8_t exponents[2][kBlock8];
  const int64_t e = blockIdx.y;
  const int rb = blockIdx.x / tiles_k, kb = blockIdx.x - rb * tiles_k;
  const int rows = live_rows(e, R, counts);
  if (fills && blockIdx.x == 0 && threadIdx.x == 0) fills[e] = rows;
  if (zeros) {                                                      // the same rows of another matrix, those that do not exist: shared by the tiles of a row of them
    const int first = max(rows, rb * kBlock8), last = min(R, (rb + 1) * kBlock8);
    uint4* to = zeros + (e * R + first) * (int64_t)zero_pieces;
    for (int i = kb * 256 + threadIdx.x; i < (last - first) * zero_pieces; i += tiles_k * 256) to[i] = make_uint4(0, 0, 0, 0);
  }
  if (rb * kBlock8 >= rows) return;
  const int t = threadIdx.x, rg = t >> 4, cg = t & 15, wave = t >> 6;
  const int r0 = rb * kBlock8 + rg * 8, c0 = kb * kBlock8 + cg * 8;
  float v[8][8];
  if (r0 + 8 <= rows && c0 < K) {
    const ET* at = src + (e * R + r0) * (int64_t)K + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i) load8(at + (int64_t)i * K, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
      if (r0 + i < rows && c0 < K) load8(src + (e * R + r0 + i) * (int64_t)K + c0, v[i]);
    }
  }
  // one row, or column, at a time: its largest magnitude, its exponent, its values (and for the tile's own exponent, that first)
  uint32_t tile_scale = 0;
  if (BLOCKS) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, magnitude_bits(v[i][j]));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((t & 63) == 0) tops[wave][0] = top;
    __syncthreads();
    tile_scale = scale_of_amax(max(max(tops[0][0], tops[1][0]), max(tops[2][0], tops[3][0])));
  }
  if (q) {
    uint8_t* to = q + (e * R + r0) * (int64_t)row8 + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t sc = tile_scale;
      if (!BLOCKS) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude_bits(v[i][j]));
        sc = scale_of_amax(max16(top));
        if (cg == 0) exponents[0][rg * 8 + i] = (uint8_t)sc;
      }
      const float m = inverse_scale(sc);
      uint2 w;
      w.x = pack8x4(v[i][0], v[i][1], v[i][2], v[i][3], m);
      w.y = pack8x4(v[i][4], v[i][5], v[i][6], v[i][7], m);
      if (r0 + i < rows) *reinterpret_cast<uint2*>(to + (int64_t)i * row8) = w;
    }
  }
  if (qt && !BLOCKS) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(v[i][j]));
      tops[rg][cg * 8 + j] = top;
    }
    __syncthreads();
    if (t < kBlock8) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = max(top, tops[i][t]);
      exponents[1][t] = (uint8_t)scale_of_amax(top);
    }
  }
  if (!BLOCKS) __syncthreads();
  if (qt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float m = inverse_scale(BLOCKS ? tile_scale : exponents[1][cg * 8 + j]);
      uint2 w;
      w.x = pack8x4(v[0][j], v[1][j], v[2][j], v[3][j], m);
      w.y = pack8x4(v[4][j], v[5][j], v[6][j], v[7][j], m);
      *reinterpret_cast<uint2*>(tile + (cg * 8 + j) * kBlock8 + (((rg >> 1) ^ (cg & 7)) << 4) + (rg & 1) * 8) = w;
    }
  }
  // exponents: the tile's from one thread, or row t's and column t - 128's from thread t; the last tile of a row of them pads it
  const bool second = t >= kBlock8;
  const int i = t & (kBlock8 - 1), at = second ? rb : kb, pitch = second ? col_sc : row_sc, line = (second ? kb : rb) * kBlock8 + i;
  uint8_t* sc = second ? scales_t : scales;
  if (sc && (BLOCKS ? i == 0 : line < (second ? K : rows))) {
    sc += (BLOCKS ? e * (((second ? K : R) + kBlock8 - 1) / kBlock8) + line / kBlock8 : e * (second ? K : R) + line) * (int64_t)pitch + at;
    sc[0] = (uint8_t)(BLOCKS ? tile_scale : exponents[second][i]);
    if (at == (second ? (R + kBlock8 - 1) / kBlock8 : tiles_k) - 1)
      for (int p = 1; p < pitch - at; ++p) sc[p] = (uint8_t)kScaleOne;
  }
  if (!qt) return;
  __syncthreads();
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int c = s * 32 + (t >> 3), p = t & 7;
    const int col = kb * kBlock8 + c;
    if (col < K) *reinterpret_cast<uint4*>(qt + (e * K + col) * (int64_t)col8 + rb * kBlock8 + p * 16) = *reinterpret_cast<const uint4*>(tile + c * kBlock8 + ((p ^ ((c >> 3) & 7)) << 4));
  }
}

// 16 values a lane; exact in fp32 and bf16 but at the ends of the format (moe_dequantize8).
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
                            uint8_t* scales, void* qt, uint8_t* scales_t, hipStream_t s, int32_t* fills, void* zeros,
                            int64_t zero_width) {
  const dim3 grid((unsigned)(ceil_div(K, kBlock8) * ceil_div(R, kBlock8)), (unsigned)E);
#define MOE_QUANTIZE(ET, B)                                                                                                           \
  quantize8_kernel<ET, B><<<grid, dim3(256), 0, s>>>((const ET*)src, counts, (int)R, (int)K, (int)ceil_div(K, kBlock8), (uint8_t*)q, scales, (uint8_t*)qt, scales_t, \
                                                     (int)row_bytes8(K), (int)row_scales8(K), (int)row_bytes8(R), (int)row_scales8(R), \
                                                     fills, (uint4*)zeros, (int)(zero_width * (dtype == MOE_F32 ? 4 : 2) / 16))
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
