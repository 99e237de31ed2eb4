// Grouped products of 8-bit matrices with a power of two for each block of 128 (block8.h):
//   out[e][r, n] = act(sum_b 2^(ea[r, b] + eb[n, b]) * sum_{k in b} A[e][r, k] * B[e][n, k] + bias[e][n])
// on v_mfma_scale_f32_16x16x128_f8f6f4: a K-step of 128 is one block of the format, both of whose exponents go into the instruction, and the sums
// stay in fp32 accumulators from the first block to the last.  Both operands have k contiguous, so a lane's 32 bytes of a fragment are two 16-byte LDS
// reads; which k they are does not matter as long as A and B agree, since the block's exponent is the same for all of them.
//
// These instructions align a step's 128 products to the largest before they add them up and lose what is 2^-16 or so of it: 1.5e-5 of the result
// (relative, 2-norm) whatever K is, which a result rounded to bf16 (1.7e-3) or to 8 bits does not show.  fp32 results go through v_mfma_f32_16x16x32_bf16 on
// the values widened to bf16, which holds them all, exponent included: 1e-7, at less than half the rate.
#include "block8.h"
#include "ffn_device.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

// four bytes times 2^(exponent byte - 127), in bf16 without a rounding
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return byte == kScaleNaN ? __uint_as_float(0x7fc00000u) : byte == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

struct Args8 {
  Matmul8 p;
  int64_t row8, row_sc;           // bytes of a row of A and B, of its exponents
  int64_t out_row8, out_row_sc;
  int MT, NT, plain;
  bool stream;                    // the large tile's results are not kept in the caches
};

// BM x BN to a block of WM x WN waves; NS stages of a K-step in LDS.  LDS: rows of 128 bytes, 16-byte piece g of row r at g ^ (r / 2) % 8.
template <int BM, int BN, int WM, int WN, int NS, bool EXACT>
__global__ __launch_bounds__(256) void matmul8_kernel(const Args8 a) {
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
  constexpr int LA = BM / 32, LB = BN / 32, STAGE = (BM + BN) * kBlock8;
  static_assert(WM * WN == 4 && BN % kBlock8 == 0 && NS * STAGE <= 163840, "four waves, whole blocks of the output format, stages that fit a unit");
  __shared__ __attribute__((aligned(1024))) char smem[NS * STAGE];
  const Matmul8& p = a.p;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  int e, mt, nt, rows;
  if (!a.plain) {
    if (!find_tile<BM>(blockIdx.x, lane, (int)p.E, p.C, p.counts, a.NT, e, mt, nt, rows)) return;
  } else {
    e = blockIdx.y;
    mt = blockIdx.x / a.NT;
    nt = blockIdx.x % a.NT;
    rows = live_rows_of(e, p.C, p.counts);
  }
  const int64_t m0 = (int64_t)mt * BM, n0 = (int64_t)nt * BN;
  if (m0 >= rows) return;
  const int N = (int)p.N;
  int KT = (int)(a.row8 / kBlock8);
  if (p.k_counts) {
    const int64_t c = p.k_counts[e];
    const int64_t most = c < p.K ? (c > 0 ? c : 0) : p.K;
    KT = (int)ceil_div(most, kBlock8);
  }
  auto a_row = [&](int64_t r) -> int64_t {                          // rows past the fill repeat the last one (never stored)
    r = m0 + r < rows ? m0 + r : rows - 1;
    if (!p.gather) return (int64_t)e * p.C + r;
    const int t = p.gather[(int64_t)e * p.C + r];
    return (unsigned)t < (uint64_t)p.gather_rows ? t : 0;
  };
  auto b_row = [&](int n) -> int64_t { return n0 + n < N ? n0 + n : N - 1; };      // so do columns past N

  // direct loads: wave w's load q brings 8 rows, lane l the piece l % 8 of row l / 8, from where the swizzle wants it
  const char* a_at[LA];
  uint32_t b_at[LB];
  const char* b_base = (const char*)p.B + (int64_t)e * N * a.row8;
#pragma unroll
  for (int q = 0; q < LA; ++q) {
    const int r = (q * 4 + wave) * 8 + (lane >> 3);
    a_at[q] = (const char*)p.A + a_row(r) * a.row8 + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
  }
#pragma unroll
  for (int q = 0; q < LB; ++q) {
    const int r = (q * 4 + wave) * 8 + (lane >> 3);
    b_at[q] = (uint32_t)(b_row(r) * a.row8 + (((lane & 7) ^ ((r >> 1) & 7)) << 4));
  }
  const uint32_t smem_addr = (uint32_t)(uintptr_t)LDS_PTR(char, smem);
  auto load_step = [&](int kt) {
    const uint32_t to = smem_addr + (kt % NS) * STAGE + wave * 1024;
    const char* b_src = b_base + (int64_t)kt * kBlock8;
#pragma unroll
    for (int q = 0; q < LA; ++q) global_to_lds_16(a_at[q] + (int64_t)kt * kBlock8, to + q * 4096);
#pragma unroll
    for (int q = 0; q < LB; ++q) global_to_lds_16(b_src, b_at[q], to + BM * kBlock8 + q * 4096);
  };
  // exponents: a word for four K-steps, of the fragment row that the lane holds
  const uint32_t* a_sc[TM];
  const uint32_t* b_sc[TN];
  const int fr = lane & 15, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < TM; ++i) a_sc[i] = (const uint32_t*)(p.A_scales + a_row(wm * WTM + i * 16 + fr) * a.row_sc);
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t n = b_row(wn * WTN + j * 16 + fr);
    b_sc[j] = (const uint32_t*)(p.B_scales + (p.b_blocks ? (int64_t)e * ceil_div(N, kBlock8) + n / kBlock8 : (int64_t)e * N + n) * a.row_sc);
  }
  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t sa[TM], sb[TN];
#pragma unroll
  for (int t = 0; t < NS - 1; ++t) if (t < KT) load_step(t);
  for (int kt = 0; kt < KT; ++kt) {
    if (kt % 4 == 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = a_sc[i][kt / 4];
#pragma unroll
      for (int j = 0; j < TN; ++j) sb[j] = b_sc[j][kt / 4];
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (kt + NS - 1 < KT) load_step(kt + NS - 1);
    const char* as = smem + (kt % NS) * STAGE + wm * WTM * kBlock8;
    const char* bs = smem + (kt % NS) * STAGE + (BM + wn * WTN) * kBlock8;
    auto fragment = [&](const char* at, int i) -> i32x8 {
      const int sw = ((i * 16 + fr) >> 1) & 7;
      const u32x4 lo = *LDS_PTR(u32x4, at + (i * 16 + fr) * kBlock8 + ((g ^ sw) << 4));
      const u32x4 hi = *LDS_PTR(u32x4, at + (i * 16 + fr) * kBlock8 + (((g + 4) ^ sw) << 4));
      return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };
    i32x8 av[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) av[i] = fragment(as, i);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const i32x8 bv = fragment(bs, j);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if constexpr (EXACT) {
#pragma unroll
          for (int c = 0; c < 8; c += 2)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(bv[c], bv[c + 1], scale_value(sb[j] & 255)),
                                                                widen8(av[i][c], av[i][c + 1], scale_value(sa[i] & 255)), acc[i][j], 0, 0, 0);
        } else {
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bv, av[i], acc[i][j], 0, 0, 0, (int)sb[j], 0, (int)sa[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] >>= 8;
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] >>= 8;
  }
  // epilogue: the lane has row 16 i + l % 16 and columns 16 j + 4 (l / 16) .. + 3 of its wave's part
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int64_t n = n0 + wn * WTN + j * 16 + 4 * g;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float f = acc[i][j][v];
        if (n >= N) f = 0.f;                                        // N is a multiple of 8
        else {
          if (p.bias) f += p.dtype == MOE_F32 ? ((const float*)p.bias)[(int64_t)e * N + n + v] : bf16_bits_to_f32(((const uint16_t*)p.bias)[(int64_t)e * N + n + v]);
          if (p.act >= 0) f = apply_act(f, p.act);
        }
        acc[i][j][v] = f;
      }
    }
  }
  if (p.out) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t r = m0 + wm * WTM + i * 16 + fr;
      if (r >= rows) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int64_t n = n0 + wn * WTN + j * 16 + 4 * g;
        if (n >= N) continue;
        const int64_t at = ((int64_t)e * p.C + r) * N + n;
        if (p.dtype == MOE_F32) *reinterpret_cast<f32x4*>((float*)p.out + at) = acc[i][j];
        else *reinterpret_cast<uint2*>((uint16_t*)p.out + at) = make_uint2(pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3]));
      }
    }
    return;
  }
  // 8-bit output: the block's largest magnitude over the wave's columns, then over the waves that share the block of 128
  uint32_t* tops = (uint32_t*)smem;                                 // [BM][WN]
  __syncthreads();
  constexpr int WPB = kBlock8 > WTN ? kBlock8 / WTN : 1, BPW = WTN > kBlock8 ? WTN / kBlock8 : 1, JB = TN / BPW;
  static_assert(BPW == 1, "a wave's columns lie in one block");
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) top = max(top, magnitude_bits(acc[i][j][v]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if (g == 0) tops[(wm * WTM + i * 16 + fr) * WN + wn] = top;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int rl = wm * WTM + i * 16 + fr;
    const int64_t r = m0 + rl;
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < WPB; ++w) top = max(top, tops[rl * WN + wn / WPB * WPB + w]);
    const uint32_t sc = scale_of_amax(top);
    if (r >= rows) continue;
    const int64_t row = (int64_t)e * p.C + r;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int64_t n = n0 + wn * WTN + j * 16 + 4 * g;
      if (n < a.out_row8) *reinterpret_cast<uint32_t*>((uint8_t*)p.out8 + row * a.out_row8 + n) = pack8x4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], sc);
    }
    const int64_t nb = (n0 + wn * WTN) / kBlock8;
    if (wn % WPB == 0 && g == 0) {
      const int64_t blocks = a.out_row8 / kBlock8;
      if (nb < blocks) p.out8_scales[row * a.out_row_sc + nb] = (uint8_t)sc;
      if (nb == blocks - 1) for (int64_t b = blocks; b < a.out_row_sc; ++b) p.out8_scales[row * a.out_row_sc + b] = (uint8_t)kScaleOne;
    }
  }
}

template <int BM, int BN, int WM, int WN, int NS, bool EXACT>
hipError_t launch_tile(const Matmul8& p, hipStream_t s) {
  Args8 a = {p, row_bytes8(p.K), row_scales8(p.K), row_bytes8(p.N), row_scales8(p.N), (int)ceil_div(p.C, BM), (int)ceil_div(p.N, BN), 0, false};
  const int64_t all = p.E * p.C, total = p.counts && p.rows_hint ? (p.E * p.rows_hint < all ? p.E * p.rows_hint : all) : all;
  int64_t blocks = tile_grid(a.NT, live_row_tiles(p.E, p.C, total, BM));
  a.plain = p.E > kMaxExperts || blocks >= kMaxBlocks;
  if (a.plain) blocks = (int64_t)a.MT * a.NT;
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
  matmul8_kernel<BM, BN, WM, WN, NS, EXACT><<<dim3((unsigned)blocks, a.plain ? (unsigned)p.E : 1), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

#include "matmul8_large.h"

namespace {

// The forms that the large tile has: a plain product, with either form of B's exponents, and the experts' first one, which applies the activation and rounds to 8 bits.
bool large_covers(const Matmul8& p) {
  const int64_t tiles = p.E * ceil_div(p.C, kBig) * ceil_div(p.N, kBig);
  return p.dtype == MOE_BF16 && p.E <= kMaxExperts && tiles < kMaxBlocks && (p.out ? p.act < 0 : p.act >= 0 && p.b_blocks);
}

hipError_t launch_large(const Matmul8& p, hipStream_t s) {
  // Operands and results beyond the 256 MB of the last-level cache: stores that leave no line behind keep the operands there (128 experts x 2048 rows, 1024 x 4096 1480 -> 1340 us, 8 x
  // 4096, 4096 x 2048 222 -> 203).  Below, whoever reads the results next finds them (and the product itself is 2 % faster).
  const int64_t row8 = row_bytes8(p.K), rows = p.counts && p.rows_hint && p.rows_hint < p.C ? p.rows_hint : p.C;
  const bool stream = p.E * (rows * row8 + p.N * row8 + rows * p.N * (p.out ? 2 : 1)) > ((int64_t)256 << 20);
  Args8 a = {p, row8, row_scales8(p.K), row_bytes8(p.N), row_scales8(p.N), (int)ceil_div(p.C, kBig), (int)ceil_div(p.N, kBig), 0, stream};
  const int64_t all = p.E * p.C, total = p.counts && p.rows_hint ? (p.E * p.rows_hint < all ? p.E * p.rows_hint : all) : all;
  const dim3 grid((unsigned)tile_grid(a.NT, live_row_tiles(p.E, p.C, total, kBig), true)), block(256);
#define MOE_BIG(ACT, OUT8, BLOCKS) matmul8_large_kernel<ACT, OUT8, BLOCKS><<<grid, block, 0, s>>>(a)
  if (!p.b_blocks) MOE_BIG(-1, false, false);
  else if (p.out) MOE_BIG(-1, false, true);
  else if (p.act == MOE_ACT_RELU) MOE_BIG(MOE_ACT_RELU, true, true);
  else if (p.act == MOE_ACT_GELU) MOE_BIG(MOE_ACT_GELU, true, true);
  else MOE_BIG(MOE_ACT_SILU, true, true);
#undef MOE_BIG
  return hipGetLastError();
}

}  // namespace

hipError_t launch_matmul8(const Matmul8& p, hipStream_t s) {
  if (large_covers(p) && p.C >= 512 && p.N >= 256) return launch_large(p, s);
  return p.dtype == MOE_F32 ? launch_tile<128, 128, 2, 2, 2, true>(p, s) : launch_tile<128, 128, 2, 2, 2, false>(p, s);
}

}  // namespace moe
