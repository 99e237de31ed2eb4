// Grouped products of 8-bit matrices with a power of two for each block of 128 (block8.h):
//   out[e][r, n] = act(sum_b 2^(ea[r, b] + eb[n, b]) * sum_{k in b} A[e][r, k] * B[e][n, k] + bias[e][n])
// on v_mfma_scale_f32_16x16x128_f8f6f4: a K-step of 128 is one block of the format, both of whose exponents go into the instruction, and the sums
// stay in fp32 accumulators from the first block to the last.  Both operands have k contiguous, so a lane's 32 bytes of a fragment are two 16-byte LDS
// reads; which k they are does not matter as long as A and B agree, since the block's exponent is the same for all of them.
//
// These instructions align a step's 128 products to the largest before they add them up and lose what is 2^-16 or so of it: 1.5e-5 of the result
// (relative, 2-norm) whatever K is, which a result rounded to bf16 (1.7e-3) or to 8 bits does not show.  fp32 results go through v_mfma_f32_16x16x32_bf16 on
// the values widened to bf16, exponent included: 1e-7, at less than half the rate.  bf16 holds all of a block's values if its exponent is -124 to 119; values of blocks
// below that are rounded to multiples of 2^-133, and stored ones of 2^128 are infinities.  fp32 results are bound by those conversions, which each product of a fragment makes again: 8 experts x
// 4096 rows, 2048 x 2048 960 us = 0.29 PFLOP/s, where bf16 results take 122.
#include "block8.h"
#include "ffn_device.h"
#include "matmul8_rules.h"

namespace moe {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

// four bytes times 2^(exponent byte - 127), in bf16: without a rounding for exponents of -124 to 119
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

// The exponents of up to 64 K-steps in LDS, [word of four][row of A, then of B]: loads for them in the loop would hold up the direct loads' waits, which count in order, by all the way
// from memory.
constexpr int kScaleWords = 16;

// 128 x 128 to a block of four waves, 64 x 64 each; two blocks share a unit, one's products cover the other's waits.  Two stages of a K-step in LDS: rows of 128 bytes, 16-byte piece g of row r
// at g ^ (r / 2) % 8.  Fragments whose rows are all past the expert's fill are skipped.
// EXACT: fp32 results.  ACT: of 8-bit results; others apply p.act in its full form.
template <bool EXACT, bool OUT8, int ACT>
__global__ __launch_bounds__(256, 2) void matmul8_kernel(const Args8 a) {
  constexpr int kTile = 128, kStage = 2 * kTile * kBlock8, F = 4;
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStage + kScaleWords * 2 * kTile * 4];
  const Matmul8& p = a.p;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, fr = lane & 15, g = lane >> 4;
  int e, mt, nt, rows;
  if (!a.plain) {
    if (!find_tile<kTile>(blockIdx.x, lane, (int)p.E, p.C, p.counts, a.NT, e, mt, nt, rows)) return;
  } else {
    e = blockIdx.y;
    mt = blockIdx.x / a.NT;
    nt = blockIdx.x % a.NT;
    rows = live_rows_of(e, p.C, p.counts);
  }
  const int64_t m0 = (int64_t)mt * kTile, n0 = (int64_t)nt * kTile;
  if (m0 >= rows) return;
  const int N = (int)p.N, live = (int)(rows - m0 < kTile ? rows - m0 : kTile);
  const int own = (live - wm * 64 + 15) >> 4, frags = own < 0 ? 0 : (own < F ? own : F);       // of the wave's row fragments
  int KT = (int)(a.row8 / kBlock8);
  if (p.k_counts) {
    const int64_t c = p.k_counts[e];
    const int64_t most = c < p.K ? (c > 0 ? c : 0) : p.K;
    KT = (int)ceil_div(most, kBlock8);
  }
  auto a_row = [&](int r) -> int64_t {                              // rows past the fill repeat the last one (never stored)
    const int64_t c = (int64_t)e * p.C + (r < live ? m0 + r : rows - 1);
    if (!p.gather) return c;
    const int t = p.gather[c];
    return (unsigned)t < (uint64_t)p.gather_rows ? t : 0;
  };
  auto b_row = [&](int n) -> int64_t { return n0 + n < N ? n0 + n : N - 1; };      // so do columns past N

  // direct loads: wave w's load q brings 8 rows, lane l the piece l % 8 of row l / 8, from where the swizzle wants it
  const char* a_at[4];
  uint32_t b_at[4];
  const char* b_base = (const char*)p.B + (int64_t)e * N * a.row8;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = (q * 4 + wave) * 8 + (lane >> 3), piece = ((lane & 7) ^ ((r >> 1) & 7)) << 4;
    a_at[q] = (const char*)p.A + a_row(r) * a.row8 + piece;
    b_at[q] = (uint32_t)(b_row(r) * a.row8 + piece);
  }
  const uint32_t smem_addr = (uint32_t)(uintptr_t)LDS_PTR(char, smem);
  auto load_step = [&](int kt) {
    const uint32_t to = smem_addr + (kt & 1) * kStage + wave * 1024;
    const char* b_src = b_base + (int64_t)kt * kBlock8;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q * 32 < live) global_to_lds_16(a_at[q] + (int64_t)kt * kBlock8, to + q * 4096);
#pragma unroll
    for (int q = 0; q < 4; ++q) global_to_lds_16(b_src, b_at[q], to + kTile * kBlock8 + q * 4096);
  };
  // thread t has row t of A, or column t - 128 of B
  const uint8_t* sc_at;
  if (threadIdx.x < kTile) {
    sc_at = p.A_scales + a_row(threadIdx.x) * a.row_sc;
  } else {
    const int64_t n = b_row(threadIdx.x - kTile);
    sc_at = p.B_scales + (p.b_blocks ? (int64_t)e * ceil_div(N, kBlock8) + n / kBlock8 : (int64_t)e * N + n) * a.row_sc;
  }
  auto load_scales = [&](int first) {                               // of the K-steps from `first`, a multiple of 64
    const int left = (int)(a.row_sc - first) / 4, words = left < kScaleWords ? left : kScaleWords;
    for (int w = 0; w < words; ++w) global_to_lds_4(sc_at + first + 4 * w, smem_addr + 2 * kStage + w * 1024 + wave * 256);
  };
  f32x4 acc[F][F];
  if (KT > 0) {
    load_scales(0);
    load_step(0);
  }
#pragma unroll
  for (int j = 0; j < F; ++j) {
    const int64_t n = n0 + wn * 64 + j * 16 + 4 * g;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (p.bias && n < N) {
      const int64_t at = (int64_t)e * N + n;
      if (p.dtype == MOE_F32) v = *reinterpret_cast<const f32x4*>((const float*)p.bias + at);
      else {
        const u32x2 w = *reinterpret_cast<const u32x2*>((const uint16_t*)p.bias + at);
        v = f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
      }
    }
#pragma unroll
    for (int i = 0; i < F; ++i) acc[i][j] = v;
  }
  for (int kt = 0; kt < KT; ++kt) {
    if (kt > 0 && kt % (4 * kScaleWords) == 0) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      load_scales(kt);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (kt + 1 < KT) load_step(kt + 1);
    const char* as = smem + (kt & 1) * kStage + wm * 64 * kBlock8;
    const char* bs = smem + (kt & 1) * kStage + (kTile + wn * 64) * kBlock8;
    const char* sc = smem + 2 * kStage + (kt >> 2 & (kScaleWords - 1)) * 1024 + (kt & 3) + fr * 4;
    auto fragment = [&](const char* at, int i) -> i32x8 {
      const int sw = (fr >> 1) & 7;
      const u32x4 lo = *LDS_PTR(u32x4, at + (i * 16 + fr) * kBlock8 + ((g ^ sw) << 4));
      const u32x4 hi = *LDS_PTR(u32x4, at + (i * 16 + fr) * kBlock8 + (((g + 4) ^ sw) << 4));
      return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };
    i32x8 bv[F];
    uint32_t sb[F];
#pragma unroll
    for (int j = 0; j < F; ++j) {
      bv[j] = fragment(bs, j);
      sb[j] = *LDS_PTR(uint8_t, sc + (kTile + wn * 64 + j * 16) * 4);
    }
#pragma unroll
    for (int i = 0; i < F; ++i) {
      if (i >= frags) break;
      const i32x8 av = fragment(as, i);
      const uint32_t sa = *LDS_PTR(uint8_t, sc + (wm * 64 + i * 16) * 4);
#pragma unroll
      for (int j = 0; j < F; ++j) {
        if constexpr (EXACT) {
#pragma unroll
          for (int c = 0; c < 8; c += 2)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(bv[j][c], bv[j][c + 1], scale_value(sb[j])), widen8(av[c], av[c + 1], scale_value(sa)), acc[i][j], 0, 0, 0);
        } else {
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bv[j], av, acc[i][j], 0, 0, 0, (int)sb[j], 0, (int)sa);
        }
      }
    }
  }
  // lane (16 g + fr) has row fr of fragment i and columns 16 j + 4 g .. + 3 of its wave's part
  if constexpr (!OUT8) {
#pragma unroll
    for (int i = 0; i < F; ++i) {
      if (i >= frags) break;
      const int r = wm * 64 + i * 16 + fr;
#pragma unroll
      for (int j = 0; j < F; ++j) {
        const int64_t n = n0 + wn * 64 + j * 16 + 4 * g, at = ((int64_t)e * p.C + m0 + r) * N + n;
        f32x4 v = acc[i][j];
        if (p.act >= 0)
#pragma unroll
          for (int c = 0; c < 4; ++c) v[c] = act_full(v[c], p.act);
        if (r >= live || n >= N) continue;                          // N is a multiple of 8
        if (p.dtype == MOE_F32) *reinterpret_cast<f32x4*>((float*)p.out + at) = v;
        else *reinterpret_cast<uint2*>((uint16_t*)p.out + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
      }
    }
    return;
  }
  // 8-bit output: the block's largest magnitude over the wave's columns, then over the two waves that share the 128
  uint32_t* tops = (uint32_t*)smem;                                 // [128][2]
  __syncthreads();                                                  // every wave is done with the stages
#pragma unroll
  for (int i = 0; i < F; ++i) {
    if (i >= frags) break;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float v = acc[i][j][c];
        if constexpr (EXACT) v = p.act >= 0 ? act_full(v, p.act) : v;
        else v = act8<ACT>(v);
        if (n0 + wn * 64 + j * 16 + 4 * g >= N) v = 0.f;
        acc[i][j][c] = v;
        top = max(top, magnitude_bits(v));
      }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if (g == 0) tops[(wm * 64 + i * 16 + fr) * 2 + wn] = top;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < F; ++i) {
    if (i >= frags) break;
    const int r = wm * 64 + i * 16 + fr;
    const uint32_t sc = scale_of_amax(max(tops[2 * r], tops[2 * r + 1]));
    const float inverse = inverse_scale(sc);
    if (r >= live) continue;
    const int64_t row = (int64_t)e * p.C + m0 + r;
#pragma unroll
    for (int j = 0; j < F; ++j) {
      const int64_t n = n0 + wn * 64 + j * 16 + 4 * g;              // the block of 128 exists as a whole
      *reinterpret_cast<uint32_t*>((uint8_t*)p.out8 + row * a.out_row8 + n) = pack8x4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], inverse);
    }
    if (wn == 0 && g == 0) {
      uint8_t* to = p.out8_scales + row * a.out_row_sc;
      to[nt] = (uint8_t)sc;
      if (nt == a.NT - 1)
        for (int64_t b = a.NT; b < a.out_row_sc; ++b) to[b] = (uint8_t)kScaleOne;
    }
  }
}

hipError_t launch_small(const Matmul8& p, hipStream_t s) {
  constexpr int kTile = 128;
  Args8 a = {p, row_bytes8(p.K), row_scales8(p.K), row_bytes8(p.N), row_scales8(p.N), (int)ceil_div(p.C, kTile), (int)ceil_div(p.N, kTile), 0, false};
  const int64_t all = p.E * p.C, total = p.counts && p.rows_hint ? (p.E * p.rows_hint < all ? p.E * p.rows_hint : all) : all;
  int64_t blocks = tile_grid(a.NT, live_row_tiles(p.E, p.C, total, kTile));
  a.plain = p.E > kMaxExperts || blocks >= kMaxBlocks;
  if (a.plain) blocks = (int64_t)a.MT * a.NT;
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks, a.plain ? (unsigned)p.E : 1), block(256);
#define MOE_SMALL8(EXACT, OUT8, ACT) matmul8_kernel<EXACT, OUT8, ACT><<<grid, block, 0, s>>>(a)
  if (p.out) { if (p.dtype == MOE_F32) MOE_SMALL8(true, false, -1); else MOE_SMALL8(false, false, -1); }
  else if (p.dtype == MOE_F32) MOE_SMALL8(true, true, -1);
  else if (p.act < 0) MOE_SMALL8(false, true, -1);
  else if (p.act == MOE_ACT_RELU) MOE_SMALL8(false, true, MOE_ACT_RELU);
  else if (p.act == MOE_ACT_GELU) MOE_SMALL8(false, true, MOE_ACT_GELU);
  else MOE_SMALL8(false, true, MOE_ACT_SILU);
#undef MOE_SMALL8
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
  // Stores that leave no line behind, where operands and results are 96 MB or more of the 256 MB that the last-level cache has: what the program reads before and after a product is in
  // there too.  A training pass of 8 experts x 4096 rows, 2048 x 2048 (235 MB a product) 524 -> 482 us, x 2048 rows (134 MB) 284 -> 275, 64 x 512, 1024 x 1024 (168 MB) 272 -> 250,
  // 8 x 1024, 2048 x 2048 (84 MB) 167 -> 169; a product of 128 x 2048, 1024 x 4096 1480 -> 1340.
  const int64_t row8 = row_bytes8(p.K), rows = p.counts && p.rows_hint && p.rows_hint < p.C ? p.rows_hint : p.C;
  const bool stream = p.E * (rows * row8 + p.N * row8 + rows * p.N * (p.out ? 2 : 1)) >= ((int64_t)96 << 20);
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
  const int64_t rows = p.counts && p.rows_hint > 0 && p.rows_hint < p.C ? p.rows_hint : p.C;
  if (large_covers(p) && matmul8_takes_large_tile(p.E, (double)rows, p.K, p.N)) return launch_large(p, s);
  return launch_small(p, s);
}

}  // namespace moe
