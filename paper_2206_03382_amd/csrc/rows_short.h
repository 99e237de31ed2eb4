// Products of experts' rows over few columns (ROWS, bf16, kNN and kNT):  out[r] = act(A[r] W[e] + bias[e]) + residual[r],  out[r] = A[r] W[e]^T (* act'(pre[r])).  Included by ragged.hip.
//
// With a short reduction a tile is mostly the way to its first operands and its results, and what it needs is other tiles on the unit meanwhile: one stage of 64 k, 32 KB of LDS, four
// blocks to a unit, as in rows_outer.h; K-steps follow each other without a load in advance.  Above all one block's results (activation, what they are joined with, stores) hide behind the
// others' products, which blocks of the large tiles, one or two to a unit, do one after the other.  us, with the tile that choose_tile names and here: 90820 rows of 16 experts,
// 256 x 512 47.1 and 43.6, with GeLU and kept values 84.8 and 60.9, times GeLU' 93.8 and 64.3; 512 x 512 64.1 and 64.0, 102 and 91.3, 111 and 92.7; 32768 x 776 x 2048 of 8 experts with GeLU
// and kept values 196 and 170; with 1536 columns 250 and 269.
namespace {

template <int MODE>
__global__ __launch_bounds__(256, 4) void rows_short_kernel(const TileArgs p) {
  constexpr int T = 128, WT = 64, R = WT / 16, L = T / 32;          // tile, a wave's, its fragments, its direct loads per operand and K-step
  __shared__ __attribute__((aligned(1024))) char smem[2 * T * 128];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, kq = lane >> 4;
  int e, mt, nt, rows;
  if (!find_tile<T, false, 0, false, true>(blockIdx.x, lane, p.E, p.C, p.counts, p.NT, e, mt, nt, rows)) return;
  const int64_t m0 = (int64_t)mt * T, n0 = (int64_t)nt * T;
  if (m0 >= rows) return;
  const int64_t first = first_row_of<true>(e, p.C, p.counts), live = rows - m0 - wm * WT, nw = n0 + wn * WT;

  // ---- direct loads.  k-contiguous: 8 rows, piece g of row r at g ^ (r / 2 % 8).  k-slow: [64 k][16 pieces], piece c of k row kr at c ^ swz(kr)
  auto swz = [](int kr) -> int { return (4 * (kr & 3)) ^ (2 * ((kr >> 3) & 1)); };
  const int fast_k = ((lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7)) * 8;
  const char* a_ptr[L];
  const char* b_ptr[L];
#pragma unroll
  for (int q = 0; q < L; ++q) {
    const int r = (q * 4 + wave) * 8 + (lane >> 3);
    int64_t row = first + (m0 + r < rows ? m0 + r : rows - 1);      // rows past the fill repeat the last one
    if (MODE == kNN && p.gather) {
      const int64_t t = p.gather[row];
      row = t >= 0 && t < p.gather_rows ? t : 0;
    }
    a_ptr[q] = (const char*)((const uint16_t*)p.A + row * p.K + fast_k);
    const uint16_t* w = (const uint16_t*)p.B + (int64_t)e * p.K * p.N;
    if (MODE == kNN) {
      const int kr = q * 16 + wave * 4 + (lane >> 4);
      const int64_t col = n0 + (((lane & 15) ^ swz(kr)) << 3);
      b_ptr[q] = (const char*)(w + (int64_t)kr * p.N + (col < p.N ? col : n0));    // columns past the end: any piece of the row
    } else {
      b_ptr[q] = (const char*)(w + (n0 + r < p.N ? n0 + r : p.N - 1) * p.K + fast_k);
    }
  }
  const int64_t b_step = MODE == kNN ? 128 * (int64_t)p.N : 128;
  const char* zero = (const char*)g_zero_piece;
  const uint32_t smem_addr = (uint32_t)(uintptr_t)LDS_PTR(char, smem);
  const bool has_bias = MODE == kNN && p.bias != nullptr;
  u32x2 braw[R];
  if (has_bias) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int64_t col = nw + j * 16 + 4 * kq;
      braw[j] = *reinterpret_cast<const u32x2*>((const uint16_t*)p.bias + (int64_t)e * p.N + (col < p.N ? col : n0));
    }
  }
  f32x4 acc[R][R];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < R; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int K = (int)p.K;
  for (int k0 = 0; k0 < K; k0 += 64) {
    if (k0 > 0) __syncthreads();                                    // the stage has been read
#pragma unroll
    for (int q = 0; q < L; ++q) {
      const int b_k = MODE == kNN ? q * 16 + wave * 4 + (lane >> 4) : fast_k;
      global_to_lds_16(k0 + fast_k < K ? a_ptr[q] : zero, smem_addr + (q * 4 + wave) * 1024);
      global_to_lds_16(k0 + b_k < K ? b_ptr[q] : zero, smem_addr + T * 128 + (q * 4 + wave) * 1024);
      a_ptr[q] += 128;
      b_ptr[q] += b_step;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (live <= 0) continue;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s == 1 && K - k0 <= 32) break;
      bf16x8 a[R];
#pragma unroll
      for (int i = 0; i < R; ++i) a[i] = *LDS_PTR(bf16x8, smem + (wm * WT + i * 16 + (lane & 15)) * 128 + (((4 * s + kq) ^ ((lane & 15) >> 1)) << 4));
#pragma unroll
      for (int j = 0; j < R; ++j) {
        bf16x8 b;
        if (MODE == kNN) {
          const int kr = kq * 8 + ((lane & 15) >> 2), c = wn * (WT / 8) + 2 * j + ((lane & 3) >> 1);
          const char* from = smem + T * 128 + kr * T * 2 + ((c ^ swz(kr)) << 4) + ((lane & 1) << 3) + 32 * s * T * 2;
          const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4v, from));
          const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4v, from + 4 * T * 2));
          b = __builtin_bit_cast(bf16x8, (short8v)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
          b = *LDS_PTR(bf16x8, smem + T * 128 + (wn * WT + j * 16 + (lane & 15)) * 128 + (((4 * s + kq) ^ ((lane & 15) >> 1)) << 4));
        }
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a[i], acc[i][j], 0, 0, 0);
      }
    }
  }
  __syncthreads();                                                  // the stage is done with
  if (live <= 0) return;                                            // no barrier follows

  // ---- results through the wave's own piece of LDS: register u of tile (i, j) is row 16 i + lane % 16, column 16 j + 4 kq + u; piece c of row r is at c ^ r % 8.  What the sums are
  // joined with comes into the same places before, by direct loads; a lane joins its own.
  char* tile = smem + wave * (WT * WT * 2);
  const uint32_t tile_addr = smem_addr + wave * (WT * WT * 2);
  const int64_t col = nw + ((lane & 7) ^ (lane >> 3)) * 8, out_at = (first + m0 + wm * WT) * p.N;
  const bool col_on = col < p.N;
  auto write_rows = [&](auto act_tag, uint16_t* dst, const uint16_t* with) __attribute__((always_inline)) {
    constexpr int ACT = decltype(act_tag)::value;
    if (with) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int64_t r = it * 8 + (lane >> 3);
        global_to_lds_16((const char*)(with + out_at + (r < live ? r : 0) * p.N + (col_on ? col : n0)), tile_addr + it * 1024);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = i * 16 + (lane & 15);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        auto* at = LDS_PTR(u32x2, tile + r * 128 + (((2 * j + (kq >> 1)) ^ (r & 7)) << 4) + 8 * (kq & 1));
        float v[4], w[4] = {0.f, 0.f, 0.f, 0.f};
        if (with) {
          const u32x2 x = *at;
          w[0] = __uint_as_float(x.x << 16); w[1] = __uint_as_float(x.x & 0xffff0000u);
          w[2] = __uint_as_float(x.y << 16); w[3] = __uint_as_float(x.y & 0xffff0000u);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (MODE == kNT) v[u] = with ? acc[i][j][u] * rows_act_grad<ACT>(w[u]) : acc[i][j][u];
          else v[u] = rows_act<ACT>(acc[i][j][u]) + (with ? w[u] : 0.f);
        }
        *at = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      }
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int64_t r = it * 8 + (lane >> 3);
      if (r < live && col_on) *reinterpret_cast<u32x4*>(dst + out_at + r * p.N + col) = *LDS_PTR(u32x4, tile + it * 1024 + lane * 16);
    }
    __builtin_amdgcn_wave_barrier();
  };
  if (has_bias) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const f32x4 b = {__uint_as_float(braw[j].x << 16), __uint_as_float(braw[j].x & 0xffff0000u), __uint_as_float(braw[j].y << 16), __uint_as_float(braw[j].y & 0xffff0000u)};
#pragma unroll
      for (int i = 0; i < R; ++i) acc[i][j] += b;
    }
  }
  const uint16_t* with = (const uint16_t*)p.pre;
  if (MODE == kNN && p.pre_out) write_rows(std::integral_constant<int, -1>{}, (uint16_t*)p.pre_out, nullptr);
  switch (p.act) {
    case MOE_ACT_RELU: write_rows(std::integral_constant<int, MOE_ACT_RELU>{}, (uint16_t*)p.out, with); break;
    case MOE_ACT_GELU: write_rows(std::integral_constant<int, MOE_ACT_GELU>{}, (uint16_t*)p.out, with); break;
    case MOE_ACT_SILU: write_rows(std::integral_constant<int, MOE_ACT_SILU>{}, (uint16_t*)p.out, with); break;
    default: write_rows(std::integral_constant<int, -1>{}, (uint16_t*)p.out, with); break;
  }
}

template <int MODE> hipError_t launch_short(TileArgs p, int64_t total, hipStream_t s) {
  dim3 grid;
  if (!tile_launch(p, 128, 128, total, grid) || p.plain) return hipErrorInvalidValue;
  rows_short_kernel<MODE><<<grid, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace
