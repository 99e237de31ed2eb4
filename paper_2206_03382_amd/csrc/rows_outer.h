// Weight gradients of experts with few rows each (ROWS, bf16), and how the reduction of others is shared by blocks:  out[e] = sum_r A[r]^T B[r].  Included by ragged.hip.
//
// Bound by writing the gradients: up to 64 rows are one K-step, and what a tile takes is the way to its first operands, offsets -> row numbers -> rows, not its products.  So a block has one
// stage of 64 k and no ring, 32 KB of LDS, and four of them share a unit and cover each other's waits; a longer reduction is done stage by stage.  Against the 128 x 128 tile of ffn_ring.h,
// whose rings leave room for two blocks, us: 16 tokens with 2 of 32 experts of 2048 x 1024 39 -> 23 (the gradients alone at a large copy's rate: 27), 512 with 4 of 128 of 1024 x 1024 77 -> 45
// (55), 1024 with 4 of 64 46 -> 31 (27), 8192 with 2 of 128 of 1024 x 4096 455 -> 399 (218); beyond 256 rows to an expert, or with few tiles, the rings and the 256 x 256 tile are the faster ones.
namespace {

template <bool GK>
__global__ __launch_bounds__(256, 4) void rows_outer_kernel(const TileArgs p) {
  constexpr int T = 128, WT = 64, R = WT / 16, L = T / 32;          // tile, a wave's, its fragments, its direct loads per operand and K-step
  __shared__ __attribute__((aligned(1024))) char smem[2 * T * 128];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, kq = lane >> 4;
  int e, mt, nt, rows;
  if (!find_tile<T, true>(blockIdx.x, lane, p.E, p.C, nullptr, p.NT, e, mt, nt, rows)) return;
  const int64_t m0 = (int64_t)mt * T, n0 = (int64_t)nt * T;
  const int64_t first = first_row_of<true>(e, p.K, p.kfill);        // of the expert's rows
  const int kend = live_rows_of<true>(e, p.K, p.kfill);

  // ---- direct loads: pieces of 8 columns in order, [64 k][16 pieces], piece c of k row kr at c ^ swz(kr) (as in ffn_ring.h)
  auto swz = [](int kr) -> int { return (4 * (kr & 3)) ^ (2 * ((kr >> 3) & 1)); };
  auto k_of = [&](int q) -> int { return q * 16 + wave * 4 + (lane >> 4); };
  auto source = [&](const uint16_t* base, int64_t ld, int64_t c0, int q) -> const char* {
    const int64_t col = c0 + (((lane & 15) ^ swz(k_of(q))) << 3);
    return (const char*)(base + (col < ld ? col : c0));             // columns past the end: any piece of the row
  };
  const char* zero = (const char*)g_zero_piece;
  const uint32_t smem_addr = (uint32_t)(uintptr_t)LDS_PTR(char, smem);
  f32x4 acc[R][R];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < R; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  int32_t grow[GK ? L : 1];                                         // rows of the gathered matrix, fetched a K-step ahead
  auto fetch = [&](int k0) __attribute__((always_inline)) {
    if constexpr (GK) {
#pragma unroll
      for (int q = 0; q < L; ++q) grow[q] = k0 + k_of(q) < kend ? p.gather[first + k0 + k_of(q)] : 0;
    }
  };
  fetch(0);
  for (int k0 = 0; k0 < kend; k0 += 64) {
    if (k0 > 0) __syncthreads();                                    // the stage has been read
#pragma unroll
    for (int q = 0; q < L; ++q) {
      const int64_t row = first + k0 + k_of(q);
      const bool on = k0 + k_of(q) < kend;
      const int64_t a_row = GK ? ((uint32_t)grow[GK ? q : 0] < (uint64_t)p.gather_rows ? grow[GK ? q : 0] : 0) : row;
      global_to_lds_16(on ? source((const uint16_t*)p.A, p.C, m0, q) + a_row * p.C * 2 : zero, smem_addr + (q * 4 + wave) * 1024);
      global_to_lds_16(on ? source((const uint16_t*)p.B, p.N, n0, q) + row * p.N * 2 : zero, smem_addr + T * 128 + (q * 4 + wave) * 1024);
    }
    fetch(k0 + 64);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s == 1 && kend - k0 <= 32) break;
      auto read = [&](int at, int w, int t) __attribute__((always_inline)) -> bf16x8 {
        const int kr = kq * 8 + ((lane & 15) >> 2), c = w * (WT / 8) + 2 * t + ((lane & 3) >> 1);
        const char* from = smem + at + kr * T * 2 + ((c ^ swz(kr)) << 4) + ((lane & 1) << 3) + 32 * s * T * 2;
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4v, from));
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4v, from + 4 * T * 2));
        return __builtin_bit_cast(bf16x8, (short8v)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      bf16x8 a[R];
#pragma unroll
      for (int i = 0; i < R; ++i) a[i] = read(0, wm, i);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const bf16x8 b = read(T * 128, wn, j);
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a[i], acc[i][j], 0, 0, 0);
      }
    }
  }
  __syncthreads();                                                  // the stage is done with

  // ---- results through the wave's own piece of LDS: register u of tile (i, j) is row 16 i + lane % 16, column 16 j + 4 kq + u; piece c of row r is at c ^ r % 8
  char* tile = smem + wave * (WT * WT * 2);
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int r = i * 16 + (lane & 15);
      *LDS_PTR(u32x2, tile + r * 128 + (((2 * j + (kq >> 1)) ^ (r & 7)) << 4) + 8 * (kq & 1)) =
          u32x2{pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3])};
    }
  __builtin_amdgcn_wave_barrier();
  const int64_t col = n0 + wn * WT + ((lane & 7) ^ (lane >> 3)) * 8, live = p.C - m0 - wm * WT;
  uint16_t* out = (uint16_t*)p.out + ((int64_t)e * p.C + m0 + wm * WT) * p.N;
  if (col >= p.N) return;
#pragma unroll
  for (int it = 0; it < 8; ++it) {
    const int64_t r = it * 8 + (lane >> 3);
    if (r < live) *reinterpret_cast<u32x4*>(out + r * p.N + col) = *LDS_PTR(u32x4, tile + it * 1024 + lane * 16);
  }
}

hipError_t launch_outer(TileArgs p, int64_t total, hipStream_t s) {
  dim3 grid;
  if (!tile_launch(p, 128, 128, total, grid) || p.plain) return hipErrorInvalidValue;
  if (p.gather) rows_outer_kernel<true><<<grid, dim3(256), 0, s>>>(p);
  else rows_outer_kernel<false><<<grid, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

// out = the parts' sums added up in order, n values of each; eight to a thread
template <typename OT> __global__ __launch_bounds__(256) void parts_join_kernel(const float* __restrict__ part_sums, int parts, int64_t n, OT* __restrict__ out) {
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= n) return;
  f32x4 v[2] = {};
#pragma unroll 4
  for (int u = 0; u < parts; ++u)
#pragma unroll
    for (int h = 0; h < 2; ++h) v[h] += *reinterpret_cast<const f32x4*>(part_sums + u * n + at + 4 * h);
  if constexpr (sizeof(OT) == 4) {
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(out + at + 4 * h) = v[h];
  } else {
    *reinterpret_cast<u32x4*>(out + at) = u32x4{pack_bf16x2(v[0][0], v[0][1]), pack_bf16x2(v[0][2], v[0][3]), pack_bf16x2(v[1][0], v[1][1]), pack_bf16x2(v[1][2], v[1][3])};
  }
}

hipError_t join_parts(const TileArgs& p, int dtype, hipStream_t s) {
  const int64_t n = (int64_t)p.E * p.C * p.N;
  const dim3 grid((unsigned)ceil_div(n, 2048)), block(256);
  if (dtype == MOE_F32) parts_join_kernel<float><<<grid, block, 0, s>>>(p.part_sums, p.parts, n, (float*)p.out);
  else parts_join_kernel<uint16_t><<<grid, block, 0, s>>>(p.part_sums, p.parts, n, (uint16_t*)p.out);
  return hipGetLastError();
}

}  // namespace
