// Products of experts' rows (ROWS, forward layout, bf16) where there are few rows and reading the weights is all the time there is.  Included by ragged.hip.
//
//   out[r] = act(A[r] W[e] + bias[e]) + residual[r]
//
// A block has 16 RI rows of an expert and a strip of 64 columns, and cuts the reduction itself: each of four waves takes every fourth K-step of 64 k through two LDS stages of its own,
// filled by direct loads, so that no wave waits for another until their sums meet in LDS, where they are added up in the waves' order.  Where that leaves units without a block and the
// reduction is long (thin_plan), blocks share a tile's K-steps as well and write their sums to memory, and a second launch adds those up in the blocks' order.
//
// Bound by the weights' way from HBM, and at the smallest sizes by the launches.  us, against the better of the 64-wide tiles of ffn_tile.h, whose blocks take the whole reduction in one
// chain (each call made from the host, which takes 6.5 us a launch): 1 x 4096 x 4096 12.2 and 19.0 (weights alone at a large copy's rate: 6.8), 16 rows 12.6 and 20.3, 64 16.4 and 24.1,
// 128 20.0 and 23.7; 1 x 4096 x 1024 9.5 and 16.7, 128 rows 9.9 and 17.9, 384 15.3 and 18.2; 16 x 2048 x 2048 8.0 and 10.3, 256 rows 9.5 and 11.0; 8 rows of as many of 128 experts,
// 4096 x 1024 16.8 and 19.1.  Strips of 16 and 32 columns with more waves were within 5 % at 2048 x 2048 and slower where weights count (13.0 at 1 x 4096 x 4096); loads with the
// nontemporal hint, or three stages, made no difference.
//
// LDS layouts of a stage: A [16 RI rows][8 pieces of 8 k], piece g of row r at g ^ (r / 2 % 8), as in the large tile; W [64 k][8 pieces of 8 columns], swizzled so that a transposing
// read's four k rows lie in different 64-byte windows modulo 256 and the two blocks of lanes that share a cycle, 8 k apart, in different halves of them.
namespace {

constexpr int kThinStages = 2;

__device__ __forceinline__ int thin_swz(int kr) { return (4 * ((kr >> 1) & 1)) ^ (2 * ((kr >> 3) & 1)); }        // piece c of k row kr is at c ^ thin_swz(kr)

// bias, activation, residual: four columns of a row, whose sums are v
__device__ __forceinline__ void thin_result(const TileArgs& p, int e, int64_t col, int64_t to, f32x4 v) {
  auto four = [](const void* at, int64_t i) __attribute__((always_inline)) -> f32x4 {
    const u32x2 b = *reinterpret_cast<const u32x2*>((const uint16_t*)at + i);
    return f32x4{__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xffff0000u), __uint_as_float(b.y << 16), __uint_as_float(b.y & 0xffff0000u)};
  };
  auto put = [&](void* at) __attribute__((always_inline)) {
    *reinterpret_cast<u32x2*>((uint16_t*)at + to) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  };
  if (p.bias) v += four(p.bias, (int64_t)e * p.N + col);
  if (p.pre_out) put(p.pre_out);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    switch (p.act) {
      case MOE_ACT_RELU: v[u] = rows_act<MOE_ACT_RELU>(v[u]); break;
      case MOE_ACT_GELU: v[u] = rows_act<MOE_ACT_GELU>(v[u]); break;
      case MOE_ACT_SILU: v[u] = rows_act<MOE_ACT_SILU>(v[u]); break;
      default: break;
    }
  }
  if (p.pre) v += four(p.pre, to);
  put(p.out);
}

// One expert: the parts' sums of a row, [part][R][N], added up in order; a block to 1024 columns of a row.
__global__ __launch_bounds__(256) void thin_join_kernel(const TileArgs p, int parts, const float* __restrict__ part_sums) {
  const int row = blockIdx.x;
  const int64_t col = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
  if (col >= p.N) return;
  const int64_t to = (int64_t)row * p.N + col, apart = p.C * p.N;
  f32x4 v = *reinterpret_cast<const f32x4*>(part_sums + to);
#pragma unroll 8
  for (int u = 1; u < parts; ++u) v += *reinterpret_cast<const f32x4*>(part_sums + u * apart + to);
  thin_result(p, 0, col, to, v);
}

template <int RI>
__global__ __launch_bounds__(kThinWaves * 64) void rows_thin_kernel(const TileArgs p, int parts, float* __restrict__ part_sums) {
  constexpr int CJ = kThinColumns / 16, NW = kThinWaves, D = kThinStages;
  constexpr int RT = 16 * RI, NC = kThinColumns;
  constexpr int LA = 2 * RI, LB = 2 * CJ, L = LA + LB, STAGE = (RI + CJ) * 2048, RING = NW * D * STAGE;
  constexpr int SUMS = NW * RT * NC * 4;
  __shared__ __attribute__((aligned(1024))) char smem[RING > SUMS ? RING : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kq = lane >> 4;
  int e, mt, nt, rows;
  const int part = blockIdx.y;
  if (p.counts) {
    if (!find_tile<RT, false, 0, false, true>(blockIdx.x, lane, p.E, p.C, p.counts, p.NT, e, mt, nt, rows)) return;
  } else {                                                          // one expert: runs of an eighth to an XCD, a strip's row tiles next to each other
    const int n = p.MT * p.NT, x = blockIdx.x % 8, at = (int)((int64_t)x * n / 8) + (int)(blockIdx.x / 8);
    if (at >= (int)((int64_t)(x + 1) * n / 8)) return;
    e = 0;
    mt = at % p.MT;
    nt = at / p.MT;
    rows = (int)p.C;
  }
  const int64_t first = first_row_of<true>(e, p.C, p.counts);
  const int64_t m0 = (int64_t)mt * RT, n0 = (int64_t)nt * NC;
  if (m0 >= rows) return;
  const int KT = (int)((p.K + kThinK - 1) / kThinK);
  const int turn = part * NW + wave, turns = parts * NW;            // this wave's among all that share the tile
  const int mine = turn < KT ? (KT - 1 - turn) / turns + 1 : 0;     // its K-steps

  const char* a_ptr[LA];
  const char* b_ptr[LB];
  int a_k[LA], b_k[LB];
#pragma unroll
  for (int q = 0; q < LA; ++q) {                                    // 8 rows each
    const int r = q * 8 + (lane >> 3), g = (lane & 7) ^ ((r >> 1) & 7);
    int64_t row = m0 + r < rows ? first + m0 + r : first + rows - 1;               // rows past the fill repeat the last one (never stored)
    if (p.gather) {
      const int64_t t = p.gather[row];
      row = t >= 0 && t < p.gather_rows ? t : 0;
    }
    a_k[q] = turn * kThinK + g * 8;
    a_ptr[q] = (const char*)((const uint16_t*)p.A + row * p.K + a_k[q]);
  }
  const uint16_t* w = (const uint16_t*)p.B + (int64_t)e * p.K * p.N;
#pragma unroll
  for (int q = 0; q < LB; ++q) {                                    // 8 k rows each
    const int kr = q * 8 + (lane >> 3);
    const int64_t col = n0 + ((lane & 7) ^ thin_swz(kr)) * 8;
    b_k[q] = turn * kThinK + kr;
    b_ptr[q] = (const char*)(w + (int64_t)b_k[q] * p.N + (col < p.N ? col : n0));
  }
  const uint32_t smem_addr = (uint32_t)(uintptr_t)LDS_PTR(char, smem) + wave * (D * STAGE);
  const char* own = smem + wave * (D * STAGE);
  const char* zero = (const char*)g_zero_piece;
  const int64_t a_step = (int64_t)turns * kThinK * 2, b_step = (int64_t)turns * kThinK * p.N * 2;
  auto issue = [&](int t) __attribute__((always_inline)) {          // the wave's K-step t, ascending; zeros past the end of the reduction
    const uint32_t dst = smem_addr + (uint32_t)(t % D) * STAGE;
    const int left = (int)p.K - t * (turns * kThinK);
#pragma unroll
    for (int q = 0; q < LB; ++q) { global_to_lds_16(b_k[q] < left ? b_ptr[q] : zero, dst + RI * 2048 + q * 1024); b_ptr[q] += b_step; }
#pragma unroll
    for (int q = 0; q < LA; ++q) { global_to_lds_16(a_k[q] < left ? a_ptr[q] : zero, dst + q * 1024); a_ptr[q] += a_step; }
  };
#pragma unroll
  for (int t = 0; t < D; ++t)
    if (t < mine) issue(t);
  f32x4 acc[RI][CJ];
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int j = 0; j < CJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int t = 0; t < mine; ++t) {
    wait_for_loads<D - 1, L>(mine - 1 - t);
    const char* at = own + t % D * STAGE;
    bf16x8 a[2][RI], b[2][CJ];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int j = 0; j < CJ; ++j) {
        short4v half[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int kr = 32 * s + kq * 8 + 4 * h + ((lane & 15) >> 2);
          half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(short4v, at + RI * 2048 + kr * 128 + (((2 * j + ((lane & 3) >> 1)) ^ thin_swz(kr)) << 4) + ((lane & 1) << 3)));
        }
        b[s][j] = __builtin_bit_cast(bf16x8, (short8v)__builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
      }
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        const int r = i * 16 + (lane & 15);
        a[s][i] = *LDS_PTR(bf16x8, at + r * 128 + (((4 * s + kq) ^ ((r >> 1) & 7)) << 4));
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // the stage has been read
    PIN();
    if (t + D < mine) issue(t + D);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int j = 0; j < CJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[s][j], a[s][i], acc[i][j], 0, 0, 0);
  }
  __syncthreads();                                                  // all stages are done with
  // [wave][row][column]; a lane has columns 16 j + 4 kq .. + 3 of row 16 i + lane % 16
  float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int j = 0; j < CJ; ++j)
      *LDS_PTR(f32x4, sums + (wave * RT + i * 16 + (lane & 15)) * NC + j * 16 + 4 * kq) = acc[i][j];
  __syncthreads();
  for (int at = threadIdx.x; at < RT * NC / 4; at += NW * 64) {
    const int r = at / (NC / 4), c = at % (NC / 4) * 4;
    const int64_t row = m0 + r, col = n0 + c;
    if (row >= rows || col >= p.N) continue;
    f32x4 v = *LDS_PTR(f32x4, sums + r * NC + c);
#pragma unroll
    for (int u = 1; u < NW; ++u) v += *LDS_PTR(f32x4, sums + (u * RT + r) * NC + c);
    const int64_t to = (first + row) * p.N + col;
    if (parts > 1) *reinterpret_cast<f32x4*>(part_sums + ((int64_t)part * p.C * p.N + to)) = v;
    else thin_result(p, e, col, to, v);
  }
}

template <int RI> hipError_t launch_thin_as(TileArgs t, int parts, float* part_sums, hipStream_t s) {
  t.MT = (int)ceil_div(t.C, 16 * RI);
  t.NT = (int)ceil_div(t.N, kThinColumns);
  const int64_t blocks = t.counts ? tile_grid(t.NT, live_row_tiles(t.E, t.C, t.C, 16 * RI)) : ceil_div((int64_t)t.MT * t.NT, 8) * 8;
  if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
  rows_thin_kernel<RI><<<dim3((unsigned)blocks, (unsigned)parts), dim3(kThinWaves * 64), 0, s>>>(t, parts, part_sums);
  if (parts > 1) {
    if (hipError_t err = hipGetLastError()) return err;
    thin_join_kernel<<<dim3((unsigned)t.C, (unsigned)ceil_div(t.N, 1024)), dim3(256), 0, s>>>(t, parts, part_sums);
  }
  return hipGetLastError();
}

hipError_t launch_thin(const TileArgs& t, const RowsPlan& plan, float* part_sums, hipStream_t s) {
  if (plan.ri == 1) return launch_thin_as<1>(t, plan.parts, part_sums, s);
  if (plan.ri == 2) return launch_thin_as<2>(t, plan.parts, part_sums, s);
  return launch_thin_as<4>(t, plan.parts, part_sums, s);
}

}  // namespace
