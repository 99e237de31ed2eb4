// fp32 products of experts' rows (ROWS) in the layouts kNN, kNT and kTN, on tiles of 64 x 64.  Included by ragged.hip.
//
//   kNN  out[r] = act(A[r] W[e] + bias[e]) + residual[r]      kNT  out[r] = A[r] W[e]^T (* act'(pre[r]))      kTN  out[e] = sum_r A[r]^T B[r]
//
// Bound by the matrix cores (v_mfma_f32_16x16x4_f32: 64 products a cycle and SIMD, 157 TFLOP/s), and at few tiles by how they divide among 256 units.  What feeds them: four waves of 32 x 32
// as 2 x 2 independent chains of sums, every matrix instruction followed by the LDS reads and direct loads that are due there and by next to no address arithmetic.  Read in a bunch
// ahead of 32 x 32 x 2 instructions, as in ffn_tile.h, each bunch costs a wave the length of an instruction: in a loop of nothing else, one block to a unit, 111 TFLOP/s there, 129 here;
// three 122 and 139.  us there and here: 1001 x 776 x 1544 33.8 and 31.9 (400 tiles: two to a unit at most), 3000 rows 83 and 72, its weight gradient 77 and 70, 4096 x 2048 x 2048 304 and 256
// (134 TFLOP/s), 8192 rows 573 and 509; 16 tokens, 2 of 32 experts of 2048 x 1024 73 and 43 (weights of the experts that are met at a large copy's rate: 36), their dx 48 and 29, dW 75 and
// 78.
//
// LDS ring of two stages of 32 k, filled by direct loads (three, which leave room for three blocks instead of five, were no faster and 20 % slower where dW is small sums, many writes).  What a lane takes as one matrix instruction's k is free as long as both operands agree: instruction u of a sub-step of 16
// k has k = 4 (lane / 16) + u, so that a k-contiguous operand is read 16 bytes at a time, for four instructions.  Likewise which rows make up a fragment: lane l's are 2 (l % 16)
// and the next of the wave's, one to each of its two fragments, so that a k-slow operand comes two words at a time and a lane ends up with 8 columns next to each other, which it stores as they
// are.  (A k-contiguous A's fragments are 16 rows next to each other: those that no expert's row fills are left out.)
//   k-contiguous operand: [64 rows][8 pieces of 4 k], piece g of row r at g ^ (r / 2 % 8)
//   k-slow operand: [32 k][64 columns], whose halves change places every 4 k, so that the lanes of two k rows that share a cycle cover all banks
namespace {

template <int MODE, bool GK>
__global__ __launch_bounds__(256, 5) void rows_fp32_kernel(const TileArgs p) {
  constexpr bool TRA = MODE == kTN, TRB = MODE != kNT;              // k-slow operands
  constexpr int R = 2, T = 32 * R, WT = 16 * R, BKE = 32, NS = 2;  // fragments of a wave, tile, wave's tile, k of a K-step, stages
  constexpr int HALF_STAGE = T * 128, STAGE = 2 * HALF_STAGE, L = T / 32;          // direct loads per wave, operand and K-step
  using Words = __attribute__((ext_vector_type(R))) float;
  __shared__ __attribute__((aligned(1024))) char smem[NS * STAGE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, kq = lane >> 4, l16 = lane & 15;
  int e, mt, nt, rows;
  if (!find_tile<T, MODE == kTN, 0, false, MODE != kTN>(blockIdx.x, lane, p.E, p.C, p.counts, p.NT, e, mt, nt, rows)) return;
  const int64_t m0 = (int64_t)mt * T, n0 = (int64_t)nt * T;
  if (m0 >= rows) return;
  int64_t kend = MODE == kTN ? live_rows_of<true>(e, p.K, p.kfill) : p.K;
  int64_t first = MODE == kTN ? first_row_of<true>(e, p.K, p.kfill) : first_row_of<true>(e, p.C, p.counts);      // of the expert's rows
  if (MODE == kTN && p.parts > 1) {                                 // this block's share of the reduction
    const int64_t each = ((kend + BKE - 1) / BKE + p.parts - 1) / p.parts * BKE, from = blockIdx.z * each < kend ? blockIdx.z * each : kend;
    first += from;
    kend = kend - from < each ? kend - from : each;
  }
  const int64_t tile_at = (MODE == kTN ? ((p.parts > 1 ? (int64_t)blockIdx.z * p.E : 0) + e) * p.C : first) + m0;        // its first row among the results'
  if (MODE == kTN && kend <= 0) {                                   // no rows: zeros, at once (16 such experts of 776 x 1544: 15 us, by way of a K-step of zeros 28)
    float* out = p.parts > 1 ? p.part_sums : (float*)p.out;
    const int64_t col = n0 + (threadIdx.x & 15) * 4;
#pragma unroll
    for (int q = 0; q < T / 16; ++q) {
      const int r = q * 16 + (int)(threadIdx.x >> 4);
      if (m0 + r < p.C && col < p.N) *reinterpret_cast<f32x4*>(out + (tile_at + r) * p.N + col) = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    return;
  }
  const int KT = (int)((kend + BKE - 1) / BKE);

  // ---- this lane's direct loads.  k-contiguous: block q * 4 + wave = 8 rows, lane l row + l / 8, position l % 8.  k-slow: pieces of 4 columns in order.
  auto fast_row = [&](int q) -> int { return (q * 4 + wave) * 8 + (lane >> 3); };
  auto fast_k = [&](int q) -> int { return ((lane & 7) ^ (fast_row(q) / R & 7)) * 4; };
  auto slow_k = [&](int q) -> int { return ((q * 4 + wave) * 64 + lane) / (T / 4); };
  auto swz_slow = [](int kr) -> int { return 8 * ((kr >> 2) & 1); };
  auto slow_source = [&](const float* base, int64_t ld, int64_t c0, int q) -> const char* {
    const int kr = slow_k(q);
    const int64_t col = c0 + ((((q * 4 + wave) * 64 + lane) % (T / 4)) ^ swz_slow(kr)) * 4;
    return (const char*)(base + (int64_t)kr * ld + (col < ld ? col : c0));          // columns past the end: any piece of the row
  };
  const char* a_ptr[L];
  const char* b_ptr[L];
#pragma unroll
  for (int q = 0; q < L; ++q) {
    if (TRA) {
      a_ptr[q] = slow_source((const float*)p.A + (GK ? 0 : first * p.C), p.C, m0, q);
      if (GK) a_ptr[q] -= (int64_t)slow_k(q) * p.C * 4;             // of row 0 of the gathered matrix
    } else {
      int64_t row = m0 + fast_row(q);
      row = first + (row < rows ? row : rows - 1);                  // rows past the fill repeat the last one
      if (p.gather) {
        const int64_t t = p.gather[row];
        row = t >= 0 && t < p.gather_rows ? t : 0;
      }
      a_ptr[q] = (const char*)((const float*)p.A + row * p.K + fast_k(q));
    }
    const float* b = (const float*)p.B + (MODE == kTN ? first : (int64_t)e * p.K) * p.N;
    if (TRB) {
      b_ptr[q] = slow_source(b, p.N, n0, q);
    } else {
      const int64_t row = n0 + fast_row(q);
      b_ptr[q] = (const char*)(b + (row < p.N ? row : p.N - 1) * p.K + fast_k(q));
    }
  }
  const int64_t a_step = TRA ? (int64_t)BKE * p.C * 4 : 128, b_step = TRB ? (int64_t)BKE * p.N * 4 : 128;
  const uint32_t smem_addr = (uint32_t)(uintptr_t)LDS_PTR(char, smem);
  const char* zero = (const char*)g_zero_piece;
  // ahead of the loads of the last K-step: what lies past the end of the reduction is read as zeros
  auto end_loads = [&](int left) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < L; ++q) {
      if (!GK) a_ptr[q] = (TRA ? slow_k(q) : fast_k(q)) < left ? a_ptr[q] : zero;
      b_ptr[q] = (TRB ? slow_k(q) : fast_k(q)) < left ? b_ptr[q] : zero;
    }
  };
  // gathered A: the rows of a K-step are fetched (plain loads) a K-step before its loads go out, and turned into addresses behind a wait for everything in flight
  using Rows = int[GK ? L : 1];
  using Sources = const char*[GK ? L : 1];
  Rows grow;
  Sources a_row;
  auto gather_fetch = [&](int t, Rows& to) __attribute__((always_inline)) {
    if constexpr (GK) {
#pragma unroll
      for (int q = 0; q < L; ++q) {
        const int64_t slot = (int64_t)t * BKE + slow_k(q), last = p.K - 1 - first;
        to[q] = p.gather[first + (slot < last ? slot : last)];
      }
    }
  };
  auto gather_resolve = [&](int t, const Rows& from, Sources& to) __attribute__((always_inline)) {
    if constexpr (GK) {
#pragma unroll
      for (int q = 0; q < L; ++q) {
        const char* at = a_ptr[q] + (int64_t)((uint32_t)from[q] < (uint64_t)p.gather_rows ? from[q] : 0) * p.C * 4;
        to[q] = (int64_t)t * BKE + slow_k(q) < kend ? at : zero;
      }
    }
  };
  auto load = [&](int n, const Sources& rows_of_a, uint32_t stage) __attribute__((always_inline)) {        // load n of 2 L of a K-step, into the stage at that address
    if (n < L) {
      global_to_lds_16(GK ? rows_of_a[GK ? n : 0] : a_ptr[n], stage + (n * 4 + wave) * 1024);
      if (!GK) a_ptr[n] += a_step;
    } else {
      const int q = n - L;
      global_to_lds_16(b_ptr[q], stage + HALF_STAGE + (q * 4 + wave) * 1024);
      b_ptr[q] += b_step;
    }
  };

  // ---- fragments: k-contiguous ones [fragment][u], k-slow ones [u][fragment]
  constexpr int NA = TRA ? 4 : R, NB = TRB ? 4 : R;                 // reads of a sub-step
  using PieceA = std::conditional_t<TRA, Words, f32x4>;
  using PieceB = std::conditional_t<TRB, Words, f32x4>;
  PieceA fa[2][NA];
  PieceB fb[2][NB];
  // LDS offsets of this lane's reads in a stage, by sub-step
  uint32_t a_at[2], b_at[2];
  auto read_at = [&](bool slow, int w, int row, int s) -> uint32_t {
    if (slow) {                                                     // k rows 16 s + 4 kq + u, whose swizzle u does not change
      const int kr = 16 * s + 4 * kq, c = w * WT + R * l16;
      return (uint32_t)(kr * T * 4 + ((c / 4) ^ swz_slow(kr)) * 16 + c % 4 * 4);
    }
    const int r = w * WT + row;
    return (uint32_t)(r * 128 + (((4 * s + kq) ^ (r / R & 7)) << 4));
  };
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    a_at[s] = read_at(TRA, wm, l16, s);
    b_at[s] = HALF_STAGE + read_at(TRB, wn, R * l16, s);
  }
  f32x4 acc[R][R];
  // rows of this wave that exist; of a k-contiguous A, fragments without any are left out
  const int64_t live = rows - m0 - wm * WT;
  auto main_loop = [&](auto ni_tag) __attribute__((always_inline)) {
    constexpr int NI = decltype(ni_tag)::value;
    auto read = [&](const char* stage, int s, int r, int d) __attribute__((always_inline)) {       // the k-contiguous ones first: all of them are needed from the start
      const bool is_a = TRA ? r >= NB : r < NA;
      const int n = TRA ? (is_a ? r - NB : r) : (is_a ? r : r - NA);
      if (NI == 0 || (is_a && !TRA && n >= NI)) return;
      if (is_a) fa[d][n] = *LDS_PTR(PieceA, stage + a_at[s] + n * (TRA ? T * 4 : 16 * 128));
      else fb[d][n] = *LDS_PTR(PieceB, stage + b_at[s] + n * (TRB ? T * 4 : 128));
    };
    constexpr int NM = 4 * R * R;                                   // matrix instructions of a sub-step, two to a K-step
    auto mfma = [&](int m, int d) __attribute__((always_inline)) {
      const int u = m / (R * R), i = m / R % R, j = m % R;
      if (i >= NI) return;
      const float a = TRA ? fa[d][TRA ? u : 0][TRA ? i : 0] : fa[d][TRA ? 0 : i][TRA ? 0 : u];
      const float b = TRB ? fb[d][TRB ? u : 0][TRB ? j : 0] : fb[d][TRB ? 0 : j][TRB ? 0 : u];
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b, a, acc[i][j], 0, 0, 0);
    };
    // The next sub-step's reads go out behind the first three quarters of a sub-step's products.  Behind seven eighths of sub-step 0 the stage is read and handed over, and its loads
    // of the K-step NS ahead go out behind the products that are left.
    constexpr int NR = NA + NB, SPAN = NM * 3 / 4, BAR = NM * 7 / 8, GAP = (2 * NM - BAR) / (2 * L);
    auto kstep = [&](auto dma_tag, int kt, uint32_t cur, uint32_t nxt) __attribute__((always_inline)) {
      constexpr bool DMA = decltype(dma_tag)::value;                  // K-step kt + NS exists
      if (DMA && kt + NS == KT - 1) end_loads((int)(kend - (int64_t)(kt + NS) * BKE));
#pragma unroll
      for (int m = 0; m < 2 * NM; ++m) {
        const int s = m / NM, at = m % NM;
        mfma(at, s);
        PIN();
#pragma unroll
        for (int r = (at * NR + SPAN - 1) / SPAN; r < ((at + 1) * NR + SPAN - 1) / SPAN; ++r)
          if (r < NR) read(smem + (s == 0 ? cur : nxt), 1 - s, r, 1 - s);
        if (m == BAR) {                                               // K-step kt + 1 has landed
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
          PIN();
          asm volatile("s_barrier" ::: "memory");
          PIN();
          if (DMA) {
            gather_resolve(kt + NS, grow, a_row);
            gather_fetch(kt + NS + 1, grow);
            PIN();
          }
        }
        if (DMA && m >= BAR && (m - BAR) % GAP == 0 && (m - BAR) / GAP < 2 * L) load((m - BAR) / GAP, a_row, smem_addr + cur);
        PIN();
      }
    };
    {
      Rows g[NS];
      Sources from[NS];
#pragma unroll
      for (int t = 0; t < NS; ++t) gather_fetch(t, g[t]);
      gather_fetch(NS, grow);
#pragma unroll
      for (int t = 0; t < NS; ++t) gather_resolve(t, g[t], from[t]);
#pragma unroll
      for (int t = 0; t < NS; ++t) {
        if (t >= KT) break;
        if (t == KT - 1) end_loads((int)(kend - (int64_t)t * BKE));
#pragma unroll
        for (int n = 0; n < 2 * L; ++n) load(n, from[t], smem_addr + t * STAGE);
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < R; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    PIN();
    if (KT > 1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * L) : "memory");      // loads return in order: K-step 0 has landed
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    PIN();
    asm volatile("s_barrier" ::: "memory");
    PIN();
#pragma unroll
    for (int r = 0; r < NR; ++r) read(smem, 0, r, 0);
    PIN();
    uint32_t cur = 0;
    int kt = 0;
    for (; kt + NS < KT; ++kt) {
      const uint32_t nxt = cur == (NS - 1) * STAGE ? 0 : cur + STAGE;
      kstep(std::true_type{}, kt, cur, nxt);
      cur = nxt;
    }
#pragma unroll 1
    for (; kt < KT; ++kt) {                                           // the last one reads ahead a stage that holds nothing new, for no use
      const uint32_t nxt = cur == (NS - 1) * STAGE ? 0 : cur + STAGE;
      kstep(std::false_type{}, kt, cur, nxt);
      cur = nxt;
    }
  };
  if (TRA || live > 16) main_loop(std::integral_constant<int, R>{});
  else if (live > 0) main_loop(std::integral_constant<int, 1>{});
  else main_loop(std::integral_constant<int, 0>{});

  // ---- results, from the registers: register u of tile (i, j) is column R (4 kq + u) + j of the wave's, 4 R columns next to each other a lane
  const int64_t col0 = n0 + wn * WT + 4 * R * kq;
  if (MODE == kNN && p.bias) {
#pragma unroll
    for (int g = 0; g < R; ++g) {                                   // four columns
      const f32x4 b = *reinterpret_cast<const f32x4*>((const float*)p.bias + (int64_t)e * p.N + (col0 + 4 * g < p.N ? col0 + 4 * g : n0));
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i][(4 * g + x) % R][(4 * g + x) / R] += b[x];
    }
  }
  const int64_t out_at = (tile_at + wm * WT) * p.N;
  const float* with = MODE == kTN ? nullptr : (const float*)p.pre;
  auto write_rows = [&](auto act_tag, float* dst, const float* add) __attribute__((always_inline)) {
    constexpr int ACT = decltype(act_tag)::value;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t r = TRA ? R * l16 + i : 16 * i + l16, at = out_at + r * p.N + col0;
      if (r >= live) continue;
#pragma unroll
      for (int g = 0; g < R; ++g) {
        if (col0 + 4 * g >= p.N) continue;
        f32x4 v, w = {0.f, 0.f, 0.f, 0.f};
        if (add) w = *reinterpret_cast<const f32x4*>(add + at + 4 * g);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float a = acc[i][(4 * g + x) % R][(4 * g + x) / R];
          if (MODE == kNT) v[x] = add ? a * rows_act_grad_as<float, ACT>(w[x]) : a;
          else v[x] = rows_act_as<float, ACT>(a) + (add ? w[x] : 0.f);
        }
        *reinterpret_cast<f32x4*>(dst + at + 4 * g) = v;
      }
    }
  };
  if (MODE == kNN && p.pre_out) write_rows(std::integral_constant<int, -1>{}, (float*)p.pre_out, nullptr);
  if (MODE == kTN) write_rows(std::integral_constant<int, -1>{}, p.parts > 1 ? p.part_sums : (float*)p.out, nullptr);
  else switch (p.act) {
    case MOE_ACT_RELU: write_rows(std::integral_constant<int, MOE_ACT_RELU>{}, (float*)p.out, with); break;
    case MOE_ACT_GELU: write_rows(std::integral_constant<int, MOE_ACT_GELU>{}, (float*)p.out, with); break;
    case MOE_ACT_SILU: write_rows(std::integral_constant<int, MOE_ACT_SILU>{}, (float*)p.out, with); break;
    default: write_rows(std::integral_constant<int, -1>{}, (float*)p.out, with); break;
  }
}

template <int MODE> hipError_t launch_rows_fp32(TileArgs p, int64_t total, hipStream_t s) {
  dim3 grid;
  if (!tile_launch(p, 64, 64, total, grid) || p.plain) return hipErrorInvalidValue;
  if (MODE == kTN && p.parts > 1) grid.z = (unsigned)p.parts;
  if (MODE == kTN && p.gather) rows_fp32_kernel<MODE, MODE == kTN><<<grid, dim3(256), 0, s>>>(p);
  else rows_fp32_kernel<MODE, false><<<grid, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace
