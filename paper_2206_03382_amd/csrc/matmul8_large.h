// The 8-bit products' large tile: 256 x 256 to a block of four waves, 128 x 128 each.  Included by matmul8.hip (same arguments and results).
//
// K advances by 128, a block of the format: 64 products of 16 x 16 x 128 a wave, 2048 cycles, for 64 KB of LDS that direct loads fill one K-step ahead (two stages).  A wave's rows
// are four pairs of 16-row fragments, 64 rows apart, so that both waves of a column share what a ragged tile has: NI of the pairs exist, the others are neither loaded nor
// multiplied.  A K-step runs in two halves of 8 NI products.  The first uses the fragments 0 .. NI - 1 of A and reads the others; then the next stage has to have landed
// (one wait, one barrier); the second half uses the others and reads the next K-step's B, each fragment into the registers of the one that its products have just used, and
// the next first half of A.  Its direct loads go out between the second half's products: the stage that they fill has been read by every wave at the barrier.
//
// The bodies have no branches: with conditions around the loads, or one that a product's result lives across, the compiler moved accumulators about at every one (hundreds of moves a
// K-step).  The exponents are in LDS before the first K-step (fetched in the loop, every four: 8192^3 2680 TFLOP/s instead of 2950).
//
// Measured: 8192^3 371 us = 2.96 PFLOP/s (register-only products: 3.9); 8 experts x 4096 rows, 2048 x 2048 120 us = 2.28, K = 4096 203 us = 2.70.  With four tiles to a unit, a
// K-step takes 2400 cycles; beside them a tile has 2500 until its first loads go out, 3000 to 5000 (cold operands) until they land, and 8500 for its results.  Tried and not kept: rings of
// three stages of one operand (the loads of B then have three quarters of a K-step: 10 % slower), K-steps of 64 in rings of five (rows of 64 bytes are half of what a
// request to the L2 brings: 15 % slower), stores straight from the registers (64-byte pieces of rows: 2 %), persistent blocks that load the next tile while they store (the loads'
// waits, which count in order, wait for the stores: 30 %), and fetching panels into the L2 ahead (the same waits).
namespace {

constexpr int kBig = 256, kBigStage = 2 * kBig * kBlock8;           // 64 KB
constexpr int kScaleBytes = kScaleWords * 2 * kBig * 4;             // 32 KB

// The body has no branch but the one around the exponents' fetch: past the reduction's end the direct loads bring the last K-step again and the reads what nobody uses.  With
// conditions around them the compiler moved accumulators about at every one (hundreds of moves and spills a K-step).
// Exponents in LDS: [word of four][row] of A and then of B.  set_out: gives the accumulators their first values.
// BLOCKS: B has one exponent for 128 x 128 values.
template <int NI, bool BLOCKS, typename F>
__device__ __forceinline__ void big_loop(char* smem, const char* (&a_at)[8], const char* b_base, const uint32_t (&b_at)[8], const uint8_t* a_sc, const uint8_t* b_sc,
                                         int row_sc, int KT, int a_off, int b_off, int sa_off, int sb_off, int wave, f32x4 (&acc)[8][8], F&& set_out) {
  constexpr int NB = BLOCKS ? 1 : 8, LOADS = 8 + 2 * NI;
  const uint32_t smem_addr = (uint32_t)(uintptr_t)LDS_PTR(char, smem);
  i32x8 a[2 * NI], b[8];
  uint32_t sa[2 * NI], sb[NB];                                      // exponents of this K-step
  const char* b_src = b_base;
  uint32_t fill = smem_addr + wave * 1024;                          // where the next direct loads go
  int ahead = KT - 1;                                               // K-steps after the one that is loaded next
  auto load = [&](int q) {                                          // q-th of a K-step's: 2 NI of A, 8 of B
    if (q < 2 * NI) global_to_lds_16(a_at[q], fill + q * 4096);
    else global_to_lds_16(b_src, b_at[q - 2 * NI], fill + kBig * kBlock8 + (q - 2 * NI) * 4096);
  };
  auto loaded = [&]() {
    const int step = ahead > 0 ? kBlock8 : 0;
    --ahead;
#pragma unroll
    for (int q = 0; q < 2 * NI; ++q) a_at[q] += step;
    b_src += step;
    fill ^= kBigStage;
  };
  auto load_scales = [&](int first) {                               // of the K-steps from `first`, a multiple of 64
    const int words = (row_sc - first) / 4 < kScaleWords ? (row_sc - first) / 4 : kScaleWords;
    for (int w = 0; w < words; ++w) {
      const uint32_t to = smem_addr + 2 * kBigStage + w * 2048 + wave * 256;
      global_to_lds_4(a_sc + first + 4 * w, to);
      global_to_lds_4(b_sc + first + 4 * w, to + 1024);
    }
  };
  auto read = [&](const char* at, int off) -> i32x8 {
    const u32x4 lo = *LDS_PTR(u32x4, at + off), hi = *LDS_PTR(u32x4, at + (off ^ 64));
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
  };
  auto read_a = [&](const char* st, int i) { a[i] = read(st + (i >> 1) * 8192 + (i & 1) * 2048, a_off); };
  auto read_b = [&](const char* st, int j) { b[j] = read(st + j * 2048, b_off); };
  const char* scales = smem + 2 * kBigStage;                        // of the K-step whose exponents are read next
  auto read_sa = [&](int i) { sa[i] = *LDS_PTR(uint8_t, scales + sa_off + (i >> 1) * 256 + (i & 1) * 64); };
  auto read_sb = [&](int j) { sb[j] = *LDS_PTR(uint8_t, scales + sb_off + j * 64); };
  auto product = [&](int i, int j) {
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i], acc[i][j], 0, 0, 0, (int)sb[BLOCKS ? 0 : j], 0, (int)sa[i]);
  };
  // a K-step; LOAD: with the direct loads of the one after the next
  auto step = [&](int kt, auto LOAD) {
    const char* cur = smem + (kt & 1) * kBigStage;
    const char* nxt = smem + ((kt + 1) & 1) * kBigStage;
    scales = smem + 2 * kBigStage + ((kt + 1) >> 2 & (kScaleWords - 1)) * 2048 + ((kt + 1) & 3);
    PIN();
#pragma unroll
    for (int m = 0; m < 8 * NI; ++m) {
      product(m % NI, m / NI);
      PIN();
      if (m < NI) read_a(cur, NI + m);
      PIN();
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    PIN();
#pragma unroll
    for (int m = 0; m < 8 * NI; ++m) {
      const int i = m % NI, j = m / NI;
      product(NI + i, j);
      PIN();
      if (i == NI - 1) {
        read_b(nxt, j);
        if constexpr (!BLOCKS) read_sb(j);
      }
      if (NI == 1 ? m == 0 : (m % NI == 0 && m / NI < NI)) {
        read_a(nxt, m / NI);
        read_sa(m / NI);
      }
      if constexpr (decltype(LOAD)::value) {
#pragma unroll
        for (int q = m * LOADS / (8 * NI); q < (m + 1) * LOADS / (8 * NI); ++q) load(q);       // evenly
      }
      PIN();
    }
    if constexpr (decltype(LOAD)::value) loaded();
#pragma unroll
    for (int i = NI; i < 2 * NI; ++i) read_sa(i);
    if constexpr (BLOCKS) read_sb(0);
  };
  load_scales(0);
#pragma unroll
  for (int q = 0; q < LOADS; ++q) load(q);
  loaded();
  set_out();                                                        // the accumulators' first values, while all this is on its way
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
  for (int q = 0; q < LOADS; ++q) load(q);                          // the last K-step again if there is only one
  loaded();
#pragma unroll
  for (int i = 0; i < 2 * NI; ++i) read_sa(i);
#pragma unroll
  for (int j = 0; j < NB; ++j) read_sb(j);
#pragma unroll
  for (int i = 0; i < NI; ++i) read_a(smem, i);
#pragma unroll
  for (int j = 0; j < 8; ++j) read_b(smem, j);
  int kt = 0;
#pragma unroll 1
  for (int first = 0; first < KT; first += 4 * kScaleWords) {
    if (first > 0) {
      // the last K-step of the part before has read this one's first exponents too early: all of them again
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      load_scales(first);
      asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
      scales = smem + 2 * kBigStage;
#pragma unroll
      for (int i = 0; i < 2 * NI; ++i) read_sa(i);
#pragma unroll
      for (int j = 0; j < NB; ++j) read_sb(j);
    }
    const int last = KT - 2 - first < 4 * kScaleWords ? KT - 2 : first + 4 * kScaleWords;
#pragma unroll 1
    for (; kt < last; ++kt) step(kt, std::true_type{});
    if (kt < KT - 2) continue;
    const int end = KT - first < 4 * kScaleWords ? KT : first + 4 * kScaleWords;
#pragma unroll 1
    for (; kt < end; ++kt) step(kt, std::false_type{});
  }
}

template <bool STREAM> __device__ __forceinline__ void store16(void* to, const u32x4& v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to));
  else *reinterpret_cast<u32x4*>(to) = v;
}

}  // namespace

template <int ACT, bool OUT8, bool BLOCKS>
__global__ __launch_bounds__(256, 1) void matmul8_large_kernel(const Args8 args) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * kBigStage + kScaleBytes];
  const Matmul8& p = args.p;
  const int lane = threadIdx.x & 63;
  int e, mt, nt, rows;
  if (!find_tile<kBig, false, 0, true>(blockIdx.x, lane, (int)p.E, p.C, p.counts, args.NT, e, mt, nt, rows)) return;
  const int64_t m0 = (int64_t)mt * kBig;
  if (m0 >= rows) return;
  const int n0 = nt * kBig;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, fr = lane & 15, g = lane >> 4;
  const int N = (int)p.N;
  int KT = (int)(args.row8 / kBlock8);
  if (p.k_counts) {
    const int64_t c = p.k_counts[e], most = c < p.K ? (c > 0 ? c : 0) : p.K;
    KT = (int)((most + kBlock8 - 1) / kBlock8);
  }
  const int live = (int)(rows - m0 < kBig ? rows - m0 : kBig), ni = (live + 63) >> 6;
  auto a_row = [&](int r) -> int64_t {                              // without a gather: of the expert's slab
    const int64_t c = r < live ? m0 + r : rows - 1;                 // rows past the fill repeat the last one (never stored)
    if (!p.gather) return c;
    const int t = p.gather[(int64_t)e * p.C + c];
    return (unsigned)t < (uint64_t)p.gather_rows ? t : 0;
  };
  const int64_t slab = p.gather ? 0 : (int64_t)e * p.C;
  const char* a_at[8];
  uint32_t b_at[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int r = (q * 4 + wave) * 8 + (lane >> 3), piece = ((lane & 7) ^ ((r >> 1) & 7)) << 4;
    a_at[q] = (const char*)p.A + (slab + a_row(r)) * args.row8 + piece;
    b_at[q] = (uint32_t)((int64_t)(n0 + r < N ? n0 + r : N - 1) * args.row8 + piece);
  }
  const char* b_base = (const char*)p.B + (int64_t)e * N * args.row8;
  const int NB = (N + kBlock8 - 1) / kBlock8, nw = n0 + wn * 128;
  // exponents: thread t has row t of A and column t of B
  const int64_t bn = n0 + (int)threadIdx.x < N ? n0 + threadIdx.x : N - 1;
  const uint8_t* a_sc = p.A_scales + (slab + a_row(threadIdx.x)) * args.row_sc;
  const uint8_t* b_sc = p.B_scales + (BLOCKS ? (int64_t)e * NB + bn / kBlock8 : (int64_t)e * N + bn) * args.row_sc;
  const int sw = (fr >> 1) & 7;
  const int a_off = wm * 4096 + fr * kBlock8 + ((g ^ sw) << 4), b_off = kBig * kBlock8 + wn * 16384 + fr * kBlock8 + ((g ^ sw) << 4);
  const int sa_off = (wm * 32 + fr) * 4, sb_off = 1024 + (wn * 128 + (BLOCKS ? 0 : fr)) * 4;
  f32x4 acc[8][8];
  auto set_out = [&]() {                                            // to the bias
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int n = nw + 16 * j + 4 * g;
      u32x2 w = {0, 0};
      if (p.bias && n < N) w = *reinterpret_cast<const u32x2*>((const uint16_t*)p.bias + (int64_t)e * N + n);
      const f32x4 v = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i][j] = v;
    }
  };
  if (KT == 0) set_out();
  if (KT > 0) {
#define MOE_BIG_LOOP(NI) \
  big_loop<NI, BLOCKS>(smem, a_at, b_base, b_at, a_sc, b_sc, (int)args.row_sc, KT, a_off, b_off, sa_off, sb_off, wave, acc, set_out)
    switch (ni) {
      case 4: MOE_BIG_LOOP(4); break;
      case 3: MOE_BIG_LOOP(3); break;
      case 2: MOE_BIG_LOOP(2); break;
      default: MOE_BIG_LOOP(1); break;
    }
#undef MOE_BIG_LOOP
  }
  // Lane (16 g + fr) has row fr of fragment i and columns 16 j + 4 g .. + 3 of the wave's 128: through LDS, 32 KB to a wave, to whole row pieces.
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");          // every wave is done with the stages, and nothing is on its way into them
  char* own = smem + wave * 32768;
  const int64_t blocks = args.out_row8 / kBlock8, nb = nw / kBlock8;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= 2 * ni) break;
    PIN();
    float v[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        v[j][c] = acc[i][j][c];
        v[j][c] = act8<ACT>(v[j][c]);
        if (OUT8 && nw + 16 * j + 4 * g >= N) v[j][c] = 0.f;        // N is a multiple of 8
      }
    const int r = i * 16 + fr;
    if constexpr (!OUT8) {
      // two halves of 64 columns: [128 rows][8 pieces of 8 columns], piece c of row r at c ^ r % 8
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *LDS_PTR(u32x2, own + (j >> 2) * 16384 + r * 128 + (((2 * (j & 3) + (g >> 1)) ^ (r & 7)) << 4) + 8 * (g & 1)) =
            u32x2{pack_bf16x2(v[j][0], v[j][1]), pack_bf16x2(v[j][2], v[j][3])};
    } else {
      // the wave's 128 columns are one block of the format
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) top = max(top, magnitude_bits(v[j][c]));
      top = max(top, (uint32_t)__shfl_xor((int)top, 16));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      const uint32_t sc = scale_of_amax(top);
      const float inverse = inverse_scale(sc);
#pragma unroll
      for (int j = 0; j < 8; ++j) *LDS_PTR(uint32_t, own + r * 128 + ((j ^ (r & 7)) << 4) + 4 * g) = pack8x4(v[j][0], v[j][1], v[j][2], v[j][3], inverse);
      const int row = ((i >> 1) * 2 + wm) * 32 + (i & 1) * 16 + fr;
      if (g == 0 && row < live && nb < blocks) {
        uint8_t* to = p.out8_scales + ((int64_t)e * p.C + m0 + row) * args.out_row_sc;
        to[nb] = (uint8_t)sc;
        if (nb == blocks - 1)
          for (int64_t b = blocks; b < args.out_row_sc; ++b) to[b] = (uint8_t)kScaleOne;
      }
    }
  }
  // stores of 8 rows x 128 bytes
  auto store = [&](auto STREAM) {
    constexpr bool stream = decltype(STREAM)::value;
    if constexpr (!OUT8) {
      uint16_t* oute = (uint16_t*)p.out + ((int64_t)e * p.C + m0) * N;
#pragma unroll 4
      for (int it = 0; it < 4 * ni; ++it) {
        const int r = it * 8 + (lane >> 3), c = (lane & 7) ^ (r & 7);
        const int row = ((r >> 5) * 2 + wm) * 32 + (r & 31);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const u32x4 w = *LDS_PTR(u32x4, own + half * 16384 + r * 128 + ((lane & 7) << 4));
          const int n = nw + half * 64 + c * 8;
          if (row < live && n < N) store16<stream>(oute + (int64_t)row * N + n, w);
        }
      }
    } else {
      uint8_t* oute = (uint8_t*)p.out8 + ((int64_t)e * p.C + m0) * args.out_row8;
#pragma unroll 4
      for (int it = 0; it < 4 * ni; ++it) {
        const int r = it * 8 + (lane >> 3), c = (lane & 7) ^ (r & 7);
        const int row = ((r >> 5) * 2 + wm) * 32 + (r & 31);
        const u32x4 w = *LDS_PTR(u32x4, own + r * 128 + ((lane & 7) << 4));
        const int n = nw + c * 16;
        if (row < live && n < args.out_row8) store16<stream>(oute + (int64_t)row * args.out_row8 + n, w);
      }
    }
  };
  if (args.stream) store(std::true_type{});
  else store(std::false_type{});
}
