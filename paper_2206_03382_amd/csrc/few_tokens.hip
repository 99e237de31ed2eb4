// The experts' feed-forward layer and the combine for a few tokens:
//   hidden[p, :] = act(x[t] * W1[e] + b1[e])    for every kept choice p = (t, j) with e = idx[t, j];
//   out[t, :] = sum over its kept choices j of gate_w[t, j] * (hidden[p] * W2[e] + b2[e]).
// Reading the chosen experts' weights once is all the time there is (HBM bound), so each product is cut into units of one expert and 64 columns, a block
// each: eight waves share the sum over k, every one with loads of several steps in flight, and meet in LDS.  The expert's rows, 16 to a tile, go
// through the matrix cores together, whose 16 rows cost the same whether they are filled or not.
#include "block8.h"
#include "ffn_device.h"

namespace moe {
namespace {

constexpr int kFewWaves = 8, kFewColumns = 64, kFewRows = MOE_FEW_MAX_TOKENS;
constexpr int kFewGateLogits = 1024, kFewPairs = MOE_FEW_MAX_TOKENS * 128;      // k * E <= 16384 and k <= E: at most 128 choices
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// An operand's rows in the form the matrix cores take them, and a step of the weights.  Lane l = 16 g + i has row i of the tokens; which k and columns it
// has of the weights is the weights' layout:
//   bf16 [K, N]   step of 32 k: rows k = 8 g .. + 7, columns 4 i .. + 3 in eight 8-byte loads (128 bytes of a row to 16 lanes); column c of all lanes is a
//                 fragment, put together from halves of two loads at a time;
//   fp32 [K, N]   step of 16 k: rows 4 g .. + 3, columns 4 i .. + 3 in four 16-byte loads; a component of a load is a fragment as it is;
//   8 bit [N, K]  step of 64 k: of columns 16 f + i, the k from 16 g, widened to bf16 with the block's exponent.  fp32 tokens enter as three bf16
//                 pieces, which hold their 24 bits.
// The result's lane (16 g + i) has row i and 4 values v of fragment f: column 16 g + 4 v + f, or 16 f + 4 g + v where fragments are 16 columns next to each other.
// at(): where a lane's first piece of step 0 is; columns past N repeat the last ones, rows that do not exist the first one (neither is stored).  load() and
// load_rows() take the k that exist: all of them but in the last step (TAIL), where the others are zero.
template <typename ET, bool W8> struct Few;

template <> struct Few<uint16_t, false> {
  static constexpr int kStep = 32;
  static constexpr bool kApart = false;
  struct At { uint32_t n; };
  static constexpr int depth(int rt) { return rt == 1 ? 5 : (rt == 2 ? 4 : 3); }
  struct Weights { u32x2 w[8]; };
  struct Rows { u32x4 x; };
  static __device__ __forceinline__ At at(int64_t n0, int64_t N, int64_t, int i, int g) {
    const int64_t n = n0 + 4 * i < N ? n0 + 4 * i : N - 4;
    return {(uint32_t)((8 * g * N + n) * 2)};
  }
  static __device__ __forceinline__ int64_t step_bytes(int64_t N) { return kStep * N * 2; }
  template <bool TAIL> static __device__ __forceinline__ void load(Weights& o, const char* W, const At& at, const uint8_t*, int64_t N, int, int left, int g) {
    if (TAIL && 8 * g >= left) {
      for (int r = 0; r < 8; ++r) o.w[r] = u32x2{0, 0};
      return;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) o.w[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(W + r * N * 2 + at.n));
  }
  template <bool TAIL> static __device__ __forceinline__ void load_rows(Rows& o, const uint16_t* row, int left, int g) {
    if (TAIL && 8 * g >= left) o.x = u32x4{0, 0, 0, 0};
    else o.x = *reinterpret_cast<const u32x4*>(row + 8 * g);
  }
  template <int RT> static __device__ __forceinline__ void multiply(const Weights& w, const Rows (&x)[RT], f32x4 (&acc)[RT][4]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      u32x4 b;
#pragma unroll
      for (int r = 0; r < 4; ++r) b[r] = __builtin_amdgcn_perm(w.w[2 * r + 1][c >> 1], w.w[2 * r][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int t = 0; t < RT; ++t)
        acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, x[t].x), acc[t][c], 0, 0, 0);
    }
  }
};

template <> struct Few<float, false> {
  static constexpr int kStep = 16;
  static constexpr bool kApart = false;
  struct At { uint32_t n; };
  static constexpr int depth(int rt) { return rt == 1 ? 5 : (rt == 2 ? 4 : 3); }
  struct Weights { f32x4 w[4]; };
  struct Rows { f32x4 x; };
  static __device__ __forceinline__ At at(int64_t n0, int64_t N, int64_t, int i, int g) {
    const int64_t n = n0 + 4 * i < N ? n0 + 4 * i : N - 4;
    return {(uint32_t)((4 * g * N + n) * 4)};
  }
  static __device__ __forceinline__ int64_t step_bytes(int64_t N) { return kStep * N * 4; }
  template <bool TAIL> static __device__ __forceinline__ void load(Weights& o, const char* W, const At& at, const uint8_t*, int64_t N, int, int left, int g) {
    if (TAIL && 4 * g >= left) {
      for (int r = 0; r < 4; ++r) o.w[r] = f32x4{0.f, 0.f, 0.f, 0.f};
      return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) o.w[r] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(W + r * N * 4 + at.n));
  }
  template <bool TAIL> static __device__ __forceinline__ void load_rows(Rows& o, const float* row, int left, int g) {
    if (TAIL && 4 * g >= left) o.x = f32x4{0.f, 0.f, 0.f, 0.f};
    else o.x = *reinterpret_cast<const f32x4*>(row + 4 * g);
  }
  template <int RT> static __device__ __forceinline__ void multiply(const Weights& w, const Rows (&x)[RT], f32x4 (&acc)[RT][4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.w[r][c], x[t].x[r], acc[t][c], 0, 0, 0);
  }
};

template <typename ET> struct Few<ET, true> {
  static constexpr int kStep = 64, kPieces = sizeof(ET) == 4 ? 3 : 1, kWords = sizeof(ET) / 2;
  static constexpr bool kApart = true;
  static constexpr int depth(int rt) { return rt == 1 ? 4 : (rt == 2 ? 3 : (sizeof(ET) == 4 ? 1 : 2)); }
  struct Weights { u32x4 w[4]; uint32_t exponent; };
  struct Rows { u32x4 x[2][kWords]; };                              // k from 16 g + 8 q
  struct At { uint32_t n[4]; };
  static __device__ __forceinline__ At at(int64_t n0, int64_t N, int64_t row8, int i, int g) {
    At a;
#pragma unroll
    for (int f = 0; f < 4; ++f) a.n[f] = (uint32_t)((n0 + 16 * f + i < N ? n0 + 16 * f + i : N - 1) * row8 + 16 * g);
    return a;
  }
  static __device__ __forceinline__ int64_t step_bytes(int64_t) { return kStep; }
  // rows of 8-bit values are padded to whole blocks with zeros
  template <bool TAIL> static __device__ __forceinline__ void load(Weights& o, const char* W, const At& at, const uint8_t* sc, int64_t, int step, int, int) {
#pragma unroll
    for (int f = 0; f < 4; ++f) o.w[f] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(W + at.n[f]));
    o.exponent = sc[step / 2];
  }
  template <bool TAIL> static __device__ __forceinline__ void load_rows(Rows& o, const ET* row, int left, int g) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int d = 0; d < kWords; ++d) {
        if (TAIL && 16 * g + 8 * q >= left) o.x[q][d] = u32x4{0, 0, 0, 0};
        else o.x[q][d] = *reinterpret_cast<const u32x4*>((const char*)(row + 16 * g + 8 * q) + 16 * d);
      }
  }
  template <int RT> static __device__ __forceinline__ void multiply(const Weights& w, const Rows (&x)[RT], f32x4 (&acc)[RT][4]) {
    const uint32_t e = w.exponent;
    const float scale = e == kScaleNaN ? __uint_as_float(0x7fc00000u) : e == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(e << 23);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      bf16x8 b[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int lo = (int)w.w[f][2 * q], hi = (int)w.w[f][2 * q + 1];
        const bf16x2 b0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        const bf16x2 b2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), b3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
        b[f] = bf16x8{b0.x, b0.y, b1.x, b1.y, b2.x, b2.y, b3.x, b3.y};
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if constexpr (kPieces == 1) {
#pragma unroll
          for (int f = 0; f < 4; ++f) acc[t][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[f], __builtin_bit_cast(bf16x8, x[t].x[q][0]), acc[t][f], 0, 0, 0);
        } else {
          bf16x8 a[3];
#pragma unroll
          for (int j = 0; j < 8; ++j) {                             // the upper 16 bits, of what is left the upper 16, and what is left then: exact
            const float v = __uint_as_float(x[t].x[q][j >> 2][j & 3]);
            const float hi = __uint_as_float(__float_as_uint(v) & 0xffff0000u), r1 = v - hi;
            const float mid = __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
            a[0][j] = (__bf16)hi;
            a[1][j] = (__bf16)mid;
            a[2][j] = (__bf16)(r1 - mid);
          }
#pragma unroll
          for (int d = 2; d >= 0; --d)
#pragma unroll
            for (int f = 0; f < 4; ++f) acc[t][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[f], a[d], acc[t][f], 0, 0, 0);
        }
      }
    }
  }
};

// One expert's rows times 64 columns of its weights, the sum over k shared by the block's waves; done(row, column, sum) for each result, by one thread.
// rows[r]: where row r of the operand is; pitch: N, or the bytes of a row of 8-bit weights.
template <typename ET, bool W8, int RT, typename F>
__device__ __forceinline__ void few_product(const char* W, const uint8_t* sc, int64_t pitch, const ET* const* rows, int n_rows, int64_t K, int64_t N, int64_t n0,
                                            float* sums, F&& done) {
  typedef Few<ET, W8> L;
  constexpr int D = L::depth(RT);                                   // steps in flight
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const ET* row[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) row[t] = rows[16 * t + i < n_rows ? 16 * t + i : 0];
  f32x4 acc[RT][4];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const typename L::At at = L::at(n0, N, pitch, i, g);
  const int64_t step_bytes = L::step_bytes(pitch);
  typename L::Weights w[D];
  typename L::Rows x[D][RT];
  const int full = (int)(K / L::kStep);
  auto fetch = [&](int s, int d) {
    if (s >= full) return;
    L::template load<false>(w[d], W + s * step_bytes, at, sc, pitch, s, 0, g);
#pragma unroll
    for (int t = 0; t < RT; ++t) L::template load_rows<false>(x[d][t], row[t] + s * L::kStep, 0, g);
  };
#pragma unroll
  for (int d = 0; d < D; ++d) fetch(wave + d * kFewWaves, d);
  for (int s = wave; s < full; s += D * kFewWaves) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (s + d * kFewWaves >= full) break;
      L::template multiply<RT>(w[d], x[d], acc);
      fetch(s + (d + D) * kFewWaves, d);
    }
  }
  if (const int left = (int)(K - (int64_t)full * L::kStep); left > 0 && wave == full % kFewWaves) {
    L::template load<true>(w[0], W + full * step_bytes, at, sc, pitch, full, left, g);
#pragma unroll
    for (int t = 0; t < RT; ++t) L::template load_rows<true>(x[0][t], row[t] + (int64_t)full * L::kStep, left, g);
    L::template multiply<RT>(w[0], x[0], acc);
  }
  // the waves' sums meet in LDS, 16 rows at a time: [wave][row][column], read back in the order of the waves
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (t > 0) {
      if (16 * t >= n_rows) break;
      __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int v = 0; v < 4; ++v) sums[(wave * 16 + i) * (kFewColumns + 4) + (L::kApart ? 16 * c + 4 * g + v : 16 * g + 4 * v + c)] = acc[t][c][v];
    __syncthreads();
    for (int q = threadIdx.x; q < 16 * kFewColumns; q += 64 * kFewWaves) {
      const int r = q / kFewColumns, c = q % kFewColumns;
      if (16 * t + r >= n_rows || n0 + c >= N) continue;
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < kFewWaves; ++u) s += sums[(u * 16 + r) * (kFewColumns + 4) + c];
      done(16 * t + r, n0 + c, s);
    }
  }
}

// Gate logits of few tokens and experts: part[s][t][e] = the sum over a slice of the model dim in fp64; whoever reads them adds the slices up in order, so the sum is
// rounded once, like moe_gate_logits'.  A single block would wait for one load after the other (16 tokens x 8 experts, M = 2048: 12 us).
constexpr int kGateStage = 8192;                                    // floats of the slice that a block holds at a time
template <typename ET>
__global__ __launch_bounds__(512) void few_logits_kernel(const ET* __restrict__ x, const ET* __restrict__ Wg, int T, int M, int E, int slice, int stage,
                                                         int group_bits, double* __restrict__ part) {
  __shared__ float tokens[kGateStage];                              // [T][stage] and then [stage][E]
  float* weights = tokens + T * stage;
  const int m_end = min(M, (int)(blockIdx.x + 1) * slice), pairs = T * E;
  const int group = 1 << group_bits, sub = threadIdx.x & (group - 1);
  constexpr int kTurns = 2;                                         // pairs of a thread: T * E <= 1024
  double sum[kTurns] = {};
  for (int m0 = blockIdx.x * slice; m0 < m_end; m0 += stage) {
    const int n = min(stage, m_end - m0);
    __syncthreads();
    for (int q = threadIdx.x; q < T * n; q += 512) tokens[q / n * stage + q % n] = load_as_f32(x + (int64_t)(q / n) * M + m0 + q % n);
    const ET* w = Wg + (int64_t)m0 * E;
#pragma unroll 4
    for (int q = threadIdx.x; q < n * E; q += 512) weights[q] = load_as_f32(w + q);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      const int p = u * (512 >> group_bits) + (threadIdx.x >> group_bits);
      if (p >= pairs) break;
      const float* a = tokens + p / E * stage;
      const float* b = weights + p % E;
      for (int m = sub; m < n; m += group) sum[u] += (double)a[m] * (double)b[m * E];
    }
  }
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    const int p = u * (512 >> group_bits) + (threadIdx.x >> group_bits);
    for (int d = 1; d < group; d <<= 1) sum[u] += __shfl_xor(sum[u], d);
    if (p < pairs && sub == 0) part[(int64_t)blockIdx.x * pairs + p] = sum[u];
  }
}

// Columns of x that a slice has: a thread's share of the products should be short, and so should what every block adds up again.
inline int few_gate_slice(int64_t M, int64_t T, int64_t E) {
  int64_t slices = 16384 / (T * E);
  slices = slices > 32 ? 32 : slices;
  return (int)(ceil_div(ceil_div(M, slices), 8) * 8);
}

// What the first product's blocks work out of the gate: LDS that the sums take over later.
struct FewGate {
  uint32_t keys[kFewGateLogits];                                    // logits [T][E] as integers in the same order
  int cnt[512];                                                     // arrivals per expert
  int idx[kFewPairs];                                               // experts in the order of arrival: all first choices, all second ones, ...
};

__device__ __forceinline__ uint32_t ordered(float v) {              // -0 as +0
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// Experts of every token from the logits' slices (p.slices > 0) or from idx as the gate's own kernels left it, arrivals per expert; in every block, since a
// launch of its own would take longer.  A choice's rank is the number of experts with a larger logit, or an equal one and a lower index.
__device__ __forceinline__ void few_choose(const FewTokens& p, FewGate& s) {
  constexpr int threads = 64 * kFewWaves;
  const int T = (int)p.T, E = (int)p.E, k = p.k;
  for (int e = threadIdx.x; e < E; e += threads) s.cnt[e] = 0;
  if (p.slices == 0) {
    for (int o = threadIdx.x; o < T * k; o += threads) s.idx[o] = p.idx[o % T * k + o / T];
    __syncthreads();
  } else {
    for (int q = threadIdx.x; q < T * E; q += threads) {
      double v = 0.0;
#pragma unroll 8
      for (int c = 0; c < p.slices; ++c) v += p.logit_parts[(int64_t)c * T * E + q];
      if (p.gate_bias) v += (double)p.gate_bias[q % E];
      s.keys[q] = ordered((float)v);
    }
    __syncthreads();
    for (int q = threadIdx.x; q < T * E; q += threads) {
      const int t = q / E, e = q - t * E;
      const uint32_t own = s.keys[q];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < E; ++o) {
        const uint32_t other = s.keys[t * E + o];
        rank += other > own || (other == own && o < e) ? 1 : 0;
      }
      if (rank < k) s.idx[rank * T + t] = e;
    }
    __syncthreads();
  }
  for (int o = threadIdx.x; o < T * k; o += threads) atomicAdd(&s.cnt[s.idx[o]], 1);
  __syncthreads();
}

// The routing as the caller sees it, by one block.
__device__ __forceinline__ void few_report(const FewTokens& p, const FewGate& s) {
  constexpr int threads = 64 * kFewWaves;
  const int T = (int)p.T, E = (int)p.E, k = p.k, lane = threadIdx.x & 63;
  for (int e = threadIdx.x; e < E; e += threads) p.counts[e] = s.cnt[e];
  for (int q = threadIdx.x; q < T * E; q += threads) p.logits[q] = unordered(s.keys[q]);
  for (int o = threadIdx.x; o < T * k; o += threads) {
    int before = 0;
    for (int u = 0; u < o; ++u) before += s.idx[u] == s.idx[o] ? 1 : 0;
    p.idx[o % T * k + o / T] = s.idx[o];
    p.loc[o % T * k + o / T] = before;
  }
  for (int t = threadIdx.x >> 6; t < T; t += kFewWaves) {           // a wave to a token
    const float top = unordered(s.keys[t * E + s.idx[t]]);
    float all = 0.f, chosen = 0.f;
    for (int e = lane; e < E; e += 64) all += expf(unordered(s.keys[t * E + e]) - top);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d);
    for (int j = 0; j < k; ++j) chosen += expf(unordered(s.keys[t * E + s.idx[j * T + t]]) - top);
    for (int j = lane; j < k; j += 64) p.gate_w[t * k + j] = expf(unordered(s.keys[t * E + s.idx[j * T + t]]) - top) / (p.normalize ? chosen : all);
  }
}

// The a-th expert that has arrivals, or -1.
__device__ __forceinline__ int active_expert(int a, const int* cnt, int E) {
  const int lane = threadIdx.x & 63;
  for (int e0 = 0; e0 < E; e0 += 64) {
    unsigned long long m = __ballot(e0 + lane < E && cnt[e0 + lane] > 0);
    const int n = __builtin_popcountll(m);
    if (a < n) {
      for (; a > 0; --a) m &= m - 1;
      return e0 + __builtin_ctzll(m);
    }
    a -= n;
  }
  return -1;
}

// Block x, y: 64 columns, the y-th expert that has arrivals.  The first product finds its expert's rows and leaves them for the second (p.plan: expert, number
// of rows, 64 pairs).
template <typename ET, bool W8, bool UP>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(const FewTokens p) {
  constexpr int kSums = kFewWaves * 16 * (kFewColumns + 4);
  union Lds {
    FewGate gate;
    float sums[kSums];
  };
  __shared__ Lds lds;
  __shared__ int pair_of[kFewRows], found[2];
  __shared__ const ET* rows[kFewRows];
  __shared__ int last;
  const int64_t K = UP ? p.M : p.H, N = UP ? p.H : p.M, n0 = (int64_t)blockIdx.x * kFewColumns;
  int32_t* plan = p.plan + (int64_t)blockIdx.y * kFewPlan;
  if constexpr (UP) {
    if (blockIdx.y == 0) {                                          // the arrivals of the next launch's blocks start from zero
      const int64_t at = (int64_t)blockIdx.x * (64 * kFewWaves) + threadIdx.x;
      for (int64_t s = at; s < ceil_div(p.M, kFewColumns); s += (int64_t)gridDim.x * (64 * kFewWaves)) p.arrived[s] = 0;
    }
    few_choose(p, lds.gate);
    if (p.slices > 0 && blockIdx.x == 0 && blockIdx.y == 0) few_report(p, lds.gate);
    const int e = active_expert(blockIdx.y, lds.gate.cnt, (int)p.E), lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {                                         // one wave goes through the arrivals
      int n = 0;
      const int most = (int)(p.C < kFewRows ? p.C : kFewRows);
      for (int o0 = 0; e >= 0 && o0 < p.T * p.k; o0 += 64) {
        const int o = o0 + lane;
        const bool mine = o < p.T * p.k && lds.gate.idx[o] == e;
        const unsigned long long m = __ballot(mine);
        const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
        if (mine && at < most) pair_of[at] = (int)(o % p.T * p.k + o / p.T);
        n += __builtin_popcountll(m);
      }
      n = n < most ? n : most;
      if (blockIdx.x == 0) {
        if (lane < n) plan[2 + lane] = pair_of[lane];
        if (lane == 0) plan[0] = e;
        if (lane == 0) plan[1] = n;
      }
      if (lane == 0) found[0] = e;
      if (lane == 0) found[1] = n;
    }
  } else {
    if (threadIdx.x < kFewPlan) {
      const int v = plan[threadIdx.x];
      if (threadIdx.x < 2) found[threadIdx.x] = v;
      else pair_of[threadIdx.x - 2] = v;
    }
  }
  __syncthreads();
  const int e = found[0], n_rows = found[1];
  if (threadIdx.x < n_rows) {
    const int q = pair_of[threadIdx.x];
    rows[threadIdx.x] = UP ? (const ET*)p.x + (int64_t)(q / p.k) * K : (const ET*)p.hidden + (int64_t)q * K;
  }
  __syncthreads();
  if (n_rows > 0) {
    const int64_t row8 = row_bytes8(K), pitch = W8 ? row8 : N;
    const char* W = (const char*)(UP ? p.W1 : p.W2) + (W8 ? (int64_t)e * N * row8 : (int64_t)e * K * N * sizeof(ET));
    const uint8_t* sc = W8 ? (UP ? p.s1 : p.s2) + ((int64_t)e * ceil_div(N, kBlock8) + n0 / kBlock8) * row_scales8(K) : nullptr;
    const ET* bias = (const ET*)(UP ? p.b1 : p.b2);
    auto done = [&](int r, int64_t n, float s) {
      if (bias) s += load_as_f32(bias + (int64_t)e * N + n);
      const int64_t q = pair_of[r];
      if (UP) store_from_f32((ET*)p.hidden + q * N + n, apply_act(s, p.act));
      else p.partial[q * N + n] = s;
    };
    if (n_rows <= 16) few_product<ET, W8, 1>(W, sc, pitch, rows, n_rows, K, N, n0, lds.sums, done);
    else if (n_rows <= 32) few_product<ET, W8, 2>(W, sc, pitch, rows, n_rows, K, N, n0, lds.sums, done);
    else few_product<ET, W8, 4>(W, sc, pitch, rows, n_rows, K, N, n0, lds.sums, done);
  }
  if (UP) return;
  // The last block of these columns to arrive adds up every token's choices, in their order: the same sums whoever it is, and nobody waits.  One wave releases what
  // the block has written: with a fence in every wave, 16 tokens x 8 experts of 2048 x 2048 took 50 us instead of 22.
  __syncthreads();
  if (threadIdx.x == 0) last = __hip_atomic_fetch_add(p.arrived + blockIdx.x, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.y - 1;
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  for (int64_t q = threadIdx.x; q < p.T * kFewColumns; q += 64 * kFewWaves) {
    const int64_t t = q / kFewColumns, n = n0 + q % kFewColumns;
    if (n >= N) continue;
    float s = 0.f;
    for (int j = 0; j < p.k; ++j)
      if (p.loc[t * p.k + j] < p.C) s += p.gate_w[t * p.k + j] * p.partial[(t * p.k + j) * N + n];
    store_from_f32((ET*)p.out + t * N + n, s);
  }
}

template <typename ET> hipError_t launch_few_logits(const FewTokens& p, hipStream_t s) {
  const int T = (int)p.T, E = (int)p.E, M = (int)p.M, slice = few_gate_slice(p.M, p.T, p.E);
  int stage = kGateStage / (T + E), bits = 0;
  if (stage > slice) stage = slice;
  while (bits < 6 && (T * E << (bits + 1)) <= 512) ++bits;          // threads to a sum: as many as there are
  few_logits_kernel<ET><<<dim3((unsigned)p.slices), dim3(512), 0, s>>>((const ET*)p.x, (const ET*)p.Wg, T, M, E, slice, stage, bits, p.logit_parts);
  return hipGetLastError();
}

template <typename ET, bool W8> hipError_t launch_few(const FewTokens& p, hipStream_t s) {
  if (p.slices > 0)
    if (hipError_t err = launch_few_logits<ET>(p, s)) return err;
  const unsigned experts = (unsigned)(p.E < p.T * p.k ? p.E : p.T * p.k);
  few_kernel<ET, W8, true><<<dim3((unsigned)ceil_div(p.H, kFewColumns), experts), dim3(64 * kFewWaves), 0, s>>>(p);
  if (hipError_t err = hipGetLastError()) return err;
  few_kernel<ET, W8, false><<<dim3((unsigned)ceil_div(p.M, kFewColumns), experts), dim3(64 * kFewWaves), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

// Slices of the model dim that the fused gate sums its logits in: 0 where the gate runs its own kernels.
int few_gate_slices(int64_t T, int64_t M, int64_t E, int k) {
  if (T * E > kFewGateLogits || E > 512) return 0;
  return (int)ceil_div(M, few_gate_slice(M, T, E));
}

size_t few_arrivals_bytes(int64_t M) { return (size_t)ceil_div(M, kFewColumns) * 4; }

hipError_t launch_few_tokens(const FewTokens& p, hipStream_t s) {
  if (p.dtype == MOE_F32) return p.s1 ? launch_few<float, true>(p, s) : launch_few<float, false>(p, s);
  return p.s1 ? launch_few<uint16_t, true>(p, s) : launch_few<uint16_t, false>(p, s);
}

}  // namespace moe
