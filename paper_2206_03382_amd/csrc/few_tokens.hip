// The experts' feed-forward layer and the combine for a few tokens:
//   hidden[p, :] = act(x[t] * W1[e] + b1[e])    for every kept choice p = (t, j) with e = idx[t, j];
//   out[t, :] = sum over its kept choices j of gate_w[t, j] * (hidden[p] * W2[e] + b2[e]).
// Reading the chosen experts' weights once is all the time there is (HBM bound), so each product is cut into units of one expert and 64 or 32 columns, a block
// each: eight waves share the sum over k, every one with loads of several steps in flight, and meet in LDS; where that makes few blocks, several share a unit's sum.  The expert's
// rows, 16 to a tile, go through the matrix cores together, whose 16 rows cost the same whether they are filled or not.
// Measured: 64 tokens, top-2 of 64 experts of 1024 x 4096 in bf16 104 and 99 us a product, 0.51 and 0.49 GB read = 4.9 TB/s (0.47 are the weights of experts that have a token); 16 tokens, 8 experts of 2048 x 2048 17.8 each for 13 of HBM; 1 token, 8 of 128 experts of
// 4096 x 1024 in 8 bits 17 and 15 for 6.5; a layer of 5 tokens, 4 experts of 256 x 512 in fp32 12.6.
#include <type_traits>

#include "block8.h"
#include "few_rules.h"
#include "ffn_device.h"

namespace moe {
namespace {

constexpr int kFewWaves = 8, kFewRows = MOE_FEW_MAX_TOKENS;
constexpr int kFewArrival = 32;                                     // columns to an arrival counter, at least
constexpr int kFewExperts = 512;
constexpr int kFewPartBits = 3;                                     // at most 8 parts of a sum over k
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// An operand's rows in the form the matrix cores take them, and a step of the weights of 16 C columns.  Lane l = 16 g + i has row i of the tokens; which k and columns it
// has of the weights is the weights' layout:
//   bf16 [K, N]   step of 32 k: rows k = 8 g .. + 7, columns C i .. + C - 1 in eight loads (C = 4: 128 bytes of a row to 16 lanes); column c of all lanes is a fragment, put together
//                 from halves of two loads at a time;
//   fp32 [K, N]   step of 16 k: rows 4 g .. + 3, columns C i .. in four loads; a component of a load is a fragment as it is;
//   8 bit [N, K]  step of 64 k: of columns 16 c + i, the k from 16 g, widened to bf16 with the block's exponent (exact but at the format's ends, moe_dequantize8).  fp32 tokens enter as three bf16 pieces, which hold their 24 bits.
// The result's lane (16 g + i) has row i and 4 values v of fragment c: column 4 C g + C v + c, or 16 c + 4 g + v where fragments are 16 columns next to each other (kApart).
// at(): where a lane's first piece of step 0 is; columns past N repeat the last ones, rows that do not exist the first one (neither is stored).  load() and
// load_rows() take the k that exist: all of them but in the last step (TAIL), where the others are zero.
template <typename ET, bool W8, int C> struct Few;

template <int C> struct Few<uint16_t, false, C> {
  static constexpr int kStep = 32;
  static constexpr bool kApart = false;
  static __device__ __forceinline__ int step(int wave, int j) { return wave + j * kFewWaves; }
  static constexpr int depth(int rt) { return rt == 4 ? 3 : 4; }
  typedef __attribute__((ext_vector_type(C / 2))) uint32_t Piece;
  struct At { uint32_t n; };
  struct Weights { Piece w[8]; };
  struct Rows { u32x4 x; };
  static __device__ __forceinline__ At at(int64_t n0, int64_t N, int64_t, int i, int g) {
    const int64_t n = n0 + C * i < N ? n0 + C * i : N - C;
    return {(uint32_t)((8 * g * N + n) * 2)};
  }
  static __device__ __forceinline__ int64_t step_bytes(int64_t N) { return kStep * N * 2; }
  template <bool TAIL> static __device__ __forceinline__ void load(Weights& o, const char* W, const At& at, const uint8_t*, int64_t N, int, int left, int g) {
    if (TAIL && 8 * g >= left) {
      for (int r = 0; r < 8; ++r) o.w[r] = Piece(0);
      return;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) o.w[r] = __builtin_nontemporal_load(reinterpret_cast<const Piece*>(W + r * N * 2 + at.n));
  }
  template <bool TAIL> static __device__ __forceinline__ void load_rows(Rows& o, const uint16_t* row, int left, int g) {
    if (TAIL && 8 * g >= left) o.x = u32x4{0, 0, 0, 0};
    else o.x = *reinterpret_cast<const u32x4*>(row + 8 * g);
  }
  template <int RT> static __device__ __forceinline__ void multiply(const Weights& w, const Rows (&x)[RT], f32x4 (&acc)[RT][C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      u32x4 b;
#pragma unroll
      for (int r = 0; r < 4; ++r) b[r] = __builtin_amdgcn_perm(w.w[2 * r + 1][c >> 1], w.w[2 * r][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int t = 0; t < RT; ++t)
        acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, x[t].x), acc[t][c], 0, 0, 0);
    }
  }
};

template <int C> struct Few<float, false, C> {
  static constexpr int kStep = 16;
  static constexpr bool kApart = false;
  static __device__ __forceinline__ int step(int wave, int j) { return wave + j * kFewWaves; }
  static constexpr int depth(int rt) { return C == 4 ? (rt == 1 ? 5 : (rt == 2 ? 4 : 3)) : (rt == 4 ? 4 : 6); }
  typedef __attribute__((ext_vector_type(C))) float Piece;
  struct At { uint32_t n; };
  struct Weights { Piece w[4]; };
  struct Rows { f32x4 x; };
  static __device__ __forceinline__ At at(int64_t n0, int64_t N, int64_t, int i, int g) {
    const int64_t n = n0 + C * i < N ? n0 + C * i : N - C;
    return {(uint32_t)((4 * g * N + n) * 4)};
  }
  static __device__ __forceinline__ int64_t step_bytes(int64_t N) { return kStep * N * 4; }
  template <bool TAIL> static __device__ __forceinline__ void load(Weights& o, const char* W, const At& at, const uint8_t*, int64_t N, int, int left, int g) {
    if (TAIL && 4 * g >= left) {
      for (int r = 0; r < 4; ++r) o.w[r] = Piece(0.f);
      return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) o.w[r] = __builtin_nontemporal_load(reinterpret_cast<const Piece*>(W + r * N * 4 + at.n));
  }
  template <bool TAIL> static __device__ __forceinline__ void load_rows(Rows& o, const float* row, int left, int g) {
    if (TAIL && 4 * g >= left) o.x = f32x4{0.f, 0.f, 0.f, 0.f};
    else o.x = *reinterpret_cast<const f32x4*>(row + 4 * g);
  }
  template <int RT> static __device__ __forceinline__ void multiply(const Weights& w, const Rows (&x)[RT], f32x4 (&acc)[RT][C]) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.w[r][c], x[t].x[r], acc[t][c], 0, 0, 0);
  }
};

template <typename ET, int C> struct Few<ET, true, C> {
  static constexpr int kStep = 64, kPieces = sizeof(ET) == 4 ? 3 : 1, kWords = sizeof(ET) / 2;
  static constexpr bool kApart = true;
  static __device__ __forceinline__ int step(int wave, int j) { return 2 * (wave + (j >> 1) * kFewWaves) + (j & 1); }      // two make a line of 128 bytes
  static constexpr int depth(int rt) { return sizeof(ET) == 4 ? (rt == 1 ? (C == 4 ? 1 : 3) : (rt == 2 ? 2 : 1)) : (rt == 1 ? (C == 4 ? 3 : 4) : (rt == 2 ? 3 : 2)); }
  struct At { uint32_t n[C]; };
  struct Weights { u32x4 w[C]; uint32_t exponent; };
  struct Rows { u32x4 x[2][kWords]; };                              // k from 16 g + 8 q
  static __device__ __forceinline__ At at(int64_t n0, int64_t N, int64_t row8, int i, int g) {
    At a;
#pragma unroll
    for (int c = 0; c < C; ++c) a.n[c] = (uint32_t)((n0 + 16 * c + i < N ? n0 + 16 * c + i : N - 1) * row8 + 16 * g);
    return a;
  }
  static __device__ __forceinline__ int64_t step_bytes(int64_t) { return kStep; }
  // rows of 8-bit values are padded to whole blocks with zeros
  template <bool TAIL> static __device__ __forceinline__ void load(Weights& o, const char* W, const At& at, const uint8_t* sc, int64_t, int step, int, int) {
#pragma unroll
    for (int c = 0; c < C; ++c) o.w[c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(W + at.n[c]));
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
  template <int RT> static __device__ __forceinline__ void multiply(const Weights& w, const Rows (&x)[RT], f32x4 (&acc)[RT][C]) {
    const uint32_t e = w.exponent;
    const float scale = e == kScaleNaN ? __uint_as_float(0x7fc00000u) : e == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(e << 23);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      bf16x8 b[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int lo = (int)w.w[c][2 * q], hi = (int)w.w[c][2 * q + 1];
        const bf16x2 b0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        const bf16x2 b2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), b3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
        b[c] = bf16x8{b0.x, b0.y, b1.x, b1.y, b2.x, b2.y, b3.x, b3.y};
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if constexpr (kPieces == 1) {
#pragma unroll
          for (int c = 0; c < C; ++c) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[c], __builtin_bit_cast(bf16x8, x[t].x[q][0]), acc[t][c], 0, 0, 0);
        } else {
          bf16x8 a[3];
#pragma unroll
          for (int j = 0; j < 8; ++j) {                             // the upper 16 bits, of what is left the upper 16, and what is left then: exact
            const float v = __uint_as_float(x[t].x[q][j >> 2][j & 3]);
            const float hi = __uint_as_float(__float_as_uint(v) & 0xffff0000u), r1 = __builtin_isinf(v) ? 0.f : v - hi;      // nothing is left of an infinity
            const float mid = __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
            a[0][j] = (__bf16)hi;
            a[1][j] = (__bf16)mid;
            a[2][j] = (__bf16)(r1 - mid);
          }
#pragma unroll
          for (int d = 2; d >= 0; --d)
#pragma unroll
            for (int c = 0; c < C; ++c) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[c], a[d], acc[t][c], 0, 0, 0);
        }
      }
    }
  }
};

// A block's part of an expert's weights, and the first steps of each wave's share: their loads go out as soon as the expert is known, before its rows are.
template <typename ET, bool W8, int C, int TILES> struct FewWeights {
  typedef Few<ET, W8, C> L;
  static constexpr int kFirst = L::depth(TILES) < 2 ? 1 : 2;
  const char* W;
  const uint8_t* sc;
  int64_t pitch, step_bytes;                                        // pitch: N, or the bytes of a row of 8-bit weights
  typename L::At at;
  int first, last;                                                  // of the whole steps, this block's
  bool end;                                                         // and what is left behind them
  typename L::Weights w[kFirst];

  __device__ __forceinline__ void start(const void* weights, const uint8_t* scales, int64_t e, int64_t K, int64_t N, int64_t n0, int part, int part_bits) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    pitch = W8 ? row_bytes8(K) : N;
    W = (const char*)weights + (W8 ? e * N * pitch : e * K * N * (int64_t)sizeof(ET));
    sc = W8 ? scales + (e * ceil_div(N, kBlock8) + n0 / kBlock8) * row_scales8(K) : nullptr;
    step_bytes = L::step_bytes(pitch);
    at = L::at(n0, N, pitch, lane & 15, lane >> 4);
    const int pairs = (int)(K / L::kStep + 1) / 2;                  // two steps of 8-bit weights are a line
    first = (pairs * part >> part_bits) * 2;
    end = part + 1 == 1 << part_bits;
    last = end ? (int)(K / L::kStep) : (pairs * (part + 1) >> part_bits) * 2;
#pragma unroll
    for (int d = 0; d < kFirst; ++d) {
      const int s = first + L::step(wave, d);
      if (s < last) L::template load<false>(w[d], W + s * step_bytes, at, sc, pitch, s, 0, lane >> 4);
    }
  }
};

// One expert's rows times 16 C columns of its weights, the sum over k shared by the block's waves; done(row, column, sum) for each result, by one thread.
// rows[r]: where row r of the operand is.
template <typename ET, bool W8, int C, int TILES, int RT, typename F>
__device__ __forceinline__ void few_product(const FewWeights<ET, W8, C, TILES>& o, const ET* const* rows, int n_rows, int64_t K, int64_t N, int64_t n0, float* sums, F&& done) {
  typedef Few<ET, W8, C> L;
  constexpr int D = L::depth(RT), kFirst = FewWeights<ET, W8, C, TILES>::kFirst, kColumns = 16 * C;        // D: steps in flight
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const ET* row[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) row[t] = rows[16 * t + i < n_rows ? 16 * t + i : 0];
  f32x4 acc[RT][C];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int c = 0; c < C; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  typename L::Weights w[D];
  typename L::Rows x[D][RT];
  const int first = o.first, last = o.last;
  auto fetch_rows = [&](int s, int d) {
#pragma unroll
    for (int t = 0; t < RT; ++t) L::template load_rows<false>(x[d][t], row[t] + s * L::kStep, 0, g);
  };
  auto fetch = [&](int s, int d) {
    if (s >= last) return;
    L::template load<false>(w[d], o.W + s * o.step_bytes, o.at, o.sc, o.pitch, s, 0, g);
    fetch_rows(s, d);
  };
#pragma unroll
  for (int d = 0; d < D; ++d) {
    const int s = first + L::step(wave, d);
    if (d >= kFirst) fetch(s, d);
    else if (s < last) {
      w[d] = o.w[d];
      fetch_rows(s, d);
    }
  }
  for (int j = 0; first + L::step(wave, j) < last; j += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (first + L::step(wave, j + d) >= last) break;
      L::template multiply<RT>(w[d], x[d], acc);
      fetch(first + L::step(wave, j + d + D), d);
    }
  }
  if (const int left = (int)(K - (int64_t)last * L::kStep); o.end && left > 0 && wave == last % kFewWaves) {
    L::template load<true>(w[0], o.W + last * o.step_bytes, o.at, o.sc, o.pitch, last, left, g);
#pragma unroll
    for (int t = 0; t < RT; ++t) L::template load_rows<true>(x[0][t], row[t] + (int64_t)last * L::kStep, left, g);
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
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int v = 0; v < 4; ++v) sums[(wave * 16 + i) * (kColumns + 4) + (L::kApart ? 16 * c + 4 * g + v : 4 * C * g + C * v + c)] = acc[t][c][v];
    __syncthreads();
    for (int q = threadIdx.x; q < 16 * kColumns; q += 64 * kFewWaves) {
      const int r = q / kColumns, c = q % kColumns;
      if (16 * t + r >= n_rows || n0 + c >= N) continue;
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < kFewWaves; ++u) s += sums[(u * 16 + r) * (kColumns + 4) + c];
      done(16 * t + r, n0 + c, s);
    }
  }
}

// Gate logits of few tokens and experts, a block to TOKENS tokens, 8 experts and a slice of the model dim: its threads take 8 of it each at a time, all their loads go out together,
// and the products are exact and summed in fp64.  part[slice][t][e], or the logit itself of a single slice; whoever reads them adds up the slices, so a logit is rounded once, like moe_gate_logits'.  VECTOR: rows of Wg in
// pieces of 8 experts, of which there is one at least, on 4 bytes.
constexpr int kLogitExperts = 8, kLogitThreads = 256, kLogitSliceBits = 2;      // twice the threads where there are no slices
struct __attribute__((packed, aligned(4))) Words4 { uint32_t x, y, z, w; };
__device__ __forceinline__ uint4 load16_any(const void* p) {
  const Words4 v = *reinterpret_cast<const Words4*>(p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <typename ET, int TOKENS, bool VECTOR>
__global__ __launch_bounds__(2 * kLogitThreads) void few_logits_kernel(const ET* __restrict__ x, const ET* __restrict__ Wg, const float* __restrict__ gate_bias, int T, int M, int E, int slice,
                                                                   double* __restrict__ part, float* __restrict__ logits,
                                                                   int32_t* __restrict__ counts, int32_t* __restrict__ arrived, int arrivals) {
  constexpr int kSums = TOKENS * kLogitExperts, V = Vec16<ET>::N;
  __shared__ double wave_sums[2 * kLogitThreads / 64][kSums];
  const int e0 = VECTOR && (int)blockIdx.x * kLogitExperts > E - kLogitExperts ? E - kLogitExperts : blockIdx.x * kLogitExperts;      // the last ones may be in two blocks
  const int t0 = blockIdx.y * TOKENS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.z == 0)                                              // of the products' blocks
    for (int i = (blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x; i < arrivals; i += gridDim.x * gridDim.y * blockDim.x) arrived[i] = 0;
  double sum[kSums] = {};
  const int end = min(M, (int)(blockIdx.z + 1) * slice);
  for (int m = blockIdx.z * slice + threadIdx.x * 8; m < end; m += blockDim.x * 8) {
    float a[TOKENS][8], b[8][kLogitExperts];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const ET* w = Wg + (int64_t)(m + r) * E + e0;
#pragma unroll
      for (int c = 0; c < kLogitExperts; c += V) {
        if constexpr (VECTOR) {
          float f[V];
          Vec16<ET>::unpack(load16_any(w + c), f);
#pragma unroll
          for (int j = 0; j < V; ++j) b[r][c + j] = f[j];
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) b[r][c + j] = load_as_f32(w + min(c + j, E - 1 - e0));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TOKENS; ++i)
#pragma unroll
      for (int c = 0; c < 8; c += V) {
        float f[V];
        Vec16<ET>::unpack(*reinterpret_cast<const uint4*>(x + (int64_t)min(t0 + i, T - 1) * M + m + c), f);
#pragma unroll
        for (int j = 0; j < V; ++j) a[i][c + j] = f[j];
      }
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int i = 0; i < TOKENS; ++i)
#pragma unroll
        for (int j = 0; j < kLogitExperts; ++j) sum[i * kLogitExperts + j] += (double)a[i][r] * (double)b[r][j];
  }
  // a wave's lanes: each turn halves the sums that a lane goes on with, so lane l ends with the one whose index is l's low bits, reversed
  int at = 0;
#pragma unroll
  for (int half = kSums / 2, d = 1; d < 64; d <<= 1, half >>= 1) {
    const bool upper = lane & d;
    if (half == 0) sum[0] += __shfl_xor(sum[0], d);
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const double give = upper ? sum[i] : sum[i + half], keep = upper ? sum[i + half] : sum[i];
      sum[i] = keep + __shfl_xor(give, d);
    }
    at += upper ? half : 0;
  }
  if (lane < kSums) wave_sums[wave][at] = sum[0];
  __syncthreads();
  const int t = t0 + threadIdx.x / kLogitExperts, e = e0 + threadIdx.x % kLogitExperts;
  if (threadIdx.x >= kSums || t >= T || e >= E) return;
  if (t == 0 && blockIdx.z == 0) counts[e] = 0;                     // what has arrivals is counted later
  double s = 0.0;
  for (int u = 0; u < (int)blockDim.x / 64; ++u) s += wave_sums[u][threadIdx.x];
  if (gridDim.z == 1) logits[(int64_t)t * E + e] = (float)(s + (gate_bias ? (double)gate_bias[e] : 0.0));
  else part[((int64_t)blockIdx.z * T + t) * E + e] = s;
}

// A logit of expert e, from its slices if there are several.
struct FewSlices {
  const double* part;
  const float *bias, *logits;
  int all, E, bits;
  __device__ __forceinline__ explicit FewSlices(const FewTokens& p)
      : part(p.logit_parts), bias(p.gate_bias), logits(p.logits), all((int)(p.T * p.E)), E((int)p.E), bits(p.slice_bits) {}
  template <int N> __device__ __forceinline__ float sum(int at, int e) const {
    double v[N], s = bias ? (double)bias[e] : 0.0;
#pragma unroll
    for (int u = 0; u < N; ++u) v[u] = part[u * all + at];
#pragma unroll
    for (int u = 0; u < N; ++u) s += v[u];
    return (float)s;
  }
  __device__ __forceinline__ float operator()(int t, int e) const {
    const int at = t * E + e;
    return bits == 0 ? logits[at] : bits == 1 ? sum<2>(at, e) : sum<4>(at, e);
  }
};

__device__ __forceinline__ uint32_t ordered(float v) {              // -0 as +0
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// The logits of very few tokens and experts, by every block of the first product for itself: pieces of 2 tokens and 4 experts, each to one or more waves.  fp64 as above.
constexpr int kAloneTokens = 8, kAloneExperts = 64;
// Tokens x experts x model dim up to here: a launch less.  us of a layer with the logits' own launch and without: 5 x 4 x 256 (fp32) 16.8, 13.8; 2 x 4 x 768 20.4, 16.7;
// 1 x 8 x 1024 17.5, 17.2; 1 x 8 x 2048 23.8, 23.9; 4 x 8 x 1024 19.7, 21.8; 8 x 8 x 1024 20.6, 26.5.
constexpr int64_t kAloneWork = 1 << 13;
struct FewAlone {
  double sums[kAloneTokens / 2 * kAloneExperts / 4][8];
  float logits[kAloneTokens * kAloneExperts];
};
__device__ __forceinline__ void load4(const float* p, float (&v)[4]) { Vec16<float>::unpack(*reinterpret_cast<const uint4*>(p), v); }
__device__ __forceinline__ void load4(const uint16_t* p, float (&v)[4]) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
  v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
}
struct FewNone {};
struct FewWorkedOut {
  const float* logits;
  int E;
  __device__ __forceinline__ float operator()(int t, int e) const { return logits[t * E + e]; }
};
// in LDS, or in one piece (more than 16 tokens: few_slice_bits), or in slices
template <int TILES> __device__ __forceinline__ FewWorkedOut few_logits_of(const FewTokens& p, const FewAlone& s) { return {s.logits, (int)p.E}; }
template <int TILES> __device__ __forceinline__ typename std::conditional<TILES == 1, FewSlices, FewWorkedOut>::type few_logits_of(const FewTokens& p, const FewNone&) {
  if constexpr (TILES == 1) return FewSlices(p);
  else return {p.logits, (int)p.E};
}
template <typename ET> __device__ __forceinline__ void few_alone_logits(const FewTokens& p, FewAlone& s) {
  const int T = (int)p.T, E = (int)p.E, M = (int)p.M, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int across = (E + 3) / 4, pieces = (T + 1) / 2 * across, parts = pieces >= kFewWaves ? 1 : kFewWaves / pieces;
  const ET *x = (const ET*)p.x, *Wg = (const ET*)p.Wg;
  const bool vector = E % 4 == 0 && (reinterpret_cast<uintptr_t>(Wg) & 15) == 0;
  for (int piece = wave / parts; piece < pieces; piece += kFewWaves / parts) {
    const int t0 = piece / across * 2, e0 = piece % across * 4, t1 = t0 + 1 < T ? t0 + 1 : t0;
    double sum[8] = {};
    for (int m = (wave % parts * 64 + lane) * 4; m < M; m += parts * 256) {
      float a[2][4], b[4][4];
      load4(x + (int64_t)t0 * M + m, a[0]);
      load4(x + (int64_t)t1 * M + m, a[1]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const ET* w = Wg + (int64_t)(m + r) * E + e0;
        if (vector) load4(w, b[r]);
        else {
#pragma unroll
          for (int j = 0; j < 4; ++j) b[r][j] = load_as_f32(w + min(j, E - 1 - e0));
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[4 * i + j] += (double)a[i][r] * (double)b[r][j];
    }
    int at = 0;
#pragma unroll
    for (int half = 4, d = 1; d < 64; d <<= 1, half >>= 1) {        // as in few_logits_kernel
      const bool upper = lane & d;
      if (half == 0) sum[0] += __shfl_xor(sum[0], d);
#pragma unroll
      for (int i = 0; i < half; ++i) {
        const double give = upper ? sum[i] : sum[i + half], keep = upper ? sum[i + half] : sum[i];
        sum[i] = keep + __shfl_xor(give, d);
      }
      at += upper ? half : 0;
    }
    if (lane < 8) s.sums[piece * parts + wave % parts][at] = sum[0];
  }
  __syncthreads();
  if (threadIdx.x < T * E) {
    const int t = threadIdx.x / E, e = threadIdx.x % E;
    double sum = p.gate_bias ? (double)p.gate_bias[e] : 0.0;
    for (int u = 0; u < parts; ++u) sum += s.sums[((t >> 1) * across + (e >> 2)) * parts + u][(t & 1) * 4 + (e & 3)];
    s.logits[threadIdx.x] = (float)sum;
  }
  __syncthreads();
}

// Units of work of both products: an expert each, or, where there are fewer choices than experts, a choice each, of which the first one to arrive at its expert does the work.
__host__ __device__ __forceinline__ int few_units(const FewTokens& p) { return (int)(p.E < p.T * p.k ? p.E : p.T * p.k); }

// A token's logits as integers in the same order, and their ranks: the number of experts with a larger logit, or an equal one and a lower index.
struct FewRanks {
  uint32_t keys[kFewExperts];
  int rank[kFewExperts];
};
template <typename L> __device__ __forceinline__ void few_rank(const FewTokens& p, const L& logits, int t, FewRanks& s) {
  const int E = (int)p.E, group = 1 << p.expert_bits, sub = threadIdx.x & (group - 1), e = threadIdx.x >> p.expert_bits;     // threads to an expert, in one wave
  if (threadIdx.x < E) s.keys[threadIdx.x] = ordered(logits(t, threadIdx.x));
  __syncthreads();
  int rank = 0;
  if (e < E) {
    const uint32_t own = s.keys[e];
#pragma unroll 8
    for (int o = sub; o < E; o += group) {
      const uint32_t other = s.keys[o];
      rank += other > own || (other == own && o < e) ? 1 : 0;
    }
  }
  for (int d = 1; d < group; d <<= 1) rank += __shfl_xor(rank, d);
  if (e < E && sub == 0) s.rank[e] = rank;
  __syncthreads();
}

// Tokens' logits, choices and gate weights as the caller sees them: the b-th block has 8 tokens, a wave each, or, of more than 64 experts, one token.
inline __host__ __device__ int few_token_blocks(const FewTokens& p) { return (int)(p.E <= 64 ? (p.T + kFewWaves - 1) / kFewWaves : p.T); }
template <typename L> __device__ __forceinline__ void few_report(const FewTokens& p, const L& logits, int b, FewRanks& s) {
  const int E = (int)p.E, k = p.k, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int t = b;
  if (E <= 64) {
    t = b * kFewWaves + wave;
    if (t >= p.T) return;
    const uint32_t own = lane < E ? ordered(logits(t, lane)) : 0;
    int rank = 0;
    for (int o = 0; o < E; ++o) {
      const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)own, o);
      rank += other > own || (other == own && o < lane) ? 1 : 0;
    }
    if (lane < E) s.keys[wave * 64 + lane] = own;
    if (lane < E) s.rank[wave * 64 + lane] = rank;
  } else {
    few_rank(p, logits, t, s);
    if (wave > 0) return;
  }
  const uint32_t* keys = s.keys + (E <= 64 ? wave * 64 : 0);
  const int* ranks = s.rank + (E <= 64 ? wave * 64 : 0);
  uint32_t most = 0;
  for (int e = lane; e < E; e += 64) {
    most = max(most, keys[e]);
    if (p.alone || p.slice_bits > 0) p.logits[(int64_t)t * E + e] = unordered(keys[e]);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
  const float top = unordered(most);
  float sum = 0.f;                                                  // over all experts, or the chosen ones
  for (int e = lane; e < E; e += 64) sum += !p.normalize || ranks[e] < k ? expf(unordered(keys[e]) - top) : 0.f;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  for (int e = lane; e < E; e += 64) {
    if (ranks[e] >= k) continue;
    p.idx[(int64_t)t * k + ranks[e]] = e;
    p.gate_w[(int64_t)t * k + ranks[e]] = expf(unordered(keys[e]) - top) / sum;
  }
}

// The pairs (t, j) that expert e has, from the logits: a group of threads finds its rank for one token, and one wave the order of the arrivals: all first choices, all second ones ...
template <typename L> __device__ __forceinline__ int few_own_rank(const FewTokens& p, const L& logits, int e) {
  const int E = (int)p.E, group = 1 << p.token_bits, sub = threadIdx.x & (group - 1), t = (int)(threadIdx.x >> p.token_bits), row = t < p.T ? t : 0;
  const uint32_t own = ordered(logits(row, e));
  int rank = 0;
  for (int o0 = sub; o0 < E; o0 += 4 * group) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = logits(row, o0 + i * group < E ? o0 + i * group : e);      // e itself counts for nothing
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t other = ordered(v[i]);
      rank += other > own || (other == own && o0 + i * group < e) ? 1 : 0;
    }
  }
  for (int d = 1; d < group; d <<= 1) rank += __shfl_xor(rank, d);
  return rank;
}
// into pair_of; returns, in wave 0, how many there are, up to the capacity, if the first is the one given (any if negative), else 0
__device__ __forceinline__ int few_own_pairs(const FewTokens& p, int e, int rank, int first, bool report, uint32_t* arrivals, int* pair_of) {
  const int T = (int)p.T, lane = threadIdx.x & 63, t = threadIdx.x >> p.token_bits;
  if (t < T && (threadIdx.x & ((1 << p.token_bits) - 1)) == 0) arrivals[t] = rank < p.k ? (uint32_t)(rank * T + t) : 0xffffffffu;
  __syncthreads();
  if (threadIdx.x >= 64) return 0;
  const uint32_t key = lane < T ? arrivals[lane] : 0xffffffffu;
  int before = 0;
  for (int u = 0; u < T; ++u) before += (uint32_t)__builtin_amdgcn_readlane((int)key, u) < key ? 1 : 0;
  const bool mine = key != 0xffffffffu;
  if (first >= 0 && __ballot((int)key == first && before == 0) == 0) return 0;
  const int q = lane * p.k + (int)(key / (uint32_t)T), n = __builtin_popcountll(__ballot(mine));
  const int most = (int)(p.C < kFewRows ? p.C : kFewRows);
  if (mine && before < most) pair_of[before] = q;
  if (report && mine) p.loc[q] = before;
  if (report && lane == 0 && n > 0) p.counts[e] = n;
  return n < most ? n : most;
}

// The expert of choice o = j T + t.
template <typename L> __device__ __forceinline__ int few_chosen(const FewTokens& p, const L& logits, int o, FewRanks& s, int* found) {
  few_rank(p, logits, o % (int)p.T, s);
  if (threadIdx.x < p.E && s.rank[threadIdx.x] == o / (int)p.T) *found = threadIdx.x;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(*found);
}

// plan: for the y-th blocks of the second product, or of both: their expert, its number of rows and its pairs.
__device__ __forceinline__ void few_write_plan(int32_t* plan, int e, int n, const int* pair_of) {
  const int lane = threadIdx.x & 63;
  if (lane < n) plan[2 + lane] = pair_of[lane];
  if (lane == 0) plan[0] = e;
  if (lane == 0) plan[1] = n;
}

// The plan in a launch of its own: a block to a unit, then those that report the tokens' choices.
__global__ __launch_bounds__(64 * kFewWaves) void few_plan_kernel(const FewTokens p) {
  __shared__ FewRanks ranks;
  __shared__ uint32_t arrivals[kFewRows];
  __shared__ int pair_of[kFewRows], found;
  const FewSlices logits(p);
  const int units = few_units(p);
  int e = blockIdx.x;
  if (e >= units) {
    few_report(p, logits, e - units, ranks);
    return;
  }
  const bool direct = units == p.E;
  if (!direct) e = few_chosen(p, logits, blockIdx.x, ranks, &found);
  const int n = few_own_pairs(p, e, few_own_rank(p, logits, e), direct ? -1 : (int)blockIdx.x, true, arrivals, pair_of);
  if (threadIdx.x < 64) few_write_plan(p.plan + (int64_t)blockIdx.x * kFewPlan, e, n, pair_of);
}

// Block x, y, z: 16 C columns of unit y's expert, part z of the sum over k.
// TILES: of 16 rows that an expert can have at most, 1 or 4; with 1 two blocks fit a CU (not beside the logits, which would spill).  STAGE: the first product, from the logits or the plan; with the logits worked out by each
// block itself; the second product.
constexpr int kFewUp = 0, kFewUpAlone = 1, kFewDown = 2;
template <typename ET, bool W8, int C, int TILES, int STAGE>
__global__ __launch_bounds__(64 * kFewWaves, TILES == 1 && STAGE != kFewUpAlone ? 4 : 2) void few_kernel(const FewTokens p) {
  constexpr bool UP = STAGE != kFewDown, ALONE = STAGE == kFewUpAlone, SPLIT = TILES == 1 && !ALONE;
  constexpr int kColumns = 16 * C, kSums = kFewWaves * 16 * (kColumns + 4);
  union Lds {
    FewRanks ranks;
    uint32_t arrivals[kFewRows];
    float sums[kSums];
  };
  __shared__ Lds lds;
  __shared__ int pair_of[kFewRows], found[2];
  __shared__ const ET* rows[kFewRows];
  __shared__ int last;
  __shared__ typename std::conditional<ALONE, FewAlone, FewNone>::type alone;
  const auto logits = few_logits_of<TILES>(p, alone);
  const int64_t K = UP ? p.M : p.H, N = UP ? p.H : p.M, n0 = (int64_t)blockIdx.x * kColumns;
  const int units = few_units(p), part_bits = SPLIT ? (UP ? p.up_bits : p.down_bits) : 0, parts = 1 << part_bits;
  const int unit = blockIdx.y, part = SPLIT ? blockIdx.z : 0;
  if constexpr (ALONE) few_alone_logits<ET>(p, alone);
  if constexpr (UP) {
    // The tokens' choices: rows of blocks after the others, the last to start, so that it is theirs to share a CU (16 tokens x 8 experts of 2048 x 2048, 256 + 8 blocks: 41.1 us,
    // and 45.8 with these among the others).
    if (unit >= units) {
      const int b = (unit - units) * gridDim.x + blockIdx.x;
      if (b >= few_token_blocks(p) || part > 0) return;
      few_report(p, logits, b, lds.ranks);
      if constexpr (ALONE) {                                        // one block has all tokens
        __syncthreads();
        if (threadIdx.x < p.E) {
          int n = 0;
          for (int t = 0; t < p.T; ++t) n += lds.ranks.rank[t * 64 + threadIdx.x] < p.k ? 1 : 0;
          p.counts[threadIdx.x] = n;
        }
      }
      return;
    }
    if (ALONE && blockIdx.x == 0 && blockIdx.y == 0)                // the arrivals of the next launch's blocks
      for (int64_t s = threadIdx.x; s < ceil_div(p.M, kFewArrival); s += 64 * kFewWaves) p.arrived[s] = 0;
  }
  const bool direct = units == p.E;      // the weights' expert is known before its rows are
  int32_t* plan = p.plan + (int64_t)unit * kFewPlan;
  FewWeights<ET, W8, C, TILES> weights;
  const void* W = UP ? p.W1 : p.W2;
  const uint8_t* sc = UP ? p.s1 : p.s2;
  if (direct) weights.start(W, sc, unit, K, N, n0, part, part_bits);
  const bool planned = !UP || p.planned;
  int unit_e = unit, v = 0;
  if (planned) v = threadIdx.x < kFewPlan ? plan[threadIdx.x] : 0;
  else {
    if (!direct) unit_e = few_chosen(p, logits, unit, lds.ranks, found);
    v = few_own_rank(p, logits, unit_e);
  }
  if (planned) {
    if (threadIdx.x < 2) found[threadIdx.x] = v;
    else if (threadIdx.x < kFewPlan) pair_of[threadIdx.x - 2] = v;
  } else {
    const int n = few_own_pairs(p, unit_e, v, direct ? -1 : unit, blockIdx.x == 0 && part == 0, lds.arrivals, pair_of);
    if (threadIdx.x < 64) {
      if (blockIdx.x == 0 && part == 0) few_write_plan(plan, unit_e, n, pair_of);
      if (threadIdx.x == 0) found[0] = unit_e;
      if (threadIdx.x == 0) found[1] = n;
    }
  }
  __syncthreads();
  const int e = __builtin_amdgcn_readfirstlane(found[0]), n_rows = __builtin_amdgcn_readfirstlane(found[1]);
  if (!direct && n_rows > 0) weights.start(W, sc, e, K, N, n0, part, part_bits);
  if (threadIdx.x < n_rows) {
    const int q = pair_of[threadIdx.x];
    rows[threadIdx.x] = UP ? (const ET*)p.x + (int64_t)(q / p.k) * K : (const ET*)p.hidden + (int64_t)q * K;
  }
  __syncthreads();
  const ET* bias = (const ET*)(UP ? p.b1 : p.b2);
  const int64_t pairs = p.T * p.k;
  if (n_rows > 0) {
    // Activations are stored as the second product's matrix instructions take them: bf16 is a rounding of 2^-8 of each at most, which with the output's own makes 2.3e-3 of the result
    // where that alone is 1.7e-3; their other form, three bf16 pieces, is three times the instructions.  Partial sums stay fp32.
    auto done = [&](int r, int64_t n, float s) {
      if (bias && part == 0) s += load_as_f32(bias + (int64_t)e * N + n);
      const int64_t q = pair_of[r];
      if (UP && parts == 1) store_from_f32((ET*)p.hidden + q * N + n, act_full(s, p.act));
      else if (!UP && p.k == 1 && parts == 1) store_from_f32((ET*)p.out + q * N + n, p.gate_w[q] * s);
      else __hip_atomic_store(p.partial + (part * pairs + q) * N + n, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    if (TILES == 1 || n_rows <= 16) few_product<ET, W8, C, TILES, 1>(weights, rows, n_rows, K, N, n0, lds.sums, done);
    else if (n_rows <= 32) few_product<ET, W8, C, TILES, 2>(weights, rows, n_rows, K, N, n0, lds.sums, done);
    else few_product<ET, W8, C, TILES, 4>(weights, rows, n_rows, K, N, n0, lds.sums, done);
  }
  if (UP && parts == 1) return;
  if (!UP && p.k == 1 && parts == 1) {                              // nothing to add up: what has no row here is zero
    if (blockIdx.y > 0) return;
    for (int64_t q = threadIdx.x; q < p.T * kColumns; q += 64 * kFewWaves) {
      const int64_t t = q / kColumns, n = n0 + q % kColumns;
      if (n < N && p.loc[t] >= p.C) store_from_f32((ET*)p.out + t * N + n, 0.f);
    }
    return;
  }
  // The last block of these columns to arrive (first product: with this unit) adds up what there is for them, in the order of choices and parts: the same sums whoever it is, and nobody waits.  The partial sums are stored and loaded
  // past what each XCD caches for itself (agent scope), so that a wave which has waited for its stores has them where every XCD sees them, and the last block, whose loads go out after
  // its count has come back, finds them there.  All accesses are atomic, but their order is none that the language's memory model promises: it is what gfx950 does, whose stores at agent scope are counted as done when they have
  // reached what all XCDs share, and this file is built for nothing else.  Counting needs no release then, which would write back all of an L2, and reading no acquire, which would drop it: 64 tokens x 64 experts of
  // 1024 x 4096 took 259 us with a release by one wave of each block instead of 227; 1 x 2 of 8, 4096 x 4096 in 8 bits 41.6 with an acquire instead of 35.3.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  int32_t* arrived = UP ? p.arrived + ceil_div(p.M, kFewArrival) + (int64_t)unit * gridDim.x : p.arrived;
  if (threadIdx.x == 0) last = __hip_atomic_fetch_add(arrived + blockIdx.x, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (UP ? parts : units * parts) - 1;
  __syncthreads();
  if (!last) return;
  if constexpr (UP) {
    for (int q0 = threadIdx.x; q0 < n_rows * kColumns; q0 += 64 * kFewWaves) {
      const int64_t q = pair_of[q0 / kColumns], n = n0 + q0 % kColumns;
      if (n >= N) continue;
      float v[1 << kFewPartBits];
#pragma unroll
      for (int u = 0; u < 1 << kFewPartBits; ++u) v[u] = __hip_atomic_load(p.partial + ((u < parts ? u : 0) * pairs + q) * N + n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < 1 << kFewPartBits; ++u) s += u < parts ? v[u] : 0.f;
      store_from_f32((ET*)p.hidden + q * N + n, act_full(s, p.act));
    }
    return;
  }
  for (int64_t q = threadIdx.x; q < p.T * kColumns; q += 64 * kFewWaves) {
    const int64_t t = q / kColumns, n = n0 + q % kColumns;
    if (n >= N) continue;
    float s = 0.f;
    for (int j0 = 0; j0 < p.k * parts; j0 += 8) {                   // their loads together; a choice without a row has no sums to read a value from
      float w[8], v[8];
      bool kept[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = j0 + j < p.k * parts ? j0 + j : 0, choice = at >> part_bits;
        const int64_t o = t * p.k + choice;
        kept[j] = j0 + j < p.k * parts && p.loc[o] < p.C;
        w[j] = p.gate_w[o];
        v[j] = __hip_atomic_load(p.partial + ((at & (parts - 1)) * pairs + o) * N + n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) s += kept[j] ? w[j] * v[j] : 0.f;
    }
    store_from_f32((ET*)p.out + t * N + n, s);
  }
}

// Parts of the sum over k, 2^bits, for up to as many blocks as there are CUs: one takes 25 GB/s or so from memory whatever its waves ask for.  Parts of 512 k at least, or 2048 of 8-bit
// weights.  us without and with: 1 token x 2 experts of 2048 x 2048 in bf16 (64 blocks) 29.0, 24.7; 1 x 4 of 4096 x 1024 (64 and 256) 36.5, 31.0; 4 x 8 of 64 of 1024 x 4096 (512 and 128)
// 43.4, 37.9; 16 x 4 of 2048 x 4096 (256 and 128) 52.1, 47.2; parts of 256 k, 16 x 8 of 512 x 512 20.1, 22.3; of 1024, 1 x 2 of 2048 x 2048 in 8 bits 21.2, 22.0.  More than 16 tokens: 40 x 2
// of 1024 x 1024 27.6, 30.4.
inline int few_part_bits(int64_t T, int64_t blocks, int64_t K, bool w8) {
  int bits = 0;
  while (T <= 16 && bits < kFewPartBits && blocks << (bits + 1) <= 256 && K >> (bits + 1) >= (w8 ? 2048 : 512)) ++bits;
  return bits;
}

// Slices of the model dim, 2^bits: one turn of a block's threads each, up to four; more than 16 tokens make blocks enough.  A block's reads of Wg bring whole lines for 16 bytes of each: 1 token, 8 of 128 experts of 4096 x 1024
// 39.7 us without, 37.5 with them, 8 of 256 of 8192 x 1024 72.6, 65.0; 2 of 8 of 2048 x 2048 in two slices 24.2, 25.0.
inline int few_slice_bits(int64_t T, int64_t M) {
  int bits = 0;
  while (T <= 16 && bits < kLogitSliceBits && M > kLogitThreads * 8 << bits) ++bits;
  return bits;
}

template <typename ET, int TOKENS> void launch_few_logits(const FewTokens& p, hipStream_t s) {
  const int slices = 1 << p.slice_bits, slice = (int)(ceil_div(ceil_div(p.M, slices), 8) * 8), arrivals = (int)(few_arrivals_bytes(p.M) / 4);
  const dim3 grid((unsigned)ceil_div(p.E, kLogitExperts), (unsigned)ceil_div(p.T, TOKENS), (unsigned)slices), block(p.T > 16 ? 2 * kLogitThreads : kLogitThreads);
  const bool vector = p.E >= kLogitExperts && (sizeof(ET) == 4 || p.E % 2 == 0) && (reinterpret_cast<uintptr_t>(p.Wg) & 3) == 0;
#define MOE_FEW_LOGITS(V) few_logits_kernel<ET, TOKENS, V><<<grid, block, 0, s>>>((const ET*)p.x, (const ET*)p.Wg, p.gate_bias, (int)p.T, (int)p.M, (int)p.E, slice, p.logit_parts, p.logits, p.counts, p.arrived, arrivals)
  if (vector) MOE_FEW_LOGITS(true);
  else MOE_FEW_LOGITS(false);
#undef MOE_FEW_LOGITS
}

template <typename ET, bool W8, int C, int STAGE> void launch_few_units(FewTokens p, hipStream_t s) {
  constexpr bool UP = STAGE != kFewDown;
  const int64_t columns = ceil_div(UP ? p.H : p.M, 16 * C), reports = UP && !p.planned ? ceil_div(few_token_blocks(p), columns) : 0;
  const int bits = STAGE == kFewUpAlone ? 0 : few_part_bits(p.T, columns * few_units(p), UP ? p.M : p.H, W8);
  (UP ? p.up_bits : p.down_bits) = bits;
  const dim3 grid((unsigned)columns, (unsigned)(few_units(p) + reports), 1u << bits), block(64 * kFewWaves);
  if (STAGE == kFewUpAlone || p.T <= 16) few_kernel<ET, W8, C, 1, STAGE><<<grid, block, 0, s>>>(p);
  else if constexpr (STAGE != kFewUpAlone) few_kernel<ET, W8, C, 4, STAGE><<<grid, block, 0, s>>>(p);
}

template <typename ET, bool W8, int STAGE> void launch_few_product(const FewTokens& p, hipStream_t s) {
  constexpr bool kBf16 = !W8 && sizeof(ET) == 2;
  if constexpr (kBf16) launch_few_units<ET, W8, 4, STAGE>(p, s);
  else if (few_columns(p.T, few_units(p), STAGE != kFewDown ? p.H : p.M, kBf16) == 64) launch_few_units<ET, W8, 4, STAGE>(p, s);
  else launch_few_units<ET, W8, 2, STAGE>(p, s);
}

template <typename ET, bool W8> hipError_t launch_few(const FewTokens& p, hipStream_t s) {
  if (p.alone) launch_few_product<ET, W8, kFewUpAlone>(p, s);
  else {
    if (p.T == 1) launch_few_logits<ET, 1>(p, s);
    else launch_few_logits<ET, 4>(p, s);
    if (hipError_t err = hipGetLastError()) return err;
    if (p.planned) {
      few_plan_kernel<<<dim3((unsigned)(few_units(p) + few_token_blocks(p))), dim3(64 * kFewWaves), 0, s>>>(p);
      if (hipError_t err = hipGetLastError()) return err;
    }
    launch_few_product<ET, W8, kFewUp>(p, s);
  }
  if (hipError_t err = hipGetLastError()) return err;
  launch_few_product<ET, W8, kFewDown>(p, s);
  return hipGetLastError();
}

}  // namespace

// counters of arrivals: for columns of the second product, and for blocks of the first one where they share a sum, which are 128 at most
size_t few_arrivals_bytes(int64_t M) { return (size_t)(ceil_div(M, kFewArrival) + 128) * 4; }

size_t few_logit_bytes(int64_t T, int64_t M, int64_t E) { return (size_t)T * E * 8 << few_slice_bits(T, M); }

// sums that blocks leave for each other
size_t few_partial_bytes(int64_t T, int64_t M, int64_t H, int64_t E, int k) {
  const int64_t units = E < T * k ? E : T * k;
  const int64_t up = H << few_part_bits(T, ceil_div(H, 64) * units, M, false), down = M << few_part_bits(T, ceil_div(M, 64) * units, H, false);      // the most that either kind of weights takes
  return (size_t)T * k * (up > down ? up : down) * 4;
}

hipError_t launch_few_tokens(const FewTokens& given, hipStream_t s) {
  FewTokens p = given;
  p.planned = few_planned(p.T, p.H, p.E, p.k, p.dtype == MOE_BF16 && !p.s1);
  p.alone = !p.planned && p.T <= kAloneTokens && p.E <= kAloneExperts && p.T * p.E * p.M <= kAloneWork;
  p.slice_bits = few_slice_bits(p.T, p.M);
  p.expert_bits = p.token_bits = 0;                                 // as many threads to an expert, and to a token, as there are
  while (p.expert_bits < 6 && (p.E << (p.expert_bits + 1)) <= 64 * kFewWaves) ++p.expert_bits;
  while (p.token_bits < 6 && (p.T << (p.token_bits + 1)) <= 64 * kFewWaves) ++p.token_bits;
  if (p.dtype == MOE_F32) return p.s1 ? launch_few<float, true>(p, s) : launch_few<float, false>(p, s);
  return p.s1 ? launch_few<uint16_t, true>(p, s) : launch_few<uint16_t, false>(p, s);
}

}  // namespace moe
