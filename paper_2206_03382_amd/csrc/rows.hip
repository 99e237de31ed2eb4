// Operators around the products of experts' rows that lie one behind the other: the rows of a router's choices, the weighted combine of their results, dropout,
// the activation's derivative with the bias gradient.  All of them move memory once, 16 bytes a lane; what bounds them is HBM.
#include "philox.h"
#include "rows.h"
#include "rows_act.h"

namespace moe {
namespace {

// ---- dropout -------------------------------------------------------------------------------------------------------------
// The generator: philox.h.  The probability is a multiple of 2^-16.  Seed and offset are read on the device, so that a captured step can be given others.
constexpr int kGroup = 8;

// v of group g: dropped elements become zero whatever they were.
__device__ __forceinline__ void drop(float (&v)[kGroup], const Philox& rng, uint64_t g, uint32_t below, float scale) {
  uint32_t w[4];
  rng.bits(g, w);
#pragma unroll
  for (int i = 0; i < kGroup; ++i) {
    const uint32_t u = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
    v[i] = u < below ? 0.f : v[i] * scale;
  }
}

// A group of eight elements: one 16-byte piece of bf16, two of fp32.
template <typename ET> constexpr int kPieces = (int)sizeof(ET) / 2;
template <typename ET> struct Group { uint4 piece[kPieces<ET>]; };
template <typename ET, bool STREAM> __device__ __forceinline__ Group<ET> load_group(const uint4* at) {
  Group<ET> r;
#pragma unroll
  for (int i = 0; i < kPieces<ET>; ++i) r.piece[i] = STREAM ? load_stream(at + i) : at[i];
  return r;
}
template <typename ET> __device__ __forceinline__ void unpack_group(const Group<ET>& r, float (&v)[kGroup]) {
  constexpr int N = Vec16<ET>::N;
#pragma unroll
  for (int i = 0; i < kPieces<ET>; ++i) {
    float f[N];
    Vec16<ET>::unpack(r.piece[i], f);
#pragma unroll
    for (int u = 0; u < N; ++u) v[i * N + u] = f[u];
  }
}
template <typename ET> __device__ __forceinline__ void store_group(uint4* at, const float (&v)[kGroup]) {
  constexpr int N = Vec16<ET>::N;
#pragma unroll
  for (int i = 0; i < kPieces<ET>; ++i) {
    float f[N];
#pragma unroll
    for (int u = 0; u < N; ++u) f[u] = v[i * N + u];
    at[i] = Vec16<ET>::pack(f);
  }
}

// out = residual + dropout(x); one rounding.
template <typename ET, bool RES, bool DROP>
__global__ __launch_bounds__(256) void dropout_kernel(const uint4* __restrict__ x, const uint4* residual, const uint64_t* __restrict__ seed, uint32_t below, float scale,
                                                      int64_t groups, uint4* out) {
  constexpr int P = kPieces<ET>;
  const int64_t stride = (int64_t)gridDim.x * 256;
  const Philox rng = DROP ? Philox(seed) : Philox();
  for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += stride) {
    float v[kGroup], r[kGroup];
    const Group<ET> a = load_group<ET, false>(x + g * P);
    Group<ET> b;
    if (RES) b = load_group<ET, false>(residual + g * P);
    unpack_group<ET>(a, v);
    if (DROP) drop(v, rng, (uint64_t)g, below, scale);
    if (RES) {
      unpack_group<ET>(b, r);
#pragma unroll
      for (int i = 0; i < kGroup; ++i) v[i] += r[i];
    }
    store_group<ET>(out + g * P, v);
  }
}

// ---- the rows of a router's choices --------------------------------------------------------------------------------------
// Expert e has min(counts[e], C) rows behind those of the experts before it; the choice (t, j) has row offsets[idx] + loc.  Every block adds up the counts by itself: they are 2 KB at
// most, and a launch for them would take longer than all the rest.
constexpr int kMaxRowExperts = 512;

__global__ __launch_bounds__(256) void ragged_rows_kernel(const int32_t* __restrict__ idx, const int32_t* __restrict__ loc, const int32_t* __restrict__ counts, int64_t n,
                                                          int E, int k, int64_t C, int32_t* __restrict__ offsets, int32_t* __restrict__ row_src,
                                                          int32_t* __restrict__ row_of) {
  __shared__ int32_t at[kMaxRowExperts + 1];
  __shared__ int64_t sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // two experts to a thread; prefix sums of the threads' pairs
  int64_t own[2], pair = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = 2 * tid + i;
    int64_t c = e < E ? counts[e] : 0;
    c = c < 0 ? 0 : c;
    c = c < C ? c : C;
    own[i] = c < n ? c : n;
    pair += own[i];
  }
  int64_t upto = pair;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t v = __shfl_up(upto, d, 64);
    if (lane >= d) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int64_t first = upto - pair;
  for (int w = 0; w < wave; ++w) first += sums[w];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = 2 * tid + i;
    if (e <= E) at[e] = (int32_t)(first < n ? first : n);
    first += own[i];
  }
  if (tid == 255 && E == kMaxRowExperts) at[E] = (int32_t)(first < n ? first : n);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = tid; e <= E; e += 256) offsets[e] = at[e];
  const int total = at[E];
  for (int64_t p = (int64_t)blockIdx.x * 256 + tid; p < n; p += (int64_t)gridDim.x * 256) {
    const int e = idx[p], l = loc[p];
    int row = -1;
    if ((unsigned)e < (unsigned)E && l >= 0 && l < at[e + 1] - at[e]) row = at[e] + l;
    row_of[p] = row;
    if (row >= 0) row_src[row] = (int32_t)(p / k);
    if (p >= total) row_src[p] = -1;
  }
}

// ---- combine -------------------------------------------------------------------------------------------------------------
// out[t] = residual[t] + dropout(sum over the choices j, ascending, of gate_w[t,j] * Y[row_of[t,j]]), in fp32, rounded once; choices without a row are left out.  A wave has 64 groups of
// one token's row: its rows and weights are the same for all lanes, and it has up to eight rows in flight.
template <typename ET, bool STREAM, bool DROP>
__global__ __launch_bounds__(256) void ragged_combine_kernel(const uint4* __restrict__ Y, int64_t R, const int32_t* __restrict__ row_of, const float* __restrict__ gate_w,
                                                             const uint4* residual, const uint64_t* __restrict__ seed, uint32_t below, float scale, int64_t units, int per_row,
                                                             int groups, int k, uint4* out) {
  constexpr int P = kPieces<ET>;
  const int lane = threadIdx.x & 63;
  const Philox rng = DROP ? Philox(seed) : Philox();
  for (int64_t u = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6))); u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t t = u / per_row;
    const int g = (int)(u - t * per_row) * 64 + lane;
    if (g >= groups) continue;
    float v[kGroup];
#pragma unroll
    for (int i = 0; i < kGroup; ++i) v[i] = 0.f;
    const int64_t here = (t * groups + g) * P;
    Group<ET> res;
    if (residual) res = load_group<ET, STREAM>(residual + here);
    for (int j0 = 0; j0 < k; j0 += 8) {
      Group<ET> y[8];
      float w[8];
      bool on[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        on[j] = false;
        if (j0 + j < k) {
          const int64_t row = row_of[t * k + j0 + j];
          on[j] = row >= 0 && row < R;
          if (on[j]) {
            w[j] = gate_w ? gate_w[t * k + j0 + j] : 1.0f;
            y[j] = load_group<ET, STREAM>(Y + (row * groups + g) * P);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!on[j]) continue;
        float f[kGroup];
        unpack_group<ET>(y[j], f);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) v[i] = fmaf(w[j], f[i], v[i]);
      }
    }
    if (DROP) drop(v, rng, (uint64_t)(t * groups + g), below, scale);
    if (residual) {
      float f[kGroup];
      unpack_group<ET>(res, f);
#pragma unroll
      for (int i = 0; i < kGroup; ++i) v[i] += f[i];
    }
    store_group<ET>(out + here, v);
  }
}

// d = dropout(d_out), dY[row_of[t,j]] = gate_w[t,j] * d[t], dgate_w[t,j] = <d[t], Y[row_of[t,j]]>.  W waves to a token (4: rows of more than 128 groups); d_out is read once for
// eight choices.  The order of the sums is fixed by the sizes.
template <typename ET, bool STREAM, bool DROP, int W>
__global__ __launch_bounds__(256) void ragged_combine_backward_kernel(const uint4* __restrict__ d_out, const uint4* __restrict__ Y, int64_t R, const int32_t* __restrict__ row_of,
                                                                      const float* __restrict__ gate_w, const uint64_t* __restrict__ seed, uint32_t below, float scale,
                                                                      int64_t T, int groups, int k, uint4* __restrict__ dY, float* __restrict__ dgate_w) {
  constexpr int P = kPieces<ET>;
  __shared__ float part[4][8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Philox rng = DROP ? Philox(seed) : Philox();
  const int64_t step = (int64_t)gridDim.x * (4 / W);
  for (int64_t t = (int64_t)blockIdx.x * (4 / W) + (W == 4 ? 0 : wave); t < T; t += step) {
    for (int j0 = 0; j0 < k; j0 += 8) {
      int64_t row[8];
      float w[8], acc[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        row[j] = -1;
        w[j] = acc[j] = 0.f;
        if (j0 + j < k) {
          const int64_t r = row_of[t * k + j0 + j];
          if (r >= 0 && r < R) {
            row[j] = r;
            w[j] = gate_w ? gate_w[t * k + j0 + j] : 1.0f;
          }
        }
      }
      for (int g = (W == 4 ? wave * 64 : 0) + lane; g < groups; g += W * 64) {
        const Group<ET> a = load_group<ET, false>(d_out + (t * groups + g) * P);
        Group<ET> y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (row[j] >= 0) y[j] = load_group<ET, STREAM>(Y + (row[j] * groups + g) * P);
        float d[kGroup];
        unpack_group<ET>(a, d);
        if (DROP) drop(d, rng, (uint64_t)(t * groups + g), below, scale);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (row[j] < 0) continue;
          float f[kGroup], o[kGroup];
          unpack_group<ET>(y[j], f);
#pragma unroll
          for (int i = 0; i < kGroup; ++i) {
            acc[j] = fmaf(d[i], f[i], acc[j]);
            o[i] = w[j] * d[i];
          }
          store_group<ET>(dY + (row[j] * groups + g) * P, o);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j0 + j >= k) break;
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) acc[j] += __shfl_xor(acc[j], m, 64);
        if (W == 1) {
          if (lane == 0) dgate_w[t * k + j0 + j] = acc[j];
        } else if (lane == 0) {
          part[wave][j] = acc[j];
        }
      }
      if (W == 4) {
        __syncthreads();
        if ((int)threadIdx.x < 8 && j0 + (int)threadIdx.x < k) {
          const int j = threadIdx.x;
          dgate_w[t * k + j0 + j] = part[0][j] + part[1][j] + part[2][j] + part[3][j];
        }
        __syncthreads();
      }
    }
  }
}

// ---- the activation's derivative and the bias gradient ---------------------------------------------------------------------
// dp[r] = dy[r] * act'(pre[r]) and, in the same pass, db[e] = sum of dp over the expert's rows.  A block has a strip of 32 groups (512 bytes of bf16: 80 us for 32768 x 2048, where strips of
// 256 and 1024 bytes take 94 and 86) and a chunk of rows, whoever's they are, so that a gate that gives most rows to few experts costs nothing.  It goes through the experts' pieces of its
// chunk: 8 classes of rows, each summed in ascending order by one thread, then class by class.  An expert whose rows all lie in one chunk has its sum; of one that goes on in
// another, the chunk keeps the sum of the piece, `head` if the expert began before the chunk, `tail` if it begins in it, and a second launch adds those up in order.  The order is fixed by sizes and
// offsets.  The sums are of dp before its rounding.  dp is rounded to the storage type: the matrix cores take it as an operand.
// Slices of every expert's rows instead, however many there are, took 217 us for 32768 rows of 64 experts x 1024 under a Zipf-shaped gate where this takes 55.
constexpr int kStrip = 32, kClasses = 8;

__device__ __forceinline__ int64_t clamp_row(int64_t v, int64_t R) { return v < 0 ? 0 : (v < R ? v : R); }

// The first expert from e on whose rows end behind `row`, the same in every lane, and where they lie; E if there is none.  Without offsets there is one expert.
__device__ __forceinline__ int expert_behind(const int32_t* __restrict__ offsets, int e, int E, int64_t R, int64_t row, int64_t& lo, int64_t& hi) {
  if (!offsets) {
    lo = 0, hi = R;
    return e < 1 && row < R ? 0 : 1;
  }
  const int lane = threadIdx.x & 63;
  for (; e < E; e += 64) {
    const int x = e + lane < E ? e + lane : E - 1;
    const int64_t end = clamp_row(offsets[x + 1], R), from = clamp_row(offsets[x], R);
    const unsigned long long hit = __ballot(e + lane < E && end > row && end > from);
    if (hit == 0) continue;
    const int l = __builtin_ctzll(hit);
    lo = __shfl(from, l, 64), hi = __shfl(end, l, 64);
    return e + l;
  }
  return E;
}

template <typename ET, int ACT, bool SUM>
__global__ __launch_bounds__(256) void rows_act_backward_kernel(const uint4* __restrict__ dy, const uint4* __restrict__ pre, const int32_t* __restrict__ offsets, int64_t R, int E,
                                                                int groups, int64_t chunk, uint4* __restrict__ dp, float* __restrict__ sums, ET* __restrict__ db) {
  constexpr int P = kPieces<ET>;
  static_assert(kStrip * kGroup == 256 && kStrip * kClasses == 256, "a column, and a group of a class, to a thread");
  __shared__ float part[kClasses][kStrip * kGroup + 1];
  const int64_t from = blockIdx.y * chunk, to = from + chunk < R ? from + chunk : R, N = (int64_t)groups * kGroup;
  const int cls = threadIdx.x / kStrip, g = blockIdx.x * kStrip + threadIdx.x % kStrip;
  const int64_t col = (int64_t)blockIdx.x * kStrip * kGroup + threadIdx.x;
  int64_t lo, hi;
  int e = 0, known = 0;                                             // experts below `known` have their sums, if all rows are in this chunk
  for (int64_t row = from; row < to;) {
    e = expert_behind(offsets, e, E, R, row, lo, hi);
    if (e >= E) break;
    const int64_t begin = lo > row ? lo : row, end = hi < to ? hi : to;
    if (begin >= to) break;
    float s[kGroup];
#pragma unroll
    for (int i = 0; i < kGroup; ++i) s[i] = 0.f;
    if (g < groups) {
      constexpr int U = 4;                                          // rows of a class in flight
      auto one = [&](int64_t at, const Group<ET>& a, const Group<ET>& b) __attribute__((always_inline)) {
        float v[kGroup], p[kGroup];
        unpack_group<ET>(a, v);
        if (ACT >= 0) {
          unpack_group<ET>(b, p);
#pragma unroll
          for (int i = 0; i < kGroup; ++i) v[i] *= rows_act_grad_as<ET, ACT>(p[i]);
          store_group<ET>(dp + at, v);
        }
        if (SUM) {
#pragma unroll
          for (int i = 0; i < kGroup; ++i) s[i] += v[i];
        }
      };
      int64_t r = begin + cls;
      for (; r + (U - 1) * kClasses < end; r += U * kClasses) {
        Group<ET> a[U], b[U];
#pragma unroll
        for (int i = 0; i < U; ++i) a[i] = load_group<ET, false>(dy + ((r + i * kClasses) * groups + g) * P);
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (ACT >= 0) b[i] = load_group<ET, false>(pre + ((r + i * kClasses) * groups + g) * P);
#pragma unroll
        for (int i = 0; i < U; ++i) one(((r + i * kClasses) * groups + g) * P, a[i], b[i]);
      }
      for (; r < end; r += kClasses) {
        const int64_t at = (r * groups + g) * P;
        const Group<ET> a = load_group<ET, false>(dy + at);
        Group<ET> b;
        if (ACT >= 0) b = load_group<ET, false>(pre + at);
        one(at, a, b);
      }
    }
    if (SUM) {
#pragma unroll
      for (int i = 0; i < kGroup; ++i) part[cls][threadIdx.x % kStrip * kGroup + i] = s[i];
      __syncthreads();
      if (col < N) {
        float t = 0.f;
#pragma unroll
        for (int c = 0; c < kClasses; ++c) t += part[c][threadIdx.x];
        if (lo >= from && hi <= to) store_from_f32<ET>(db + e * N + col, t);
        else sums[(blockIdx.y * 2 + (lo < from ? 0 : 1)) * N + col] = t;             // head, tail
        if (gridDim.y == 1)                                         // no second launch: experts without rows
          for (; known < e; ++known) store_from_f32<ET>(db + known * N + col, 0.f);
        known = e + 1;
      }
      __syncthreads();
    }
    row = end;
    ++e;
  }
  if (SUM && gridDim.y == 1 && col < N)
    for (; known < E; ++known) store_from_f32<ET>(db + known * N + col, 0.f);
}

// db of the experts whose rows lie in several chunks, and of those without any.  A block has 64 columns of an expert and a part of its chunks to each of its waves: one thread for 64 was
// a chain of loads, 17 us for 2048 columns.  16 waves where experts have more than 8 chunks in the mean (32768 rows x 256 of one expert, in all: 17 us, with 4 waves 30), 4 below (2048 rows
// of 128 experts x 1024: 16 us, with 16 waves 21).
template <typename ET, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void chunk_sum_kernel(const float* __restrict__ sums, const int32_t* __restrict__ offsets, int64_t R, int64_t chunk, int64_t N, ET* __restrict__ db) {
  __shared__ float part[WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.y;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane, lo = offsets ? clamp_row(offsets[e], R) : 0, hi = offsets ? clamp_row(offsets[e + 1], R) : R;
  if (hi <= lo) {
    if (wave == 0 && i < N) store_from_f32<ET>(db + e * N + i, 0.f);
    return;
  }
  const int64_t first = lo / chunk, last = (hi - 1) / chunk, n = last - first + 1;
  if (n == 1) return;
  float t = 0.f;
  if (i < N) {
    const int64_t to = first + (wave + 1) * n / WAVES;
#pragma unroll 8
    for (int64_t c = first + wave * n / WAVES; c < to; ++c) t += sums[(c * 2 + (c * chunk <= lo ? 1 : 0)) * N + i];
  }
  part[wave][lane] = t;
  __syncthreads();
  if (wave == 0 && i < N) {
    t = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) t += part[w][lane];
    store_from_f32<ET>(db + e * N + i, t);
  }
}

// Rows of a chunk: all of up to 128 with eight experts' pieces at most, which need no second launch (128 rows of one expert x 1024: 11.4 us, in two launches 14.6; but 128 rows of 128
// experts x 2048, piece behind piece: 112 us, in chunks of 16 rows 23, of 4 15).  Else as few as leave the second launch little to add (8192 x 2048 of one expert: 16 rows to a chunk 24.8 us, 32 23.6, 64
// 21.7, 256 26.7; 3002 rows of 17 experts x 1544, fp32: 22.7, 30, 38, 58) and the first about 4096 blocks.
int64_t act_backward_chunk(int64_t R, int64_t E, int64_t N) {
  if (R <= 128 && (R < E ? R : E) <= 8) return 128;
  int64_t chunk = 4;
  while (chunk < 16 && ceil_div(R, chunk) > 64) chunk *= 2;
  while (chunk < 64 && ceil_div(R, chunk) > 192) chunk *= 2;
  while ((chunk < 256 && ceil_div(R, chunk) * ceil_div(N / kGroup, kStrip) > 4096) || ceil_div(R, chunk) > 65535) chunk *= 2;      // and no more chunks than a grid's second dimension has
  return chunk;
}

unsigned blocks_for(int64_t work, int64_t per_block, int64_t most) {
  const int64_t b = ceil_div(work, per_block);
  return (unsigned)(b < most ? b : most);
}

// beyond this, data that is read once is loaded past the caches
constexpr double kStreamBytes = 536870912.0;

}  // namespace

hipError_t launch_dropout(const void* x, const void* residual, const Dropout& d, int dtype, int64_t n, void* out, hipStream_t s) {
  const int64_t groups = n / kGroup;
  const dim3 grid(blocks_for(groups, 256, 1 << 20)), block(256);
#define MOE_LAUNCH_DROPOUT(ET, RES, DROP) \
  dropout_kernel<ET, RES, DROP><<<grid, block, 0, s>>>((const uint4*)x, (const uint4*)residual, d.seed, d.below, d.scale, groups, (uint4*)out)
#define MOE_LAUNCH_DROPOUT_ET(ET)                              \
  do {                                                         \
    if (residual && d.below) MOE_LAUNCH_DROPOUT(ET, true, true);   \
    else if (residual) MOE_LAUNCH_DROPOUT(ET, true, false);    \
    else if (d.below) MOE_LAUNCH_DROPOUT(ET, false, true);     \
    else MOE_LAUNCH_DROPOUT(ET, false, false);                 \
  } while (0)
  if (dtype == MOE_F32) MOE_LAUNCH_DROPOUT_ET(float);
  else MOE_LAUNCH_DROPOUT_ET(uint16_t);
#undef MOE_LAUNCH_DROPOUT_ET
#undef MOE_LAUNCH_DROPOUT
  return hipGetLastError();
}

hipError_t launch_ragged_rows(const int32_t* idx, const int32_t* loc, const int32_t* counts, int64_t T, int64_t E, int k, int64_t C, int32_t* offsets, int32_t* row_src,
                              int32_t* row_of, hipStream_t s) {
  ragged_rows_kernel<<<dim3(blocks_for(T * k, 256, 1024)), dim3(256), 0, s>>>(idx, loc, counts, T * k, (int)E, k, C > 0 ? C : T * k, offsets, row_src, row_of);
  return hipGetLastError();
}

hipError_t launch_ragged_combine(const void* Y, int64_t R, const int32_t* row_of, const float* gate_w, const void* residual, const Dropout& d, int dtype, int64_t T,
                                 int64_t M, int k, void* out, hipStream_t s) {
  const int groups = (int)(M / kGroup), per_row = (int)ceil_div(groups, 64);
  const int64_t units = T * per_row;
  const dim3 grid(blocks_for(units, 4, 1 << 20)), block(256);
  const bool stream = (double)R * M * (dtype == MOE_F32 ? 4 : 2) >= kStreamBytes;
#define MOE_LAUNCH_COMBINE(ET, STREAM, DROP)                                                                                                                        \
  ragged_combine_kernel<ET, STREAM, DROP><<<grid, block, 0, s>>>((const uint4*)Y, R, row_of, gate_w, (const uint4*)residual, d.seed, d.below, d.scale, units, per_row, \
                                                                 groups, k, (uint4*)out)
#define MOE_LAUNCH_COMBINE_ET(ET)                                \
  do {                                                           \
    if (stream && d.below) MOE_LAUNCH_COMBINE(ET, true, true);   \
    else if (stream) MOE_LAUNCH_COMBINE(ET, true, false);        \
    else if (d.below) MOE_LAUNCH_COMBINE(ET, false, true);       \
    else MOE_LAUNCH_COMBINE(ET, false, false);                   \
  } while (0)
  if (dtype == MOE_F32) MOE_LAUNCH_COMBINE_ET(float);
  else MOE_LAUNCH_COMBINE_ET(uint16_t);
#undef MOE_LAUNCH_COMBINE_ET
#undef MOE_LAUNCH_COMBINE
  return hipGetLastError();
}

hipError_t launch_ragged_combine_backward(const void* d_out, const void* Y, int64_t R, const int32_t* row_of, const float* gate_w, const Dropout& d, int dtype, int64_t T,
                                          int64_t M, int k, void* dY, float* dgate_w, hipStream_t s) {
  const int groups = (int)(M / kGroup);
  const bool stream = (double)R * M * (dtype == MOE_F32 ? 4 : 2) >= kStreamBytes, wide = groups > 128;
  const dim3 grid(blocks_for(T, wide ? 1 : 4, 1 << 20)), block(256);
#define MOE_LAUNCH_BACKWARD(ET, STREAM, DROP, W)                                                                                                                      \
  ragged_combine_backward_kernel<ET, STREAM, DROP, W><<<grid, block, 0, s>>>((const uint4*)d_out, (const uint4*)Y, R, row_of, gate_w, d.seed, d.below, d.scale, T, groups, \
                                                                             k, (uint4*)dY, dgate_w)
#define MOE_LAUNCH_BACKWARD_W(ET, STREAM, DROP)                \
  do {                                                         \
    if (wide) MOE_LAUNCH_BACKWARD(ET, STREAM, DROP, 4);        \
    else MOE_LAUNCH_BACKWARD(ET, STREAM, DROP, 1);             \
  } while (0)
#define MOE_LAUNCH_BACKWARD_ET(ET)                               \
  do {                                                           \
    if (stream && d.below) MOE_LAUNCH_BACKWARD_W(ET, true, true);   \
    else if (stream) MOE_LAUNCH_BACKWARD_W(ET, true, false);     \
    else if (d.below) MOE_LAUNCH_BACKWARD_W(ET, false, true);    \
    else MOE_LAUNCH_BACKWARD_W(ET, false, false);                \
  } while (0)
  if (dtype == MOE_F32) MOE_LAUNCH_BACKWARD_ET(float);
  else MOE_LAUNCH_BACKWARD_ET(uint16_t);
#undef MOE_LAUNCH_BACKWARD_ET
#undef MOE_LAUNCH_BACKWARD_W
#undef MOE_LAUNCH_BACKWARD
  return hipGetLastError();
}

size_t rows_act_backward_bytes(int64_t R, int64_t E, int64_t N) {
  const int64_t chunks = ceil_div(R, act_backward_chunk(R, E, N));
  return chunks > 1 ? (size_t)chunks * 2 * N * 4 : 0;
}

hipError_t launch_rows_act_backward(const void* dy, const void* pre, int act, int dtype, const int32_t* offsets, int64_t R, int64_t E, int64_t N, void* ws, void* dp,
                                    void* db, hipStream_t s) {
  if (act < 0 && !db) return hipSuccess;
  const int groups = (int)(N / kGroup);
  const int64_t chunk = act_backward_chunk(R, E, N), chunks = ceil_div(R, chunk);
  const dim3 grid((unsigned)ceil_div(groups, kStrip), (unsigned)chunks), block(256);
#define MOE_LAUNCH_ACT(ET, ACT, SUM) \
  rows_act_backward_kernel<ET, ACT, SUM><<<grid, block, 0, s>>>((const uint4*)dy, (const uint4*)pre, offsets, R, (int)E, groups, chunk, (uint4*)dp, (float*)ws, (ET*)db)
#define MOE_LAUNCH_ACT_SUM(ET, ACT)              \
  do {                                           \
    if (db) MOE_LAUNCH_ACT(ET, ACT, true);       \
    else MOE_LAUNCH_ACT(ET, ACT, false);         \
  } while (0)
#define MOE_LAUNCH_ACT_ET(ET)                                                   \
  do {                                                                          \
    switch (act) {                                                              \
      case MOE_ACT_RELU: MOE_LAUNCH_ACT_SUM(ET, MOE_ACT_RELU); break;           \
      case MOE_ACT_GELU: MOE_LAUNCH_ACT_SUM(ET, MOE_ACT_GELU); break;           \
      case MOE_ACT_SILU: MOE_LAUNCH_ACT_SUM(ET, MOE_ACT_SILU); break;           \
      default: MOE_LAUNCH_ACT(ET, -1, true);                                    \
    }                                                                           \
  } while (0)
  if (dtype == MOE_F32) MOE_LAUNCH_ACT_ET(float);
  else MOE_LAUNCH_ACT_ET(uint16_t);
#undef MOE_LAUNCH_ACT_ET
#undef MOE_LAUNCH_ACT_SUM
#undef MOE_LAUNCH_ACT
  if (hipError_t err = hipGetLastError()) return err;
  if (!db || chunks == 1) return hipSuccess;
  const dim3 sum_grid((unsigned)ceil_div(N, 64), (unsigned)E);
#define MOE_LAUNCH_CHUNK_SUM(ET)                                                                                                                                  \
  do {                                                                                                                                                            \
    if (chunks > 8 * E) chunk_sum_kernel<ET, 16><<<sum_grid, dim3(1024), 0, s>>>((const float*)ws, offsets, R, chunk, N, (ET*)db);                                \
    else chunk_sum_kernel<ET, 4><<<sum_grid, dim3(256), 0, s>>>((const float*)ws, offsets, R, chunk, N, (ET*)db);                                                 \
  } while (0)
  if (dtype == MOE_F32) MOE_LAUNCH_CHUNK_SUM(float);
  else MOE_LAUNCH_CHUNK_SUM(uint16_t);
#undef MOE_LAUNCH_CHUNK_SUM
  return hipGetLastError();
}

}  // namespace moe
