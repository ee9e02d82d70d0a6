// What the head's losses share: the softmax's granules and numerators that the logits' product leaves, and the pass over a row that joins them.
#pragma once
#include "../csrc/mhcl_common.h"
#include "mhcl_head.h"
#include "mhcl_product.h"

namespace mhcl {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// ---- epilogues
// A number e in [0, 1] as 16 bits: 6 of the exponent, 10 of the mantissa (2^-62 .. 1 to 2^-11 of itself; what is less is off by up to 2^-63).  These are
// bits 28 .. 13 of e 2^-64.
constexpr float kCodeScale = 0x1p-64f;
__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
  return (__float_as_uint(lo * kCodeScale) + 0x1000u) >> 13 | ((__float_as_uint(hi * kCodeScale) + 0x1000u) << 3 & 0xffff0000u);
}
__device__ __forceinline__ float decode(uint32_t code) { return code ? __uint_as_float((code << 13) + (64u << 23)) : 0.f; }

// exp(x), x <= 0: the library's for fp32 operands; for bf16 ones by the instruction, to 2^-23 (1 + |x|) of itself, the rounding of
// x log2(e) and its own.  (The codes' 2^-64 is a product after it: as a term of the exponent, -64 + x log2(e), it would leave that an ulp of
// 2^-17 whatever x is, 2.6e-6 of every number and of the sums.)
template <bool WIDE>
__device__ __forceinline__ float exp_of(float x) {
  if constexpr (WIDE) return expf(x);
  return __builtin_amdgcn_exp2f(x * kLog2e);
}

// Which of a token's logits a loss reads as they are, taken from the sums: its target's.  (hold: what the epilogue reads, read ahead of it.)
// MAPPED: the product's token t is the caller's row[t].
template <typename ID, bool MAPPED = false>
struct TargetLogit {
  const ID *targets;
  float *zt;
  const int32_t *row;
  template <int FN>
  struct Held {
    int64_t y[FN];
  };
  template <int FM, int FN>
  __device__ __forceinline__ Held<FN> hold(int64_t, int64_t n0, int64_t T) const {
    Held<FN> h;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t t = n0 + 16 * j + (threadIdx.x & 15), from = t < T ? t : T - 1;    // (loads under a condition would wait for each other)
      h.y[j] = static_cast<int64_t>(targets[MAPPED ? row[from] : from]);
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) h.y[j] = n0 + 16 * j + (threadIdx.x & 15) < T ? h.y[j] : -1;
    return h;
  }
  __device__ __forceinline__ float factor() const { return 1.f; }
  static constexpr bool kFactor = false, kEarly = false;
  template <int FM, int FN>
  __device__ __forceinline__ void take(const f32x4 (&acc)[FM][FN], const Held<FN> &held, int j, int64_t t, int64_t m0, int q) const {
    const int64_t y = held.y[j] - m0 - 4 * q;
    if (__ballot(y >= 0 && y < FM * 16) != 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (y == 16 * i + e) zt[t] = acc[i][j][e];
    }
  }
};

// m: vocabulary, n: tokens.  STORE: the numerators too.  WIDE: fp32 numerators.  COUNTED: `tokens` bounds them.
template <typename Wanted, bool STORE, bool WIDE, bool COUNTED = false>
struct LogitsEpilogue {
  static constexpr bool kWide = WIDE, kPaired = false, kEarly = Wanted::kEarly, kCounted = COUNTED;
  Wanted wanted;
  float2 *stat;
  char *E;
  int64_t most, V, ld, granules;     // `most`: tokens
  TokenCount tokens;
  __device__ __forceinline__ int64_t rows() const {
    if constexpr (COUNTED) return tokens.of(most);
    return most;
  }
  template <int FM, int FN>
  __device__ __forceinline__ auto hold(int64_t m0, int64_t n0) const {
    return wanted.template hold<FM, FN>(m0, n0, rows());
  }
  // stores of a wave where all of a tile's tokens are there
  template <int FM, int FN>
  static constexpr int stores() { return FN * (1 + (!STORE ? 0 : (WIDE ? FM : FM / 2))); }
  __device__ __forceinline__ bool whole(int64_t, int64_t n_end) const { return n_end <= rows(); }
  template <int FM, int FN>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[FM][FN], const typename Wanted::template Held<FN> &held, int64_t m0, int64_t n0, int) const {
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int64_t T = rows();
    if constexpr (Wanted::kFactor) {
      const float f = wanted.factor();
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] *= f;
    }
    if (m0 + FM * 16 > V) {   // rows beyond the vocabulary
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool out = m0 + 16 * i + 4 * q + e >= V;
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j][e] = out ? -INFINITY : acc[i][j][e];
        }
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t t = n0 + 16 * j + r;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[i][j][e]);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      wanted.take(acc, held, j, t, m0, q);
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[i][j][e] = exp_of<WIDE>(acc[i][j][e] - base);
          sum += acc[i][j][e];
        }
        if constexpr (STORE && WIDE) {
          if (t < T) *reinterpret_cast<f32x4 *>(E + (t * ld + m0 + 16 * i + 4 * q) * 4) = acc[i][j];
        } else if constexpr (STORE) {
          if (i % 2 == 1) {
            const f32x4 u = acc[i - 1][j], v = acc[i][j];
            const uint4 eight = join_pairs(make_uint2(encode2(u[0], u[1]), encode2(u[2], u[3])),
                                           make_uint2(encode2(v[0], v[1]), encode2(v[2], v[3])));
            if (t < T) *reinterpret_cast<uint4 *>(E + (t * ld + m0 + 16 * (i - 1 + (q & 1)) + 8 * (q >> 1)) * 2) = eight;
          }
        }
      }
      sum += __shfl_xor(sum, 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      if (q == 0 && t < T) stat[t * granules + m0 / (FM * 16)] = make_float2(top, sum);
    }
  }
};

// ---------------------------------------------------------------- rows
// The factor c that all weights have in common, which the two products multiply their sums by: a token's g is rounded with weight / c
// alone, so that equal weights do not round a whole gradient's scale (16384 tokens, the mean's 1 / 15560 in bf16: g_h, g_W off by 0.0030 of their
// 2-norms with the weight in g, 0.0024 without).  The mean's: c = 1 / (targets that are not negative), weight / c = 1.  The caller's: c
// the largest |weight| of a target that is not negative (1 where that is no positive number).
// (A count and a maximum: the same bits whoever takes them.)  `factor`, what a loss multiplies every weight by, goes into c.
template <int THREADS, typename ID>
__device__ __forceinline__ float common_weight(const ID *__restrict__ targets, const float *__restrict__ weight, int64_t T) {
  __shared__ float red[THREADS / 64];
  float most = 0.f;
  int count = 0;
  // (four tokens' loads side by side, none under a condition, where each would wait for the one before: 16384 tokens 10.0 us / 5.3)
  for (int64_t t = threadIdx.x; t < T; t += 4 * THREADS) {
    ID y[4];
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = targets[t + i * THREADS < T ? t + i * THREADS : t];
    if (weight) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = weight[t + i * THREADS < T ? t + i * THREADS : t];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool counts = t + i * THREADS < T && y[i] >= 0;
      count += counts ? 1 : 0;
      if (weight && counts) most = fmaxf(most, fabsf(w[i]));
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    most = fmaxf(most, __shfl_xor(most, off, 64));
    count += __shfl_xor(count, off, 64);
  }
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = weight ? most : __int_as_float(count);
  __syncthreads();
  int all = 0;
  for (int i = 0; i < THREADS / 64; ++i) {
    most = fmaxf(most, weight ? red[i] : 0.f);
    all += weight ? 0 : __float_as_int(red[i]);
  }
  if (!weight) most = all > 0 ? 1.f / static_cast<float>(all) : 0.f;
  return most > 0.f && most <= 3.4028235e38f ? most : 1.f;
}
// Up to so many tokens the rows' kernel takes it itself: each of its blocks, or the first alone where only the products need it.  (us,
// 333 tokens, C = 520, 1003 rows, bf16, weights, the whole call with a launch for it / without: 31.0 / 29.5.)
constexpr int64_t kCommonTokens = 1024;

// Losses of pairs and their weights.  Where one is NaN all of g_W is, unless its weight is 0: by way of g_W's common weight, since a pair whose
// offsets are a mistake may have no token to be NaN in.
struct PairLosses {
  const float *loss, *weight;
  int32_t count;
  template <int THREADS>
  __device__ __forceinline__ float times(float common) const {
    if (count == 0) return common;
    __shared__ int red[THREADS / 64];
    bool lost = false;
#pragma unroll 8
    for (int p = threadIdx.x; p < count; p += THREADS) {
      const float w = weight ? weight[p] : 1.f;
      lost |= isnan(loss[p]) & (w != 0.f);
    }
    const bool any = __ballot(lost) != 0;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = any ? 1 : 0;
    __syncthreads();
    for (int w = 0; w < THREADS / 64; ++w) common = red[w] ? __uint_as_float(0x7fc00000u) : common;
    return common;
  }
};
template <typename ID>
__global__ __launch_bounds__(1024) void common_weight_kernel(const ID *__restrict__ targets, const float *__restrict__ weight, int64_t T,
                                                             float factor, const PairLosses pairs, float *__restrict__ common) {
  const float c = common_weight<1024>(targets, weight, T) * factor, of_W = pairs.times<1024>(c);
  if (threadIdx.x == 0) {
    common[0] = c;
    common[1] = of_W;
  }
}

struct RowArgs {
  const void *h;
  const float *weight;
  float *common;
  const float2 *stat;
  const float *zt;
  float *loss, *lse;
  char *E, *hp;
  int64_t T, ld, granules;
  int32_t V;
  int C, gran_log2;
  float factor;         // of all weights
  bool take_common;     // row kernels: T is all tokens, and `common` is not there yet
  PairLosses pairs;
  // Tokens in an order of their own: token t is the caller's row[t], h's rows lie in hp already, and those past the count have no gradient (null: none of
  // this)
  const int32_t *row;
  TokenCount tokens;
  __device__ __forceinline__ int64_t token(int64_t t) const { return row ? row[t] : t; }
  __device__ __forceinline__ bool counted(int64_t t) const { return !row || tokens.first + t < *tokens.count; }
};

// sum, and the largest, of a value over the WAVES waves of a token
template <int WAVES>
__device__ __forceinline__ float rows_sum(float v, float *red) {
  v = wave_sum(v);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = pairwise_sum<WAVES>([&](int w) { return red[w]; });
  }
  return v;
}
template <int WAVES>
__device__ __forceinline__ float rows_max(float v, float *red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v = fmaxf(v, red[w]);
  }
  return v;
}

// a row's maximum (0 where there is none) and the sum of exp(z - that) from its granules; the first ones of a lane stay in registers from the one to the
// other (us, 50257 rows in granules of 128, 8192 tokens a wave each, with 32 slots: read twice 11.5, so 8.3)
constexpr int64_t kWaveGranules = 512;     // that a wave holds
template <int WAVES>
__device__ __forceinline__ void join_granules(const float2 *stat, int64_t granules, float (*red)[16], float &base, float &sum) {
  constexpr int STRIDE = WAVES * 64, HELD = WAVES == 1 ? kWaveGranules / 64 : (WAVES <= 4 ? 4 : 1);
  const int tid = threadIdx.x % STRIDE;
  float2 held[HELD];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < HELD; ++i) held[i] = stat[tid + i * STRIDE < granules ? tid + i * STRIDE : granules - 1];   // (again: not under a condition)
#pragma unroll
  for (int i = 0; i < HELD; ++i) top = fmaxf(top, held[i].x);      // (the last one's once more is no other maximum)
  for (int64_t p = tid + HELD * STRIDE; p < granules; p += STRIDE) top = fmaxf(top, stat[p].x);
  top = rows_max<WAVES>(top, red[0]);
  base = top == -INFINITY ? 0.f : top;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (tid + i * STRIDE < granules) sum += held[i].y * expf(held[i].x - base);
  for (int64_t p = tid + HELD * STRIDE; p < granules; p += STRIDE) sum += stat[p].y * expf(stat[p].x - base);
  sum = rows_sum<WAVES>(sum, red[1]);
}

// A token's weight over what all have in common, which a block of threads leaves for the products where it is not there yet; y < 0: none
template <typename ID>
__device__ __forceinline__ float weight_over_common(const RowArgs &a, const ID *__restrict__ targets, int64_t t, int64_t y) {
  float common = 1.f;
  if (a.take_common) {
    if (a.weight || t == 0) common = common_weight<kBlock>(targets, a.weight, a.T) * a.factor;
    if (t == 0) {
      const float of_W = a.pairs.times<kBlock>(common);
      if (threadIdx.x == 0) {
        a.common[0] = common;
        a.common[1] = of_W;
      }
    }
  } else if (a.weight) {
    common = *a.common;
  }
  return y < 0 ? 0.f : (a.weight ? a.weight[a.token(t)] * a.factor / common : 1.f);
}

// The row's numerators turned into scale exp(z - base) in their place, `replace(v, g)` having the last word on the eight from v on; zeros, and zeros
// for h's row, where the token does not count.  bf16: g is of the operands' type, which is what the matrix units multiply with W and h.  (Its
// rounding is the one of the T V terms of a sum each, the gradient's own comes after it: off from 64 bits by 0.0023 of the 2-norm at 333 tokens and
// 0.0018 at 16384, where the gradient's rounding alone is 0.0017.  Where few entries outweigh the rest their roundings do not
// average, and the sum may be as far off as one of them, 2^-8.  Two bf16 parts of g instead would make each of the two products two: 13 ms
// more on 21 at 16384 tokens, C = 4096, 65536 rows.)
template <typename IO, typename F>
__device__ __forceinline__ void turn_row(const RowArgs &a, int64_t t, const float2 *stat, float base, float scale, bool counts, F &&replace) {
  const int tid = threadIdx.x;
  for (int64_t v = tid * 8; v < a.ld; v += kBlock * 8) {
    float g[8];
    if (counts) {
      const float f = scale * expf(stat[v >> a.gran_log2].x - base);
      if constexpr (IO::kVec == 8) {
        const uint4 c = *reinterpret_cast<const uint4 *>(a.E + (t * a.ld + v) * 2);
        const uint32_t code[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[2 * i] = decode(code[i] & 0xffffu) * f;
          g[2 * i + 1] = decode(code[i] >> 16) * f;
        }
      } else {
        F32::load(a.E, t * a.ld + v, reinterpret_cast<float(&)[4]>(g[0]));
        F32::load(a.E, t * a.ld + v + 4, reinterpret_cast<float(&)[4]>(g[4]));
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] *= f;
      }
      replace(v, g);
      if (v + 8 > a.V) {                         // (a row of NaN leaves the fill-up finite)
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = v + i < a.V ? g[i] : 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = 0.f;
    }
    if constexpr (IO::kVec == 8) {
      BF16::store(a.E, t * a.ld + v, g);
    } else {
      F32::store(a.E, t * a.ld + v, reinterpret_cast<const float(&)[4]>(g[0]));
      F32::store(a.E, t * a.ld + v + 4, reinterpret_cast<const float(&)[4]>(g[4]));
    }
  }
  if (a.row && counts) return;
  for (int c = tid * IO::kVec; c < a.C; c += kBlock * IO::kVec) {
    float v[IO::kVec];
    IO::load(a.h, t * a.C + c, v);
#pragma unroll
    for (int i = 0; i < IO::kVec; ++i) v[i] = counts ? v[i] : 0.f;
    IO::store(a.hp, t * a.C + c, v);
  }
}

template <typename F>
hipError_t dispatch_id(int id_dtype, F &&f) {
  if (id_dtype == MHCL_I64) return f(int64_t{});
  return f(int32_t{});
}

// Whether a pair's three offsets ascend within 0 .. T, which the host cannot see
template <typename OFF>
__device__ __forceinline__ bool ascends(const OFF *__restrict__ offsets, int64_t p, int64_t T) {
  const int64_t o[3] = {static_cast<int64_t>(offsets[2 * p]), static_cast<int64_t>(offsets[2 * p + 1]), static_cast<int64_t>(offsets[2 * p + 2])};
  return (o[0] >= 0) & (o[0] <= o[1]) & (o[1] <= o[2]) & (o[2] <= T);
}

// ---------------------------------------------------------------- order of the tokens
// Tokens that count first, each kind in the caller's order: of kOrderTokens of them by a block of threads, which counts its own, and then, knowing
// those of the blocks before, places them; a wave has 16 times 64.  A token counts where its target is not negative and (offsets) it lies from the first
// offset to the last, if all of them ascend within 0 .. T: where they do not, the ends say nothing about the pairs between them.
constexpr int kOrderTokens = kBlock * 16;
template <typename ID, typename OFF>
struct Counting {
  const ID *targets;
  const OFF *offsets;       // null: all tokens
  int64_t pairs;
  struct Range {
    int64_t from, to;
  };
  // by a block of threads
  __device__ __forceinline__ Range range(int64_t T) const {
    if (!offsets) return {0, T};
    if (pairs == 0) return {0, 0};
    __shared__ int red[kBlock / 64];
    bool wrong = false;
#pragma unroll 8
    for (int64_t p = threadIdx.x; p < pairs; p += kBlock) wrong |= !ascends(offsets, p, T);
    const bool any = __ballot(wrong) != 0;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = any ? 1 : 0;
    const int64_t from = static_cast<int64_t>(offsets[0]), to = static_cast<int64_t>(offsets[2 * pairs]);
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3] == 0 ? Range{from, to} : Range{0, T};
  }
  // a bit each for the lane's tokens t0 + 64 i whose targets are not negative, and those of them in a range
  __device__ __forceinline__ uint32_t sixteen(int64_t t0, int64_t T) const {
    ID y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = targets[t0 + 64 * i < T ? t0 + 64 * i : T - 1];     // (a load under a condition would wait for the one before)
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) bits |= t0 + 64 * i < T && y[i] >= 0 ? 1u << i : 0u;
    return bits;
  }
  __device__ __forceinline__ uint32_t within(uint32_t bits, int64_t t0, Range r) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) bits &= t0 + 64 * i >= r.from && t0 + 64 * i < r.to ? ~0u : ~(1u << i);
    return bits;
  }
};
__device__ __forceinline__ int64_t order_token(int64_t block) { return block * kOrderTokens + (threadIdx.x >> 6) * 1024 + (threadIdx.x & 63); }
template <typename ID, typename OFF>
__global__ __launch_bounds__(kBlock) void order_count_kernel(const Counting<ID, OFF> c, int64_t T, int32_t *__restrict__ counts) {
  __shared__ int red[kBlock / 64];
  const int64_t t0 = order_token(blockIdx.x);
  const uint32_t bits = c.sixteen(t0, T);
  int n = __popc(c.within(bits, t0, c.range(T)));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) counts[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}
// counts null: every block counts all tokens itself
template <typename ID, typename OFF>
__global__ __launch_bounds__(kBlock) void order_place_kernel(const Counting<ID, OFF> c, int64_t T, const int32_t *__restrict__ counts, int32_t *__restrict__ row,
                                                             int32_t *__restrict__ count) {
  __shared__ int red[3][kBlock / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t0 = order_token(blockIdx.x);
  uint32_t bits = c.sixteen(t0, T);
  const auto range = c.range(T);
  bits = c.within(bits, t0, range);
  int mine = __popc(bits), before = 0, all = 0;
  if (counts) {
    for (unsigned b = threadIdx.x; b < gridDim.x; b += kBlock) {
      all += counts[b];
      before += b < blockIdx.x ? counts[b] : 0;
    }
  } else {
    for (unsigned b = 0; b < gridDim.x; ++b) {
      const int n = __popc(c.within(c.sixteen(order_token(b), T), order_token(b), range));
      all += n;
      before += b < blockIdx.x ? n : 0;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    mine += __shfl_xor(mine, off, 64);
    before += __shfl_xor(before, off, 64);
    all += __shfl_xor(all, off, 64);
  }
  if (lane == 0) {
    red[0][wave] = mine;
    red[1][wave] = before;
    red[2][wave] = all;
  }
  __syncthreads();
  int at = 0;               // tokens that count before the wave's next 64
  all = 0;
  for (int w = 0; w < kBlock / 64; ++w) {
    at += red[1][w] + (w < wave ? red[0][w] : 0);
    all += red[2][w];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *count = all;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const bool counts_here = bits >> i & 1;
    const uint64_t there = __ballot(counts_here);
    const int64_t t = t0 + 64 * i;
    const int here = at + __popcll(there & ((uint64_t{1} << lane) - 1));
    if (t < T) row[counts_here ? here : all + (t - here)] = static_cast<int32_t>(t);
    at += __popcll(there);
  }
}

// us: the order of 16384 tokens 7.4, of 8192 of 16 pairs 7.2; gathering 16384 rows, C = 4096 44, 6 TB/s, of 8192 the 5560 that count 21.
// h's rows in the order of the tokens, a wave each; of those past the count, zeros in g_h and `ce` where they are (null: neither)
template <typename IO>
__global__ __launch_bounds__(kBlock) void gather_kernel(const void *__restrict__ h, char *__restrict__ hp, int64_t T, int C, const int32_t *__restrict__ row,
                                                        TokenCount tokens, bool all, void *__restrict__ g_h, int g_pieces, float *__restrict__ ce) {
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kBlock / 64) + (threadIdx.x >> 6);
  if (t >= T) return;
  const int lane = threadIdx.x & 63, pieces = C / IO::kVec;
  const int64_t from = row[t];
  const bool counts = t < tokens.of(T);
  if (counts || all)
    for (int p = lane; p < pieces; p += 64) reinterpret_cast<uint4 *>(hp)[t * pieces + p] = static_cast<const uint4 *>(h)[from * pieces + p];
  if (counts) return;
  if (g_h)
    for (int p = lane; p < g_pieces; p += 64) static_cast<uint4 *>(g_h)[from * g_pieces + p] = make_uint4(0, 0, 0, 0);
  if (ce && lane == 0) ce[from] = 0.f;
}

template <typename ID>
hipError_t launch_order(const ID *targets, const void *offsets, int offset_dtype, int64_t pairs, int64_t T, const TokenOrder &o, hipStream_t s) {
  return dispatch_id(offset_dtype, [&](auto off) {
    using OFF = decltype(off);
    const Counting<ID, OFF> c{targets, static_cast<const OFF *>(offsets), pairs};
    const dim3 grid(blocks(T, kOrderTokens));
    const bool apart = grid.x > 16;      // (a launch of its own costs more than counting 65536 tokens sixteen times)
    if (apart) {
      hipLaunchKernelGGL((order_count_kernel<ID, OFF>), grid, dim3(kBlock), 0, s, c, T, o.counts);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((order_place_kernel<ID, OFF>), grid, dim3(kBlock), 0, s, c, T, apart ? o.counts : nullptr, o.row, o.count);
    return hipGetLastError();
  });
}

// The head's products with a loss of the logits, of IO operands (bf16 or fp32).  The loss `way` gives
//   before(t0, T)            what a block of tokens needs before its logits
//   wanted(t0)               which logits it reads as they are
//   loss(a, t0), rows(a, t0) the launches that form the losses of a block; and besides turn its numerators into gradients on the logits
//   between(a)               what the first block needs between its logits and its rows
//   marks, weight            ([all tokens]: negative where a token does not count) and its `factor`
//   losses()                 of pairs, if its weights come of them
// ORDERED: the tokens are taken in way.order's order, and those that do not count are left out of the gradients' products, and (way.kLeavesOut) of the
// logits'.  (us, without / with: 8192 tokens, of which 5700 count, C = 4096, 65536 rows,
// pairs 10230 / 7840, their loss alone 3194 / 2367, distillation 10255 / 8692; all 8192 count 10560 / 10730.)
template <typename IO, bool ORDERED, typename Way>
hipError_t run_head(const mhcl_ends_desc &d, const void *h, const void *W, Way &way, float *loss, float *lse, void *g_h, void *g_W, bool unrounded,
                    const HeadWs &w, hipStream_t s) {
  constexpr bool WIDE = IO::kVec == 4;
  const bool floats = WIDE || unrounded;   // what g_h and g_W are of
  const HeadPlan &p = w.plan;
  const bool grad = g_W != nullptr;
  const int64_t C = d.C, V = d.V, es = WIDE ? 4 : 2;
  hipError_t e;
  const bool take_common = !ORDERED && d.T <= kCommonTokens && p.tokens == d.T;
  int gran_log2 = 0;
  while ((1 << gran_log2) < p.logits.gran) ++gran_log2;
  for (int64_t t0 = 0; t0 < d.T; t0 += p.tokens) {
    const int64_t T = d.T - t0 < p.tokens ? d.T - t0 : p.tokens;
    const TokenCount tokens{ORDERED ? way.order.count : nullptr, t0, 0, 0, 0, 0, 0};
    const int32_t *row = ORDERED ? way.order.row + t0 : nullptr;
    const int64_t shift = ORDERED ? 0 : t0;      // of what lies in the caller's order
    const void *hb = ORDERED ? way.order.hp : static_cast<const char *>(h) + t0 * C * es;
    const Operand Wk{W, C, V, C}, hk{hb, C, T, C};
    const RowArgs a{hb, way.weight ? way.weight + shift : nullptr, w.common, w.stat, w.zt, loss + shift, lse + shift, w.E, way.order.hp ? way.order.hp : w.hp,
                    T, p.ld, p.granules, d.V, d.C, gran_log2, way.factor, take_common, way.losses(), row, tokens};
    if constexpr (ORDERED) {
      hipLaunchKernelGGL((gather_kernel<IO>), dim3(blocks(T, kBlock / 64)), dim3(kBlock), 0, s, h, way.order.hp, T, d.C, row, tokens, !Way::kLeavesOut,
                         g_h, static_cast<int>(C * (floats ? 4 : 2) / 16), Way::kLeavesOut ? loss : nullptr);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if ((e = way.before(t0, T)) != hipSuccess) return e;
    const auto wanted = way.template wanted<ORDERED>(t0);
    using Wanted = std::decay_t<decltype(wanted)>;
    constexpr bool COUNTED = ORDERED && Way::kLeavesOut;
    if (!grad) {
      const LogitsEpilogue<Wanted, false, WIDE, COUNTED> ep{wanted, w.stat, w.E, T, V, p.ld, p.granules, tokens};
      if ((e = launch_gemm<true, true>(p.logits, Wk, hk, V, T, 1, ep, s, tokens)) != hipSuccess) return e;
      if ((e = way.loss(a, t0)) != hipSuccess) return e;
      continue;
    }
    {
      const LogitsEpilogue<Wanted, true, WIDE, COUNTED> ep{wanted, w.stat, w.E, T, V, p.ld, p.granules, tokens};
      if ((e = launch_gemm<true, true>(p.logits, Wk, hk, V, T, 1, ep, s, tokens)) != hipSuccess) return e;
    }
    if (t0 == 0) {
      if ((e = way.between(a)) != hipSuccess) return e;
      if (!take_common) {
        using ID = std::remove_cv_t<std::remove_pointer_t<decltype(way.marks)>>;
        hipLaunchKernelGGL((common_weight_kernel<ID>), dim3(1), dim3(1024), 0, s, way.marks, way.weight, d.T, way.factor, way.losses(), w.common);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
    }
    if ((e = way.template rows<IO>(a, t0)) != hipSuccess) return e;
    // g_h [T, C]: m over C, n over the tokens, k over the vocabulary.  g_W [V, C]: m over C, n over the vocabulary, k over the tokens; the
    // blocks of tokens add up in fp32 (in g_W itself where it is fp32).
    const Operand Wm{W, C, C, V}, gk{w.E, p.ld, T, p.ld}, hm{a.hp, C, C, T}, gm{w.E, p.ld, p.ld, T};
    void *gh_out = static_cast<char *>(g_h) + shift * C * (floats ? 4 : 2);
    float *sums = floats ? static_cast<float *>(g_W) : w.gW;
    const bool parts = p.gh_splits > 1;
    using Store = StoreEpilogue<WIDE, ORDERED>;
    TokenCount gh_tokens = tokens;
    if (ORDERED && parts) {
      gh_tokens.tiles_m = static_cast<int>(ceil_div(C, p.gh.bm));
      gh_tokens.bn = p.gh.bn;
      gh_tokens.steps = static_cast<int>(ceil_div(V, WIDE ? 32 : 64));
      gh_tokens.alone = alone_time(WIDE);
      gh_tokens.most_parts = p.gh_splits;
    }
    const Store to_gh{w.common, parts && !ORDERED ? w.slabs : (floats ? static_cast<float *>(gh_out) : nullptr), static_cast<uint16_t *>(gh_out), nullptr, C, T,
                      T * C, row, gh_tokens, false, ORDERED && parts ? w.slabs : nullptr};
    const Store to_gw{w.common + 1, p.gw_splits > 1 ? w.gw_slabs : (floats || t0 + T < d.T ? sums : nullptr), static_cast<uint16_t *>(g_W),
                      t0 > 0 ? sums : nullptr, C, V, V * C, nullptr, tokens, true, nullptr};
    if (p.pair) {
      const GemmArgs gh = gemm_args(p.gh, Wm, gk, C, T, p.gh_splits, gh_tokens), gw = gemm_args(p.gw, hm, gm, C, V, p.gw_splits, tokens, true);
      const int first = gh.tiles_m * gh.tiles_n * gh.splits;
      const dim3 grid(first + gw.tiles_m * gw.tiles_n * gw.splits);
      if (p.gh.bn < 128) hipLaunchKernelGGL((gemm_pair_kernel<true, Store>), grid, dim3(256), 0, s, gh, to_gh, gw, to_gw, first);
      else hipLaunchKernelGGL((gemm_pair_kernel<false, Store>), grid, dim3(256), 0, s, gh, to_gh, gw, to_gw, first);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    } else {
      if ((e = launch_gemm<false, true>(p.gh, Wm, gk, C, T, p.gh_splits, to_gh, s, gh_tokens)) != hipSuccess) return e;
      if ((e = launch_gemm<false, false>(p.gw, hm, gm, C, V, p.gw_splits, to_gw, s, tokens, true)) != hipSuccess) return e;
    }
    const auto join = floats ? launch_slab_sum<F32> : launch_slab_sum<IO>;
    if (parts && ORDERED) {
      const dim3 grid(blocks(T * C, kBlock * 4));
      if (floats) hipLaunchKernelGGL((slab_sum_rows_kernel<F32>), grid, dim3(kBlock), 0, s, w.slabs, gh_out, T, C, row, gh_tokens);
      else hipLaunchKernelGGL((slab_sum_rows_kernel<IO>), grid, dim3(kBlock), 0, s, w.slabs, gh_out, T, C, row, gh_tokens);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    } else if (parts && (e = join(w.slabs, gh_out, p.gh_splits, T * C, s)) != hipSuccess) {
      return e;
    }
    if (p.gw_splits > 1 && (e = join(w.gw_slabs, g_W, p.gw_splits, V * C, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace
}  // namespace mhcl
