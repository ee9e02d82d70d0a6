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

// m: vocabulary, n: tokens.  STORE: the numerators too.  WIDE: fp32 numerators.
template <typename ID, bool STORE, bool WIDE>
struct LogitsEpilogue {
  static constexpr bool kWide = WIDE, kPaired = false;
  const ID *targets;
  float2 *stat;
  float *zt;
  char *E;
  int64_t T, V, ld, granules;
  // what the epilogue reads, read ahead of it
  template <int FN>
  struct Targets {
    int64_t y[FN];
  };
  template <int FN>
  __device__ __forceinline__ Targets<FN> hold(int64_t n0) const {
    Targets<FN> h;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t t = n0 + 16 * j + (threadIdx.x & 15);
      h.y[j] = t < T ? static_cast<int64_t>(targets[t]) : -1;
    }
    return h;
  }
  // stores of a wave where all of a tile's tokens are there
  template <int FM, int FN>
  static constexpr int stores() { return FN * (1 + (!STORE ? 0 : (WIDE ? FM : FM / 2))); }
  __device__ __forceinline__ bool whole(int64_t, int64_t n_end) const { return n_end <= T; }
  template <int FM, int FN>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[FM][FN], const Targets<FN> &held, int64_t m0, int64_t n0, int) const {
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
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
      const int64_t y = held.y[j] - m0 - 4 * q;
      if (__ballot(y >= 0 && y < FM * 16) != 0) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (y == 16 * i + e) zt[t] = acc[i][j][e];
      }
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
// (A count and a maximum: the same bits whoever takes them.)
template <int THREADS, typename ID>
__device__ __forceinline__ float common_weight(const ID *__restrict__ targets, const float *__restrict__ weight, int64_t T) {
  __shared__ float red[THREADS / 64];
  float most = 0.f;
  int count = 0;
  for (int64_t t = threadIdx.x; t < T; t += THREADS) {
    const bool counts = targets[t] >= 0;
    count += counts ? 1 : 0;
    if (weight && counts) most = fmaxf(most, fabsf(weight[t]));
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
template <typename ID>
__global__ __launch_bounds__(1024) void common_weight_kernel(const ID *__restrict__ targets, const float *__restrict__ weight, int64_t T,
                                                             float *__restrict__ common) {
  const float c = common_weight<1024>(targets, weight, T);
  if (threadIdx.x == 0) *common = c;
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
  bool take_common;     // row_kernel: T is all tokens, and `common` is not there yet
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

// a row's maximum (0 where there is none) and the sum of exp(z - that) from its granules
template <int WAVES>
__device__ __forceinline__ void join_granules(const float2 *stat, int64_t granules, float (*red)[16], float &base, float &sum) {
  const int tid = threadIdx.x % (WAVES * 64);
  float top = -INFINITY;
  sum = 0.f;
  for (int64_t p = tid; p < granules; p += WAVES * 64) top = fmaxf(top, stat[p].x);
  top = rows_max<WAVES>(top, red[0]);
  base = top == -INFINITY ? 0.f : top;
  for (int64_t p = tid; p < granules; p += WAVES * 64) sum += stat[p].y * expf(stat[p].x - base);
  sum = rows_sum<WAVES>(sum, red[1]);
}

template <typename F>
hipError_t dispatch_id(int id_dtype, F &&f) {
  if (id_dtype == MHCL_I64) return f(int64_t{});
  return f(int32_t{});
}

}  // namespace
}  // namespace mhcl
