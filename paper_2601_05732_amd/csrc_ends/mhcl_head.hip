// The head's softmax cross entropy and its gradients.
//
//   z = h W^T                       [T, V]   never in memory
//   g = weight (softmax(z) - onehot)
//   g_h = g W,  g_W = g^T h
//
// Three matrix products of 2 T C V operations each.  The first one's epilogue takes, for each token, the maximum m and the sum of
// exp(z - m) over the rows of the vocabulary that a wave holds (a "granule"), and for the gradients leaves exp(z - m) in 16
// bits; a pass over a row then joins the granules, knows lse, and turns the numerators into g in place.  (Forming z again
// instead, once lse is known, is a fourth product: 2 C operations for each number in place of 4 bytes.)
#include <algorithm>

#include "mhcl_head_rows.h"

namespace mhcl {
namespace {

// loss and lse of a token: one wave each, or (WAVES > 1) a block each
template <typename ID, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kBlock : WAVES * 64) void loss_kernel(const RowArgs a, const ID *__restrict__ targets) {
  __shared__ float red[2][16];
  constexpr int TOKENS = WAVES == 1 ? kBlock / 64 : 1;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * TOKENS + (WAVES == 1 ? threadIdx.x >> 6 : 0);
  if (t >= a.T) return;
  float base, sum;
  join_granules<WAVES>(a.stat + t * a.granules, a.granules, red, base, sum);
  if (threadIdx.x % (WAVES * 64) == 0) {
    const int64_t y = static_cast<int64_t>(targets[t]);
    a.lse[t] = base + logf(sum);
    a.loss[t] = y < 0 ? 0.f : (y < a.V ? logf(sum) + (base - a.zt[t]) : __uint_as_float(0x7fc00000u));
  }
}

// The same, one block a token, and the row's numerators turned into g in their place, bf16 or (IO = F32) fp32; h's row into hp, zeros
// where the weight is 0.  bf16: g is of the operands' type, which is what the matrix units multiply with W and h.  (Its rounding is the one of the
// T V terms of a sum each, the gradient's own comes after it: off from 64 bits by 0.0023 of the 2-norm at 333 tokens and 0.0018 at 16384, where the
// gradient's rounding alone is 0.0017.  Two bf16 parts of g instead would make each of the two products two: 13 ms more on 21 at 16384
// tokens, C = 4096, 65536 rows.)  Bound by memory: 16384 tokens, 65536 rows, bf16 980 us, 4.4 TB/s; 2048, 50257, fp32 154 us, 5.4 TB/s.
template <typename ID, typename IO>
__global__ __launch_bounds__(kBlock) void row_kernel(const RowArgs a, const ID *__restrict__ targets) {
  __shared__ float red[2][16];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const float2 *stat = a.stat + t * a.granules;
  float base, sum;
  join_granules<kBlock / 64>(stat, a.granules, red, base, sum);
  // (not by way of lse, in which log(sum) is lost where the logits are large)
  const int64_t y = static_cast<int64_t>(targets[t]);
  const float bad = __uint_as_float(0x7fc00000u);
  const float loss = y < 0 ? 0.f : (y < a.V ? logf(sum) + (base - a.zt[t]) : bad);
  if (tid == 0) {
    a.lse[t] = base + logf(sum);
    a.loss[t] = loss;
  }
  float common = 1.f;
  if (a.take_common) {
    if (a.weight || t == 0) common = common_weight<kBlock>(targets, a.weight, a.T);
    if (t == 0 && tid == 0) *a.common = common;
  } else if (a.weight) {
    common = *a.common;
  }
  const float given = y < 0 ? 0.f : (a.weight ? a.weight[t] / common : 1.f);
  const bool counts = given != 0.f;
  const float weight = y < a.V ? given : bad;
  const float hit = weight * expm1f(-loss);      // p - 1 of the target
  const float scale = weight / sum;
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
      if (y >= v && y < v + 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = y == v + i ? hit : g[i];
      }
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
  for (int c = tid * IO::kVec; c < a.C; c += kBlock * IO::kVec) {
    float v[IO::kVec];
    IO::load(a.h, t * a.C + c, v);
#pragma unroll
    for (int i = 0; i < IO::kVec; ++i) v[i] = counts ? v[i] : 0.f;
    IO::store(a.hp, t * a.C + c, v);
  }
}

// sum of weight loss over the targets that are not negative, weights of 0 left out, or their mean; one block, in fp64
template <typename ID>
__global__ __launch_bounds__(1024) void total_kernel(const ID *__restrict__ targets, const float *__restrict__ loss,
                                                     const float *__restrict__ weight, int64_t T, float *__restrict__ total) {
  __shared__ double red[2][16];
  double sum = 0., count = 0.;
  for (int64_t t = threadIdx.x; t < T; t += 1024) {
    const float w = targets[t] < 0 ? 0.f : (weight ? weight[t] : 1.f);
    if (w != 0.f) sum += static_cast<double>(w) * loss[t];
    count += w != 0.f ? 1. : 0.;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    sum += __shfl_xor(sum, off, 64);
    count += __shfl_xor(count, off, 64);
  }
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = sum;
    red[1][threadIdx.x >> 6] = count;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) {
      sum += red[0][i];
      count += red[1][i];
    }
    *total = static_cast<float>(weight ? sum : (count > 0. ? sum / count : 0.));
  }
}

template <typename IO>
__global__ __launch_bounds__(kBlock) void scale_kernel(void *__restrict__ p, int64_t count, const float *__restrict__ factor) {
  const float f = *factor;
  if (f == 1.f) return;
  constexpr int VEC = IO::kVec;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kBlock * VEC;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * VEC; i < count; i += stride) {
    if (i + VEC <= count) {
      float v[VEC];
      IO::load(p, i, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] *= f;
      IO::store(p, i, v);
    } else {
      for (int64_t e = i; e < count; ++e) {
        if constexpr (VEC == 8) {
          uint16_t *q = static_cast<uint16_t *>(p);
          q[e] = f32_to_bf16(bf16_to_f32(q[e]) * f);
        } else {
          static_cast<float *>(p)[e] *= f;
        }
      }
    }
  }
}

// out = in times the factor, rounded once: what scale_kernel would round a second time.  Bound by memory:
// 268M numbers to bf16 344 us, 4.7 TB/s.
template <typename IO>
__global__ __launch_bounds__(kBlock) void scale_to_kernel(const float *__restrict__ in, void *__restrict__ out, int64_t count,
                                                          const float *__restrict__ factor) {
  const float f = *factor;
  constexpr int VEC = IO::kVec;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kBlock * VEC;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * VEC; i < count; i += stride) {
    if (i + VEC <= count) {
      float v[VEC];
#pragma unroll
      for (int e = 0; e < VEC; e += 4) F32::load(in, i + e, reinterpret_cast<float(&)[4]>(v[e]));
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] *= f;
      IO::store(out, i, v);
    } else {
      for (int64_t e = i; e < count; ++e) {
        if constexpr (VEC == 8) static_cast<uint16_t *>(out)[e] = f32_to_bf16(in[e] * f);
        else static_cast<float *>(out)[e] = in[e] * f;
      }
    }
  }
}

}  // namespace

HeadPlan::HeadPlan(const mhcl_ends_desc &d, bool grad) {
  wide = d.io_dtype == MHCL_F32;
  tokens = d.T;
  const int64_t row = ceil_div(d.V, 256) * 256;
  const int64_t row_bytes = grad ? row * (wide ? 4 : 2) : row / 32 * 8;
  const int64_t fit = static_cast<int64_t>(MHCL_HEAD_BLOCK_BYTES) / row_bytes / 256 * 256;
  if (tokens > fit) tokens = fit < 256 ? 256 : fit;
  if (tokens > d.T) tokens = d.T;
  logits = tile_for(d.V, tokens, 1, true, !wide);
  gh = tile_for(d.C, tokens, std::max<int64_t>(1, ceil_div(d.V, wide ? 32 : 64) / 8), true, !wide);
  gw = tile_for(d.C, d.V, 1, false, !wide);
  ld = ceil_div(d.V, logits.bm) * logits.bm;   // (what the first product's tiles cover)
  granules = ld / logits.gran;
  gh_splits = gw_splits = 1;
  pair = false;
  if (grad) {
    const Split h(gh, d.C, tokens, d.V, wide), w(gw, d.C, d.V, tokens, wide);
    gh_splits = h.best();
    if (tokens == d.T) gw_splits = w.best();   // (blocks of tokens add up in fp32 as they are)
    pair = gh.bm < 256 && gw.bm < 256 && h.tiles * gh_splits + w.tiles * gw_splits <= 2 * kChipBlocks;
    if (pair) {
      // side by side the shorter one need not be split (us, 333 tokens, C = 520, 1003 rows, bf16, g_h in two parts / one: 23.1 / 20.5)
      const auto time = [&](int i, int j) { return std::max(h.time(i), w.time(j)) + (i > 1 ? kSumTime : 0) + (j > 1 ? kSumTime : 0); };
      if (time(1, gw_splits) <= time(gh_splits, gw_splits)) gh_splits = 1;
      if (time(gh_splits, 1) <= time(gh_splits, gw_splits)) gw_splits = 1;
    }
  }
}

HeadWs::HeadWs(const mhcl_ends_desc &d, bool grad, void *ws) : plan(d, grad) {
  WsCursor c(ws);
  const size_t T = static_cast<size_t>(plan.tokens), V = static_cast<size_t>(d.V), C = static_cast<size_t>(d.C), es = dtype_bytes(d.io_dtype);
  hp = grad ? c.take<char>(T * C * es) : nullptr;
  E = grad ? c.take<char>(T * static_cast<size_t>(plan.ld) * es) : nullptr;
  stat = c.take<float2>(T * static_cast<size_t>(plan.granules));
  zt = c.take<float>(T);
  common = c.take<float>(1);
  slabs = plan.gh_splits > 1 ? c.take<float>(static_cast<size_t>(plan.gh_splits) * T * C) : nullptr;
  gw_slabs = plan.gw_splits > 1 ? c.take<float>(static_cast<size_t>(plan.gw_splits) * V * C) : nullptr;
  gW = grad && !plan.wide && plan.tokens < d.T ? c.take<float>(V * C) : nullptr;
  bytes = c.off;
}

namespace {

// the head of IO operands (bf16 or fp32)
template <typename ID, typename IO>
hipError_t run_head(const mhcl_ends_desc &d, const void *h, const void *W, const ID *targets, const float *weight, float *loss,
                    float *lse, void *g_h, void *g_W, bool unrounded, const HeadWs &w, hipStream_t s) {
  constexpr bool WIDE = IO::kVec == 4;
  const bool floats = WIDE || unrounded;   // what g_h and g_W are of
  const HeadPlan &p = w.plan;
  const bool grad = g_W != nullptr;
  const int64_t C = d.C, V = d.V, es = WIDE ? 4 : 2;
  hipError_t e;
  const bool take_common = d.T <= kCommonTokens && p.tokens == d.T;
  if (grad && !take_common) {
    hipLaunchKernelGGL((common_weight_kernel<ID>), dim3(1), dim3(1024), 0, s, targets, weight, d.T, w.common);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  int gran_log2 = 0;
  while ((1 << gran_log2) < p.logits.gran) ++gran_log2;
  for (int64_t t0 = 0; t0 < d.T; t0 += p.tokens) {
    const int64_t T = d.T - t0 < p.tokens ? d.T - t0 : p.tokens;
    const void *hb = static_cast<const char *>(h) + t0 * C * es;
    const ID *y = targets + t0;
    const Operand Wk{W, C, V, C}, hk{hb, C, T, C};
    const RowArgs a{hb, weight ? weight + t0 : nullptr, w.common, w.stat, w.zt, loss + t0, lse + t0, w.E, w.hp, T, p.ld, p.granules, d.V, d.C, gran_log2,
                    take_common};
    if (!grad) {
      const LogitsEpilogue<ID, false, WIDE> ep{y, w.stat, w.zt, w.E, T, V, p.ld, p.granules};
      if ((e = launch_gemm<true, true>(p.logits, Wk, hk, V, T, 1, ep, s)) != hipSuccess) return e;
      // (us, 50257 rows in granules of 32: a wave / a block of sixteen for one token 11.2 / 4.6)
      if (T < 1024) hipLaunchKernelGGL((loss_kernel<ID, 16>), dim3(static_cast<unsigned>(T)), dim3(1024), 0, s, a, y);
      else hipLaunchKernelGGL((loss_kernel<ID, 1>), dim3(blocks(T, kBlock / 64)), dim3(kBlock), 0, s, a, y);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      continue;
    }
    {
      const LogitsEpilogue<ID, true, WIDE> ep{y, w.stat, w.zt, w.E, T, V, p.ld, p.granules};
      if ((e = launch_gemm<true, true>(p.logits, Wk, hk, V, T, 1, ep, s)) != hipSuccess) return e;
    }
    hipLaunchKernelGGL((row_kernel<ID, IO>), dim3(static_cast<unsigned>(T)), dim3(kBlock), 0, s, a, y);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    // g_h [T, C]: m over C, n over the tokens, k over the vocabulary.  g_W [V, C]: m over C, n over the vocabulary, k over the tokens; the
    // blocks of tokens add up in fp32 (in g_W itself where it is fp32).
    const Operand Wm{W, C, C, V}, gk{w.E, p.ld, T, p.ld}, hm{w.hp, C, C, T}, gm{w.E, p.ld, p.ld, T};
    void *gh_out = static_cast<char *>(g_h) + t0 * C * (floats ? 4 : 2);
    float *sums = floats ? static_cast<float *>(g_W) : w.gW;
    const StoreEpilogue<WIDE> to_gh{w.common, p.gh_splits > 1 ? w.slabs : (floats ? static_cast<float *>(gh_out) : nullptr),
                                    static_cast<uint16_t *>(gh_out), nullptr, C, T, T * C};
    const StoreEpilogue<WIDE> to_gw{w.common, p.gw_splits > 1 ? w.gw_slabs : (floats || t0 + T < d.T ? sums : nullptr), static_cast<uint16_t *>(g_W),
                                    t0 > 0 ? sums : nullptr, C, V, V * C};
    if (p.pair) {
      const GemmArgs gh = gemm_args(p.gh, Wm, gk, C, T, p.gh_splits), gw = gemm_args(p.gw, hm, gm, C, V, p.gw_splits);
      const int first = gh.tiles_m * gh.tiles_n * gh.splits;
      const dim3 grid(first + gw.tiles_m * gw.tiles_n * gw.splits);
      if (p.gh.bn < 128) hipLaunchKernelGGL((gemm_pair_kernel<true, StoreEpilogue<WIDE>>), grid, dim3(256), 0, s, gh, to_gh, gw, to_gw, first);
      else hipLaunchKernelGGL((gemm_pair_kernel<false, StoreEpilogue<WIDE>>), grid, dim3(256), 0, s, gh, to_gh, gw, to_gw, first);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    } else {
      if ((e = launch_gemm<false, true>(p.gh, Wm, gk, C, T, p.gh_splits, to_gh, s)) != hipSuccess) return e;
      if ((e = launch_gemm<false, false>(p.gw, hm, gm, C, V, p.gw_splits, to_gw, s)) != hipSuccess) return e;
    }
    const auto join = floats ? launch_slab_sum<F32> : launch_slab_sum<IO>;
    if (p.gh_splits > 1 && (e = join(w.slabs, gh_out, p.gh_splits, T * C, s)) != hipSuccess) return e;
    if (p.gw_splits > 1 && (e = join(w.gw_slabs, g_W, p.gw_splits, V * C, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_head(const mhcl_ends_desc &d, const void *h, const void *W, const void *targets, const float *weight,
                       float *loss, float *lse, void *g_h, void *g_W, bool unrounded, const HeadWs &w, hipStream_t s) {
  return dispatch_id(d.id_dtype, [&](auto id) {
    return dispatch_io(d.io_dtype, [&](auto io) {
      using ID = decltype(id);
      return run_head<ID, decltype(io)>(d, h, W, static_cast<const ID *>(targets), weight, loss, lse, g_h, g_W, unrounded, w, s);
    });
  });
}

hipError_t launch_head_total(const mhcl_ends_desc &d, const void *targets, const float *loss, const float *weight, float *total,
                             hipStream_t s) {
  return dispatch_id(d.id_dtype, [&](auto id) {
    using ID = decltype(id);
    hipLaunchKernelGGL((total_kernel<ID>), dim3(1), dim3(1024), 0, s, static_cast<const ID *>(targets), loss, weight, d.T, total);
    return hipGetLastError();
  });
}

hipError_t launch_scale_to(const float *in, void *out, int dtype, int64_t count, const float *factor, hipStream_t s) {
  return dispatch_io(dtype, [&](auto io) {
    using IO = decltype(io);
    const int64_t want = ceil_div(count, kBlock * IO::kVec);
    hipLaunchKernelGGL((scale_to_kernel<IO>), dim3(static_cast<unsigned>(want < 4096 ? want : 4096)), dim3(kBlock), 0, s, in, out, count, factor);
    return hipGetLastError();
  });
}

hipError_t launch_scale(void *p, int dtype, int64_t count, const float *factor, hipStream_t s) {
  return dispatch_io(dtype, [&](auto io) {
    using IO = decltype(io);
    const int64_t want = ceil_div(count, kBlock * IO::kVec);
    hipLaunchKernelGGL((scale_kernel<IO>), dim3(static_cast<unsigned>(want < 4096 ? want : 4096)), dim3(kBlock), 0, s, p, count, factor);
    return hipGetLastError();
  });
}

}  // namespace mhcl
