// The head's softmax cross entropy, the loss of pairs of sequences that is made of it, and their gradients.
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
  if (t >= a.T || !a.counted(t)) return;
  float base, sum;
  join_granules<WAVES>(a.stat + t * a.granules, a.granules, red, base, sum);
  if (threadIdx.x % (WAVES * 64) == 0) {
    const int64_t u = a.token(t), y = static_cast<int64_t>(targets[u]);
    a.lse[u] = base + logf(sum);
    a.loss[u] = y < 0 ? 0.f : (y < a.V ? logf(sum) + (base - a.zt[t]) : __uint_as_float(0x7fc00000u));
  }
}

// The same, one block a token, and the row's numerators turned into g (turn_row).  Bound by memory: 16384 tokens, 65536 rows, bf16 980 us, 4.4 TB/s;
// 2048, 50257, fp32 154 us, 5.4 TB/s.
template <typename ID, typename IO>
__global__ __launch_bounds__(kBlock) void row_kernel(const RowArgs a, const ID *__restrict__ targets) {
  __shared__ float red[2][16];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  if (!a.counted(t)) return;
  const float2 *stat = a.stat + t * a.granules;
  float base, sum;
  join_granules<kBlock / 64>(stat, a.granules, red, base, sum);
  // (not by way of lse, in which log(sum) is lost where the logits are large)
  const int64_t u = a.token(t), y = static_cast<int64_t>(targets[u]);
  const float bad = __uint_as_float(0x7fc00000u);
  const float loss = y < 0 ? 0.f : (y < a.V ? logf(sum) + (base - a.zt[t]) : bad);
  if (tid == 0) {
    a.lse[u] = base + logf(sum);
    a.loss[u] = loss;
  }
  const float given = weight_over_common(a, targets, t, y);
  const float weight = y < a.V ? given : bad;
  const float hit = weight * expm1f(-loss);      // p - 1 of the target
  turn_row<IO>(a, t, stat, base, weight / sum, given != 0.f, [&](int64_t v, float (&g)[8]) {
    if (y >= v && y < v + 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = y == v + i ? hit : g[i];
    }
  });
}

// sum of weight loss over the targets that are not negative (null: over all), weights of 0 left out, or their mean; one block, in fp64
template <typename ID>
__global__ __launch_bounds__(1024) void total_kernel(const ID *__restrict__ targets, const float *__restrict__ loss,
                                                     const float *__restrict__ weight, int64_t T, float *__restrict__ total) {
  __shared__ double red[2][16];
  double sum = 0., count = 0.;
  for (int64_t t = threadIdx.x; t < T; t += 1024) {
    const float w = targets && targets[t] < 0 ? 0.f : (weight ? weight[t] : 1.f);
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

// Pairs of sequences, a block each: L = the sum of the tokens' -ce from one offset to the next, in fp64,
//   m = beta ((L_c - R_c) - (L_r - R_r)),  loss = (1 - s) softplus(-m) + s softplus(m)
// and the factor of each token's cross entropy in the weighted sum of the pairs, -+ beta weight dloss/dm for the chosen and the rejected sequence's,
// 0 outside of the sequences.  (loss, weights of tokens: few numbers, in fp64 until they are rounded.)  16 pairs of 8192 tokens 6.2 us, 2 of 300 4.0: a
// launch and two dependent reads.
// A token's weight is written by one block whatever the offsets are.  Those of pairs that ascend are taken as they are, so that a mistake stays in its pair;
// E, the furthest end of the ascending pairs before, is where their tokens end.  A pair writes from there on; it is a mistake as well where it begins
// before, and one that does not ascend writes nothing.  (Where all offsets ascend E is the pair's first one, and 0 for the first pair.)
constexpr int kPairThreads = 512;
template <typename OFF>
__global__ __launch_bounds__(kPairThreads) void pair_kernel(const PairArgs a, const OFF *__restrict__ offsets) {
  __shared__ double red[2][kPairThreads / 64];
  __shared__ int32_t ends[kPairThreads / 64];
  __shared__ float factor;
  const int64_t p = blockIdx.x;
  const int64_t from[3] = {static_cast<int64_t>(offsets[2 * p]), static_cast<int64_t>(offsets[2 * p + 1]), static_cast<int64_t>(offsets[2 * p + 2])};
  const bool right = ascends(offsets, p, a.T);
  const auto weighs = [&](int64_t i) { return !(a.weight && a.weight[i] == 0.f); };
  int32_t end = 0;          // E: a pair for each thread, or what pair_ends_kernel left
  if (a.pairs > kPairThreads) end = __float_as_int(a.loss[p]);
  else if (threadIdx.x < p && ascends(offsets, threadIdx.x, a.T)) end = static_cast<int32_t>(offsets[2 * threadIdx.x + 2]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) end = max(end, __shfl_xor(end, off, 64));
  if ((threadIdx.x & 63) == 0) ends[threadIdx.x >> 6] = end;
  double sum[2] = {0., 0.};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    for (int64_t t = from[i] + threadIdx.x; right && t < from[i + 1]; t += kPairThreads) sum[i] -= static_cast<double>(a.ce[t]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum[i] += __shfl_xor(sum[i], off, 64);
    if ((threadIdx.x & 63) == 0) red[i][threadIdx.x >> 6] = sum[i];
  }
  __syncthreads();
  for (int w = 0; w < kPairThreads / 64; ++w) end = max(end, ends[w]);
  const int64_t before = end;
  if (threadIdx.x == 0) {
    const bool bad = !right || (from[0] < before && from[0] < from[2]);
    double L[2] = {0., 0.}, ratio[2];
    for (int i = 0; i < 2; ++i) {
      for (int w = 0; w < kPairThreads / 64; ++w) L[i] += red[i][w];
      if (bad) L[i] = __longlong_as_double(0x7ff8000000000000ll);
      ratio[i] = L[i] - (a.reference ? static_cast<double>(a.reference[2 * p + i]) : 0.);
      a.logp[2 * p + i] = static_cast<float>(L[i]);
    }
    const double m = static_cast<double>(a.beta) * (ratio[0] - ratio[1]), s = a.smoothing;
    const double tail = log1p(exp(-fabs(m)));          // softplus(v) = max(v, 0) + tail
    a.loss[p] = static_cast<float>((s < 1. ? (1. - s) * ((m < 0. ? -m : 0.) + tail) : 0.) + (s > 0. ? s * ((m > 0. ? m : 0.) + tail) : 0.));
    const double slope = s / (1. + exp(-m)) - (1. - s) / (1. + exp(m));
    const double weight = a.weight ? static_cast<double>(a.weight[p]) : 1. / static_cast<double>(a.pairs);
    factor = weight == 0. ? 0.f : static_cast<float>(-static_cast<double>(a.beta) * slope * weight);
  }
  if (!a.token_weight) return;
  __syncthreads();
  // tokens that no pair's offsets claim any more: NaN where the pair that should have is a mistake that counts
  const float nan = __uint_as_float(0x7fc00000u);
  if (right) {
    const float gap = p > 0 && !ascends(offsets, p - 1, a.T) && weighs(p - 1) ? nan : 0.f;
    for (int64_t t = before + threadIdx.x; t < from[2]; t += kPairThreads) a.token_weight[t] = t < from[0] ? gap : (t < from[1] ? factor : -factor);
  }
  if (p == a.pairs - 1) {
    const float rest = !right && weighs(p) ? nan : 0.f;
    for (int64_t t = (right && from[2] > before ? from[2] : before) + threadIdx.x; t < a.T; t += kPairThreads) a.token_weight[t] = rest;
  }
}

// E of more pairs than a block of those has threads, left in the bits of `loss` until they replace it: a wave for a sixteenth of the pairs, 64 of them
// at a time, first for the furthest end of all and then, from that of the waves before on, pair by pair.  600 pairs 2.4 us, 100000 78 (pair_kernel: 6 and 290).
template <typename OFF>
__global__ __launch_bounds__(1024) void pair_ends_kernel(const PairArgs a, const OFF *__restrict__ offsets) {
  __shared__ int32_t ends[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int each = ((a.pairs + 15) / 16 + 63) / 64 * 64, first = min(wave * each, a.pairs), last = min(first + each, a.pairs);
  // (not under a condition: the loads of several pairs are side by side)
  const auto end_of = [&](int p) __attribute__((always_inline)) {
    const int64_t from = p < last ? p : a.pairs - 1;
    const bool right = ascends(offsets, from, a.T);
    const int64_t end = static_cast<int64_t>(offsets[2 * from + 2]);
    return right && p < last ? static_cast<int32_t>(end) : 0;
  };
  int32_t end = 0;
#pragma unroll 8
  for (int p = first + lane; p < last; p += 64) end = max(end, end_of(p));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) end = max(end, __shfl_xor(end, off, 64));
  if (lane == 0) ends[wave] = end;
  __syncthreads();
  int32_t before = 0;
  for (int w = 0; w < wave; ++w) before = max(before, ends[w]);
  int32_t next = first < last ? end_of(first + lane) : 0;
  for (int p0 = first; p0 < last; p0 += 64) {
    int32_t upto = next;
    next = end_of(p0 + 64 + lane);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int32_t other = __shfl_up(upto, off, 64);
      upto = lane >= off ? max(upto, other) : upto;
    }
    const int32_t here = __shfl_up(upto, 1, 64);
    if (p0 + lane < last) a.loss[p0 + lane] = __int_as_float(lane > 0 ? max(before, here) : before);
    before = max(before, __shfl(upto, 63, 64));
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

HeadPlan::HeadPlan(const mhcl_ends_desc &d, bool grad, bool ordered) {
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
    // (the device chooses, up to this, once it knows how many tokens there are: where they fill the chip many times over there is little to gain)
    if (ordered && h.tiles < 8 * (gh.bm == 256 ? kChipBlocks : 2 * kChipBlocks))
      gh_splits = static_cast<int>(std::max<int64_t>(gh_splits, std::min<int64_t>(4, h.steps / 8)));
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

HeadWs::HeadWs(const mhcl_ends_desc &d, bool grad, void *ws, bool ordered) : plan(d, grad, ordered) {
  WsCursor c(ws);
  const size_t T = static_cast<size_t>(plan.tokens), V = static_cast<size_t>(d.V), C = static_cast<size_t>(d.C), es = dtype_bytes(d.io_dtype);
  hp = grad ? c.take<char>(T * C * es) : nullptr;
  E = grad ? c.take<char>(T * static_cast<size_t>(plan.ld) * es) : nullptr;
  stat = c.take<float2>(T * static_cast<size_t>(plan.granules));
  zt = c.take<float>(T);
  common = c.take<float>(2);
  slabs = plan.gh_splits > 1 ? c.take<float>(static_cast<size_t>(plan.gh_splits) * T * C) : nullptr;
  gw_slabs = plan.gw_splits > 1 ? c.take<float>(static_cast<size_t>(plan.gw_splits) * V * C) : nullptr;
  gW = grad && !plan.wide && plan.tokens < d.T ? c.take<float>(V * C) : nullptr;
  bytes = c.off;
}

namespace {

// what of run_head is the cross entropy's
template <typename ID>
struct CrossEntropy {
  const ID *marks;          // the targets
  const float *weight;
  const HeadWs &w;
  hipStream_t s;
  TokenOrder order = {};
  const PairArgs *pairs = nullptr;
  static constexpr float factor = 1.f;
  static constexpr bool kLeavesOut = true;    // (taken in an order for the pairs alone, who read nothing of a token that does not count)
  hipError_t before(int64_t, int64_t) { return hipSuccess; }
  hipError_t between(const RowArgs &) { return hipSuccess; }
  PairLosses losses() const { return pairs ? PairLosses{pairs->loss, pairs->weight, pairs->pairs} : PairLosses{}; }
  template <bool ORDERED>
  TargetLogit<ID, ORDERED> wanted(int64_t t0) const {
    return {marks + (ORDERED ? 0 : t0), w.zt, ORDERED ? order.row + t0 : nullptr};
  }
  hipError_t loss(const RowArgs &a, int64_t t0) {
    if (a.row) t0 = 0;
    // (us, 50257 rows in granules of 32: a wave / a block of sixteen for one token 11.2 / 4.6)
    // (or, of pairs, where a wave holds a row's granules in registers: 300 tokens, 32 granules 4.5 / 3.8; the cross entropy alone keeps its bits)
    if (a.T < 1024 && !(pairs && a.granules <= kWaveGranules)) hipLaunchKernelGGL((loss_kernel<ID, 16>), dim3(static_cast<unsigned>(a.T)), dim3(1024), 0, s, a, marks + t0);
    else hipLaunchKernelGGL((loss_kernel<ID, 1>), dim3(blocks(a.T, kBlock / 64)), dim3(kBlock), 0, s, a, marks + t0);
    return hipGetLastError();
  }
  template <typename IO>
  hipError_t rows(const RowArgs &a, int64_t t0) {
    if (a.row) t0 = 0;
    hipLaunchKernelGGL((row_kernel<ID, IO>), dim3(static_cast<unsigned>(a.T)), dim3(kBlock), 0, s, a, marks + t0);
    return hipGetLastError();
  }
};

hipError_t launch_pairs(const PairArgs &a, const void *offsets, int offset_dtype, hipStream_t s) {
  if (a.pairs == 0) return a.token_weight ? launch_zero(a.token_weight, static_cast<size_t>(a.T) * 4, s) : hipSuccess;
  return dispatch_id(offset_dtype, [&](auto id) {
    using OFF = decltype(id);
    if (a.pairs > kPairThreads) {
      hipLaunchKernelGGL((pair_ends_kernel<OFF>), dim3(1), dim3(1024), 0, s, a, static_cast<const OFF *>(offsets));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((pair_kernel<OFF>), dim3(static_cast<unsigned>(a.pairs)), dim3(kPairThreads), 0, s, a, static_cast<const OFF *>(offsets));
    return hipGetLastError();
  });
}

// The cross entropy whose weights come of it: where all tokens are one block, their losses and the pairs' are taken between the logits and the rows
template <typename ID>
struct PairedCrossEntropy : CrossEntropy<ID> {
  const void *offsets;
  int offset_dtype;
  hipError_t between(const RowArgs &a) {
    const hipError_t e = this->loss(a, 0);
    return e != hipSuccess ? e : launch_pairs(*this->pairs, offsets, offset_dtype, this->s);
  }
};

}  // namespace

hipError_t launch_preference(const mhcl_ends_desc &d, const void *h, const void *W, const void *targets, const void *offsets, int offset_dtype,
                             PairArgs a, void *g_h, void *g_W, bool unrounded, const PreferenceWs &w, hipStream_t s) {
  const bool grad = g_W != nullptr;
  a.ce = w.ce;
  a.token_weight = grad ? w.token_weight : nullptr;
  if (d.T == 0) return launch_pairs(a, offsets, offset_dtype, s);
  return dispatch_id(d.id_dtype, [&](auto id) {
    return dispatch_io(d.io_dtype, [&](auto io) {
      using ID = decltype(id);
      using IO = decltype(io);
      const ID *y = static_cast<const ID *>(targets);
      hipError_t e;
      if (w.ordered && (e = launch_order(y, offsets, offset_dtype, a.pairs, d.T, w.order, s)) != hipSuccess) return e;
      const auto run = [&](auto &way, void *to_h, void *to_W, bool floats) {
        return w.ordered ? run_head<IO, true>(d, h, W, way, w.ce, w.lse, to_h, to_W, floats, w.head, s)
                         : run_head<IO, false>(d, h, W, way, w.ce, w.lse, to_h, to_W, floats, w.head, s);
      };
      if (grad && w.head.plan.tokens == d.T) {
        PairedCrossEntropy<ID> way{{y, w.token_weight, w.head, s, w.order, &a}, offsets, offset_dtype};
        return run(way, g_h, g_W, unrounded);
      }
      // several blocks of tokens: a pair's weight needs all of its tokens, so that their logits are formed twice
      CrossEntropy<ID> way{y, nullptr, w.head, s, w.order, &a};
      if ((e = run(way, nullptr, nullptr, false)) != hipSuccess) return e;
      if ((e = launch_pairs(a, offsets, offset_dtype, s)) != hipSuccess || !grad) return e;
      way.weight = w.token_weight;
      return run(way, g_h, g_W, unrounded);
    });
  });
}

hipError_t launch_head(const mhcl_ends_desc &d, const void *h, const void *W, const void *targets, const float *weight,
                       float *loss, float *lse, void *g_h, void *g_W, bool unrounded, const HeadWs &w, hipStream_t s) {
  return dispatch_id(d.id_dtype, [&](auto id) {
    return dispatch_io(d.io_dtype, [&](auto io) {
      using ID = decltype(id);
      CrossEntropy<ID> way{static_cast<const ID *>(targets), weight, w, s};
      return run_head<decltype(io), false>(d, h, W, way, loss, lse, g_h, g_W, unrounded, w, s);
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
