// The head against a teacher's top logits, and its gradients.
//
//   p_k = exp(a_k) / sum_j exp(a_j),  a = teacher's logits / tau        over a token's slots that hold one
//   z   = h W^T / tau                                                   [T, V]  never in memory
//   loss = sum_k p_k (log p_k - log q[id_k]),  q = softmax(z)
//   g = weight (q - p) / tau,  g_h = g W,  g_W = g^T h
//
// The cross entropy's products and passes (mhcl_head_rows.h) with K logits of a token in place of one: they are put in order of
// their ids first, so that a wave of the first product finds by one look into a table which of them lie in its granule, and takes them
// from its sums.  (A product of h with the K rows instead would read K C numbers a token again.)
#include "mhcl_head_rows.h"

namespace mhcl {
namespace {

// A token's slots, by a wave: a slot is empty where its id is negative or its logit is the lowest there is (-infinity).  LISTS: else the mark alone.
template <typename ID, bool LISTS>
__global__ __launch_bounds__(kBlock) void teacher_kernel(const ID *__restrict__ ids, const float *__restrict__ logits, int64_t T, int32_t K, int32_t V,
                                                         float inv, int gran_log2, int64_t granules, int32_t *__restrict__ mark,
                                                         int32_t *__restrict__ id_out, float2 *__restrict__ p_out, uint16_t *__restrict__ start) {
  constexpr int WAVES = kBlock / 64, PER = kMostSlots / 64;
  __shared__ int32_t key[LISTS ? WAVES : 1][kMostSlots], sorted[LISTS ? WAVES : 1][kMostSlots];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * WAVES + wave;
  if (t >= T) return;      // (waves do not meet)
  float a[PER], top = -INFINITY, sum = 0.f;
  int32_t mine[PER];
  int held = 0, past = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = i * 64 + lane;
    a[i] = -INFINITY;
    mine[i] = 0x7fffffff;
    if (k < K) {
      const int64_t id = static_cast<int64_t>(ids[t * K + k]);
      const float v = logits[t * K + k] * inv;
      const bool there = id >= 0 && !(v == -INFINITY);
      if (there) a[i] = v;
      if (there && id < V) mine[i] = static_cast<int32_t>(id);
      held += there ? 1 : 0;
      past += there && id >= V ? 1 : 0;
    }
    top = fmaxf(top, a[i]);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    top = fmaxf(top, __shfl_xor(top, off, 64));
    held += __shfl_xor(held, off, 64);
    past += __shfl_xor(past, off, 64);
  }
  if (lane == 0) mark[t] = held == 0 ? -1 : (past != 0 ? 1 : 0);
  if constexpr (LISTS) {
    const int most = (K + 63) / 64;
    for (int i = 0; i < most; ++i) key[wave][i * 64 + lane] = mine[i < PER ? i : 0];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      a[i] = mine[i] == 0x7fffffff && a[i] == -INFINITY ? -INFINITY : a[i] - top;   // (NaN where the largest is no number)
      sum += a[i] == -INFINITY ? 0.f : expf(a[i]);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    const float log_sum = logf(sum);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    int listed = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i >= most) break;
      const int k = i * 64 + lane;
      int rank = 0;
      for (int j = 0; j < most * 64; ++j) rank += key[wave][j] < mine[i] || (key[wave][j] == mine[i] && j < k) ? 1 : 0;
      sorted[wave][rank] = mine[i];      // (ranks are 0 .. 64 most - 1, each once)
      if (mine[i] != 0x7fffffff) {
        id_out[t * K + rank] = mine[i];
        p_out[t * K + rank] = make_float2(expf(a[i]) / sum, a[i] - log_sum);
        ++listed;
      }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) listed += __shfl_xor(listed, off, 64);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int64_t g = lane; g <= granules; g += 64) {
      const int64_t row = g << gran_log2;
      int lo = 0, hi = listed;
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (sorted[wave][mid] < row) lo = mid + 1;
        else hi = mid;
      }
      start[t * (granules + 1) + g] = static_cast<uint16_t>(lo);
    }
  }
}

// the logits at a teacher's ids, of logits over tau
struct TeacherLogits {
  const int32_t *id;
  const uint16_t *start;
  float *z;
  int64_t granules;
  float inv;
  int32_t K;
  template <int FN>
  struct Held {
    int from[FN], to[FN];
  };
  static constexpr bool kFactor = true;
  __device__ __forceinline__ float factor() const { return inv; }
  template <int FM, int FN>
  __device__ __forceinline__ Held<FN> hold(int64_t m0, int64_t n0, int64_t T) const {
    Held<FN> h;
    const int64_t g = m0 / (FM * 16);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t t = n0 + 16 * j + (threadIdx.x & 15);
      h.from[j] = t < T ? start[t * (granules + 1) + g] : 0;
      h.to[j] = t < T ? start[t * (granules + 1) + g + 1] : 0;
    }
    return h;
  }
  template <int FM, int FN>
  __device__ __forceinline__ void take(const f32x4 (&acc)[FM][FN], const Held<FN> &held, int j, int64_t t, int64_t m0, int q) const {
    for (int s = held.from[j]; __ballot(s < held.to[j]) != 0; ++s) {
      if (s < held.to[j]) {
        const int y = id[t * K + s] - static_cast<int>(m0) - 4 * q;
        if (y >= 0 && (y & 12) == 0) {
          float v = 0.f;
#pragma unroll
          for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) v = y == 16 * i + e ? acc[i][j][e] : v;
          z[t * K + s] = v;
        }
      }
    }
  }
};

struct TeacherArgs {
  const int32_t *mark, *id;
  const float2 *p;
  const float *z;
  const uint16_t *start;
  int32_t K;
};

// a token's loss from its slots: the threads' parts of it
template <int THREADS>
__device__ __forceinline__ float slots_loss(const TeacherArgs &a, int64_t t, int listed, float base, float log_sum) {
  float part = 0.f;
  for (int s = threadIdx.x % THREADS; s < listed; s += THREADS) {
    const float2 p = a.p[t * a.K + s];
    if (p.x != 0.f) part += p.x * (p.y - ((a.z[t * a.K + s] - base) - log_sum));
  }
  return part;
}
__device__ __forceinline__ int slots_listed(const TeacherArgs &a, int64_t t, int64_t granules) { return a.start[t * (granules + 1) + granules]; }

// loss and lse of a token: one wave each, or (WAVES > 1) a block each
template <int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kBlock : WAVES * 64) void teacher_loss_kernel(const RowArgs a, const TeacherArgs b) {
  __shared__ float red[3][16];
  constexpr int TOKENS = WAVES == 1 ? kBlock / 64 : 1;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * TOKENS + (WAVES == 1 ? threadIdx.x >> 6 : 0);
  if (t >= a.T) return;
  float base, sum;
  join_granules<WAVES>(a.stat + t * a.granules, a.granules, red, base, sum);
  const float loss = rows_sum<WAVES>(slots_loss<WAVES * 64>(b, t, slots_listed(b, t, a.granules), base, logf(sum)), red[2]);
  if (threadIdx.x % (WAVES * 64) == 0) {
    a.lse[t] = base + logf(sum);
    a.loss[t] = b.mark[t] < 0 ? 0.f : (b.mark[t] == 0 ? loss : __uint_as_float(0x7fc00000u));
  }
}

// The same, one block a token, and the row's numerators turned into g (turn_row): weight q first, then weight (q - p) at the teacher's ids, from the
// logits as they are; ids that a teacher names twice by the first of them.
template <typename IO>
__global__ __launch_bounds__(kBlock) void teacher_row_kernel(const RowArgs a, const TeacherArgs b) {
  __shared__ float red[3][16];
  const int64_t t = blockIdx.x;
  const float2 *stat = a.stat + t * a.granules;
  float base, sum;
  join_granules<kBlock / 64>(stat, a.granules, red, base, sum);
  const int listed = slots_listed(b, t, a.granules), mark = b.mark[t];
  const float loss = rows_sum<kBlock / 64>(slots_loss<kBlock>(b, t, listed, base, logf(sum)), red[2]);
  const float bad = __uint_as_float(0x7fc00000u);
  if (threadIdx.x == 0) {
    a.lse[t] = base + logf(sum);
    a.loss[t] = mark < 0 ? 0.f : (mark == 0 ? loss : bad);
  }
  const float given = weight_over_common(a, b.mark, t, mark);
  const bool counts = given != 0.f;
  const float weight = mark == 1 ? bad : given;
  turn_row<IO>(a, t, stat, base, weight / sum, counts, [](int64_t, float (&)[8]) {});
  __syncthreads();
  if (!counts) return;
  for (int s = threadIdx.x; s < listed; s += kBlock) {
    const int32_t *id = b.id + t * b.K;
    if (s > 0 && id[s - 1] == id[s]) continue;
    float p = 0.f;
    for (int i = s; i < listed && id[i] == id[s]; ++i) p += b.p[t * b.K + i].x;
    const float g = weight * (expf(b.z[t * b.K + s] - base) / sum - p);
    const int64_t at = t * a.ld + id[s];
    if constexpr (IO::kVec == 8) reinterpret_cast<uint16_t *>(a.E)[at] = f32_to_bf16(g);
    else reinterpret_cast<float *>(a.E)[at] = g;
  }
}

// what of run_head is the teacher's
template <typename ID>
struct Teacher {
  const int32_t *marks;
  const float *weight;
  float factor;             // 1 / tau
  const ID *ids;
  const float *logits;
  int64_t T;
  int32_t V, K;
  int gran_log2;
  const DistillWs &w;
  hipStream_t s;
  TeacherArgs args(int64_t t0) const { return {marks + t0, w.id, w.p, w.z, w.start, K}; }
  hipError_t before(int64_t t0, int64_t n) {
    const int64_t at = t0 * K, granules = w.head.plan.granules;
    constexpr int64_t kMostTokens = int64_t{1} << 24;      // of a launch, which has fewer than 2^32 threads
    for (int64_t t = 0; t0 == 0 && n < T && t < T; t += kMostTokens) {     // all marks, which the mean's weights need
      const int64_t some = T - t < kMostTokens ? T - t : kMostTokens;
      hipLaunchKernelGGL((teacher_kernel<ID, false>), dim3(blocks(some, kBlock / 64)), dim3(kBlock), 0, s, ids + t * K, logits + t * K, some, K, V,
                         factor, gran_log2, granules, w.mark + t, nullptr, nullptr, nullptr);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((teacher_kernel<ID, true>), dim3(blocks(n, kBlock / 64)), dim3(kBlock), 0, s, ids + at, logits + at, n, K, V, factor, gran_log2,
                       granules, w.mark + t0, w.id, w.p, w.start);
    return hipGetLastError();
  }
  hipError_t between(const RowArgs &) { return hipSuccess; }
  TeacherLogits wanted(int64_t) const { return {w.id, w.start, w.z, w.head.plan.granules, factor, K}; }
  hipError_t loss(const RowArgs &a, int64_t t0) {
    if (a.T < 1024) hipLaunchKernelGGL((teacher_loss_kernel<16>), dim3(static_cast<unsigned>(a.T)), dim3(1024), 0, s, a, args(t0));
    else hipLaunchKernelGGL((teacher_loss_kernel<1>), dim3(blocks(a.T, kBlock / 64)), dim3(kBlock), 0, s, a, args(t0));
    return hipGetLastError();
  }
  template <typename IO>
  hipError_t rows(const RowArgs &a, int64_t t0) {
    hipLaunchKernelGGL((teacher_row_kernel<IO>), dim3(static_cast<unsigned>(a.T)), dim3(kBlock), 0, s, a, args(t0));
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_distill(const mhcl_ends_desc &d, int32_t K, float temperature, const void *h, const void *W, const void *ids, const float *logits,
                          const float *weight, float *loss, float *lse, float *total, void *g_h, void *g_W, bool unrounded, const DistillWs &w,
                          hipStream_t s) {
  return dispatch_id(d.id_dtype, [&](auto id) {
    return dispatch_io(d.io_dtype, [&](auto io) {
      using ID = decltype(id);
      int gran_log2 = 0;
      while ((1 << gran_log2) < w.head.plan.logits.gran) ++gran_log2;
      Teacher<ID> way{w.mark, weight, 1.f / temperature, static_cast<const ID *>(ids), logits, d.T, d.V, K, gran_log2, w, s};
      const hipError_t e = run_head<decltype(io)>(d, h, W, way, loss, lse, g_h, g_W, unrounded, w.head, s);
      if (e != hipSuccess || !total) return e;
      mhcl_ends_desc marks = d;
      marks.id_dtype = MHCL_I32;
      return launch_head_total(marks, w.mark, loss, weight, total, s);
    });
  });
}

}  // namespace mhcl
