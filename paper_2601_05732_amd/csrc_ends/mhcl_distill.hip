// The head against a teacher's top logits, and its gradients.
//
//   p_k = exp(a_k) / sum_j exp(a_j),  a = teacher's logits / tau        over a token's slots that hold one
//   z   = h W^T / tau                                                   [T, V]  never in memory
//   loss = sum_k p_k (log p_k - log q[id_k]),  q = softmax(z)
//   g = weight (q - p) / tau,  g_h = g W,  g_W = g^T h
//
// The cross entropy's products and passes (mhcl_head_rows.h) with K logits of a token in place of one: they are put in order of
// their ids first, and a table says of each granule (the rows of a wave of the first product) which of them lie in it, so that the wave takes
// them from its sums.  (A product of h with the K rows instead would read K C numbers a token again.)
#include <string.h>

#include "mhcl_head_rows.h"

namespace mhcl {
namespace {

// What a granule holds of a token's slots in order: the first one, how many, and the first one's row in the granule
__device__ __forceinline__ uint32_t slots_word(int first, int count, int row) { return row << 18 | count << 9 | first; }
static_assert(kMostSlots < 512 && kTileBig.gran <= 1 << 14, "slots_word");

// 16384 tokens, 64 slots, 512 granules 24 us, 33 MB of table and 16 of lists; 333, 8, 32 4.5.
// A token's slots, by a wave: a slot is empty where its id is negative or its logit is the lowest there is (-infinity).  LISTS: else the mark alone.
template <typename ID, bool LISTS>
__global__ __launch_bounds__(kBlock) void teacher_kernel(const ID *__restrict__ ids, const float *__restrict__ logits, int64_t T, int32_t K, int32_t V,
                                                         float inv, int gran_log2, int64_t granules, int32_t *__restrict__ mark,
                                                         int32_t *__restrict__ id_out, float2 *__restrict__ p_out, uint32_t *__restrict__ table,
                                                         int32_t *__restrict__ listed_out, const int32_t *__restrict__ row) {
  constexpr int WAVES = kBlock / 64, PER = kMostSlots / 64;
  __shared__ int32_t key[LISTS ? WAVES : 1][kMostSlots], sorted[LISTS ? WAVES : 1][kMostSlots];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * WAVES + wave;
  if (t >= T) return;      // (waves do not meet)
  const int64_t from = row ? row[t] : t;      // the caller's
  float a[PER], top = -INFINITY, sum = 0.f;
  int32_t mine[PER];
  int held = 0, bad = 0;
  ID given[PER];
  float value[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {      // (a load under a lane's condition would wait for the one before)
    if (i * 64 >= K) break;
    const int k = i * 64 + lane < K ? i * 64 + lane : 0;
    given[i] = ids[from * K + k];
    value[i] = logits[from * K + k];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = i * 64 + lane;
    a[i] = -INFINITY;
    mine[i] = 0x7fffffff;
    if (k < K) {
      const int64_t id = static_cast<int64_t>(given[i]);
      const float v = value[i];
      const bool there = id >= 0 && !(v == -INFINITY);
      if (there) a[i] = v;
      if (there && id < V) mine[i] = static_cast<int32_t>(id);
      held += there ? 1 : 0;
      bad += there && (id >= V || !(v < INFINITY)) ? 1 : 0;      // (or NaN)
    }
    top = fmaxf(top, a[i]);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    top = fmaxf(top, __shfl_xor(top, off, 64));
    held += __shfl_xor(held, off, 64);
    bad += __shfl_xor(bad, off, 64);
  }
  if (lane == 0) mark[from] = held == 0 ? -1 : (bad != 0 ? 1 : 0);
  if constexpr (LISTS) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i * 64 < K) key[wave][i * 64 + lane] = mine[i];
      a[i] = mine[i] == 0x7fffffff && a[i] == -INFINITY ? -INFINITY : (a[i] - top) * inv;   // (NaN where the largest is no number)
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
      if (i * 64 >= K) break;
      const int k = i * 64 + lane;
      int rank = 0;
      for (int j = 0; j < K; ++j) rank += key[wave][j] < mine[i] || (key[wave][j] == mine[i] && j < k) ? 1 : 0;
      if (mine[i] != 0x7fffffff) {       // (the ranks of those are 0 .. listed - 1, each once)
        sorted[wave][rank] = mine[i];
        id_out[t * K + rank] = mine[i];
        p_out[t * K + rank] = make_float2(expf(a[i]) / sum, a[i] - log_sum);
        ++listed;
      }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) listed += __shfl_xor(listed, off, 64);
    if (lane == 0) listed_out[t] = listed;
    uint32_t *words = table + t * granules;
    for (int64_t g = lane; g < granules; g += 64) words[g] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // the first slot of a granule writes its word, after the zeros of the same wave
    for (int s = lane; s < listed; s += 64) {
      const int32_t id = sorted[wave][s], g = id >> gran_log2;
      if (s > 0 && sorted[wave][s - 1] >> gran_log2 == g) continue;
      int end = s + 1;
      while (end < listed && sorted[wave][end] >> gran_log2 == g) ++end;
      words[g] = slots_word(s, end - s, id - (g << gran_log2));
    }
  }
}

// the logits at a teacher's ids, of logits over tau.  (8192 tokens, C = 768, 50257 rows, 32 slots: the table's word, and in it the row of the first
// slot, read before the tile's first step is 50 us less than first slots by a prefix sum, read with the ids after the last step; the call takes 600.)
struct TeacherLogits {
  const int32_t *id;
  const uint32_t *table;
  float *z;
  int64_t granules, K;
  int64_t inv;              // the factor's bits (a float beside the others would be put into LDS with them)
  template <int FN>
  struct Held {
    uint32_t word[FN];
  };
  static constexpr bool kFactor = true, kEarly = true;
  __device__ __forceinline__ float factor() const { return __uint_as_float(static_cast<uint32_t>(inv)); }
  template <int FM, int FN>
  __device__ __forceinline__ Held<FN> hold(int64_t m0, int64_t n0, int64_t T) const {
    Held<FN> h;
    const int64_t g = m0 / (FM * 16);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t t = n0 + 16 * j + (threadIdx.x & 15);
      h.word[j] = table[(t < T ? t : T - 1) * granules + g];
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) h.word[j] = n0 + 16 * j + (threadIdx.x & 15) < T ? h.word[j] : 0u;
    return h;
  }
  template <int FM, int FN>
  __device__ __forceinline__ void take(const f32x4 (&acc)[FM][FN], const Held<FN> &held, int j, int64_t t, int64_t m0, int q) const {
    const uint32_t word = held.word[j];
    int s = word & 511, row = word >> 18;
    const int end = s + (word >> 9 & 511);
    while (__ballot(s < end) != 0) {
      if (s < end) {
        const int y = row - 4 * q;
        if (y >= 0 && (y & 12) == 0) {
          float v = 0.f;
#pragma unroll
          for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) v = y == 16 * i + e ? acc[i][j][e] : v;
          z[t * K + s] = v;
        }
        if (++s < end) row = id[t * K + s] - static_cast<int>(m0);
      }
    }
  }
};

struct TeacherArgs {
  const int32_t *mark, *id;
  const float2 *p;
  const float *z;
  const int32_t *listed;
  int32_t K;
};

// what a slot adds to its token's loss
__device__ __forceinline__ float slot_loss(float2 p, float z, float base, float log_sum) { return p.x != 0.f ? p.x * (p.y - ((z - base) - log_sum)) : 0.f; }

// loss and lse of a token: one wave each, or (WAVES > 1) a block each
template <int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kBlock : WAVES * 64) void teacher_loss_kernel(const RowArgs a, const TeacherArgs b) {
  __shared__ float red[3][16];
  constexpr int TOKENS = WAVES == 1 ? kBlock / 64 : 1;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * TOKENS + (WAVES == 1 ? threadIdx.x >> 6 : 0);
  if (t >= a.T) return;
  float base, sum;
  join_granules<WAVES>(a.stat + t * a.granules, a.granules, red, base, sum);
  float part = 0.f;
  for (int s = threadIdx.x % (WAVES * 64); s < b.listed[t]; s += WAVES * 64) part += slot_loss(b.p[t * b.K + s], b.z[t * b.K + s], base, logf(sum));
  const float loss = rows_sum<WAVES>(part, red[2]);
  if (threadIdx.x % (WAVES * 64) == 0) {
    a.lse[t] = base + logf(sum);
    a.loss[t] = b.mark[t] < 0 ? 0.f : (b.mark[t] == 0 ? loss : __uint_as_float(0x7fc00000u));
  }
}

// The same, one block a token, and the row's numerators turned into g (turn_row): weight q first, then weight (q - p) at the teacher's ids, from the
// logits as they are; ids that a teacher names twice by the first of them.  Bound by memory: 16384 tokens, of which 15560 count, 65536 rows, bf16 950 us,
// 4.3 TB/s.
template <typename IO>
__global__ __launch_bounds__(kBlock) void teacher_row_kernel(const RowArgs a, const TeacherArgs b) {
  static_assert(kMostSlots <= kBlock, "a thread has a slot");
  __shared__ float red[3][16];
  const int64_t t = blockIdx.x;
  const int64_t u = a.token(t);
  const int s = threadIdx.x, listed = b.listed[t], mark = b.mark[u];
  // (asked for before the row's sum is known; slots behind the last are in reach)
  const int64_t slot = t * b.K + (s < b.K ? s : 0);
  const float2 mine = b.p[slot];
  const float z = b.z[slot];
  const int32_t id = b.id[slot];
  const float2 *stat = a.stat + t * a.granules;
  float base, sum;
  join_granules<kBlock / 64>(stat, a.granules, red, base, sum);
  const float log_sum = logf(sum);
  const float loss = rows_sum<kBlock / 64>(s < listed ? slot_loss(mine, z, base, log_sum) : 0.f, red[2]);
  const float bad = __uint_as_float(0x7fc00000u);
  if (threadIdx.x == 0) {
    a.lse[u] = base + log_sum;
    a.loss[u] = mark < 0 ? 0.f : (mark == 0 ? loss : bad);
  }
  if (!a.counted(t)) return;
  const float given = weight_over_common(a, b.mark, t, mark);
  const bool counts = given != 0.f;
  const float weight = mark == 1 ? bad : given;
  turn_row<IO>(a, t, stat, base, weight / sum, counts, [](int64_t, float (&)[8]) {});
  __syncthreads();
  if (!counts || s >= listed || (s > 0 && b.id[slot - 1] == id)) return;
  float p = mine.x;
  for (int i = s + 1; i < listed && b.id[t * b.K + i] == id; ++i) p += b.p[t * b.K + i].x;
  const float g = weight * (expf(z - base) / sum - p);
  const int64_t at = t * a.ld + id;
  if constexpr (IO::kVec == 8) reinterpret_cast<uint16_t *>(a.E)[at] = f32_to_bf16(g);
  else reinterpret_cast<float *>(a.E)[at] = g;
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
  TokenOrder order = {};
  static constexpr bool kLeavesOut = false;   // lse is every token's
  TeacherArgs args(int64_t t0) const { return {marks + (order.row ? 0 : t0), w.id, w.p, w.z, w.listed, K}; }
  // all marks, which the mean's weights and the order need
  hipError_t mark_all() {
    constexpr int64_t kMostTokens = int64_t{1} << 24;      // of a launch, which has fewer than 2^32 threads
    for (int64_t t = 0; t < T; t += kMostTokens) {
      const int64_t some = T - t < kMostTokens ? T - t : kMostTokens;
      hipLaunchKernelGGL((teacher_kernel<ID, false>), dim3(blocks(some, kBlock / 64)), dim3(kBlock), 0, s, ids + t * K, logits + t * K, some, K, V,
                         factor, gran_log2, w.head.plan.granules, w.mark + t, nullptr, nullptr, nullptr, nullptr, nullptr);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  hipError_t before(int64_t t0, int64_t n) {
    hipError_t e;
    if (!order.row && t0 == 0 && n < T && (e = mark_all()) != hipSuccess) return e;
    const int64_t shift = order.row ? 0 : t0;
    hipLaunchKernelGGL((teacher_kernel<ID, true>), dim3(blocks(n, kBlock / 64)), dim3(kBlock), 0, s, ids + shift * K, logits + shift * K, n, K, V, factor,
                       gran_log2, w.head.plan.granules, w.mark + shift, w.id, w.p, w.table, w.listed, order.row ? order.row + t0 : nullptr);
    return hipGetLastError();
  }
  hipError_t between(const RowArgs &) { return hipSuccess; }
  static PairLosses losses() { return {}; }
  template <bool ORDERED>
  TeacherLogits wanted(int64_t) const {
    uint32_t bits;
    memcpy(&bits, &factor, 4);
    return {w.id, w.table, w.z, w.head.plan.granules, K, bits};
  }
  hipError_t loss(const RowArgs &a, int64_t t0) {
    if (a.T < 1024 && a.granules > kWaveGranules) hipLaunchKernelGGL((teacher_loss_kernel<16>), dim3(static_cast<unsigned>(a.T)), dim3(1024), 0, s, a, args(t0));
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
      Teacher<ID> way{w.mark, weight, 1.f / temperature, static_cast<const ID *>(ids), logits, d.T, d.V, K, gran_log2, w, s, w.order};
      hipError_t e;
      if (w.ordered) {
        if ((e = way.mark_all()) != hipSuccess || (e = launch_order(way.marks, nullptr, MHCL_I64, 0, d.T, w.order, s)) != hipSuccess) return e;
        e = run_head<decltype(io), true>(d, h, W, way, loss, lse, g_h, g_W, unrounded, w.head, s);
      } else {
        e = run_head<decltype(io), false>(d, h, W, way, loss, lse, g_h, g_W, unrounded, w.head, s);
      }
      if (e != hipSuccess || !total) return e;
      mhcl_ends_desc marks = d;
      marks.id_dtype = MHCL_I32;
      return launch_head_total(marks, w.mark, loss, weight, total, s);
    });
  });
}

}  // namespace mhcl
