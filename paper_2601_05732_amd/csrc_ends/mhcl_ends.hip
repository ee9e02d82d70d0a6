// The ends of a language model, first part: token embedding into the streams with the table's gradient, and the norm of
// the streams' sum with its backward.
#include "../csrc/mhcl_common.h"
#include "mhcl_ends.h"

namespace mhcl {
namespace {

constexpr int kBlock = 256;

template <typename F>
hipError_t dispatch_id(int id_dtype, F &&f) {
  if (id_dtype == MHCL_I64) return f(int64_t{});
  return f(int32_t{});
}

// an id as 32 bits: -1 where there is no token, V where it is none of the vocabulary's
template <typename ID>
__device__ __forceinline__ int32_t token_of(const ID *ids, int64_t t, int32_t V) {
  const ID id = ids[t];
  return id < 0 ? -1 : (id >= V ? V : static_cast<int32_t>(id));
}

// VEC elements of type W (a row's piece; VEC * sizeof(W) is 8, 16 or 32 bytes) as fp32, and back
template <typename W, int VEC>
__device__ __forceinline__ void load_as(const void *p, size_t elem, float (&v)[VEC]) {
  if constexpr (W::kVec == VEC) {
    W::load(p, elem, v);
  } else if constexpr (W::kVec == 4) {   // 8 floats
    float lo[4], hi[4];
    F32::load(p, elem, lo);
    F32::load(p, elem + 4, hi);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = lo[e], v[e + 4] = hi[e];
  } else {                               // 4 bf16
    const uint2 q = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + elem);
    v[0] = bf16lo(q.x); v[1] = bf16hi(q.x); v[2] = bf16lo(q.y); v[3] = bf16hi(q.y);
  }
}
template <typename W, int VEC>
__device__ __forceinline__ void store_as(void *p, size_t elem, const float (&v)[VEC]) {
  if constexpr (W::kVec == VEC) {
    W::store(p, elem, v);
  } else if constexpr (W::kVec == 4) {
    const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
    F32::store(p, elem, lo);
    F32::store(p, elem + 4, hi);
  } else {
    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + elem) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

// sum of a token's n streams (N of them where N > 0), in order, one piece; ONCE: read past the caches
template <typename IO, int N, bool ONCE, int VEC>
__device__ __forceinline__ void stream_sum(const void *x, int64_t t, int n, int C, int c, float (&s)[VEC]) {
  if constexpr (N > 0) {
    float v[N][VEC];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (ONCE) IO::load_once(x, (t * N + i) * C + c, v[i]);
      else IO::load(x, (t * N + i) * C + c, v[i]);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      s[e] = v[0][e];
#pragma unroll
      for (int i = 1; i < N; ++i) s[e] += v[i][e];
    }
  } else {
    IO::load(x, t * n * C + c, s);
    for (int i = 1; i < n; ++i) {
      float v[VEC];
      IO::load(x, (t * n + i) * C + c, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[e] += v[e];
    }
  }
}

// ---------------------------------------------------------------- embedding
// x[t][i] = scale table[ids[t]]: one thread per 16-byte piece of a row of C, which it reads once and writes n times.
// Bound by the writes: 32768 tokens, n = 4, C = 4096, bf16 204 us, 5.3 TB/s (two tokens a thread 223; stores past the caches 210); 16384,
// C = 1024, fp32 table 33 us.
template <typename IO, typename W, typename ID>
__global__ __launch_bounds__(kBlock) void embed_kernel(const void *__restrict__ table, const ID *__restrict__ ids,
                                                       void *__restrict__ x, int n, int C, int64_t T, int32_t V, float scale) {
  constexpr int VEC = IO::kVec;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (c >= C || t >= T) return;
  const int32_t id = token_of(ids, t, V);
  float v[VEC];
  if (id >= 0 && id < V) {
    load_as<W, VEC>(table, static_cast<size_t>(id) * C + c, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] *= scale;
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = id < 0 ? 0.f : __uint_as_float(0x7fc00000u);
  }
  for (int i = 0; i < n; ++i) IO::store(x, (t * n + i) * C + c, v);
}

// Tokens by id, equal ids in the order of the tokens.  What has no place in the table (id V here) goes last.
template <typename ID>
__device__ __forceinline__ int32_t key_of(const ID *ids, int32_t t, int32_t V) {
  const ID id = ids[t];
  return id < 0 || id >= V ? V : static_cast<int32_t>(id);
}

// Zeros for the gradient's table, by the blocks of a sort's launch that have no tokens to sort: the sort takes few compute units and
// waits for memory most of its time.  (Rows that get a gradient are then written twice.  us, sort, and a launch of its own for the rows
// without a token / this: 3001 tokens, 50257 rows of 768, fp32 32.3 / 29.5; 16384, of 1024 56 / 50; 32768, 65536 rows of 4096, bf16 110 / 102.)
// A thread stores kFillEach pieces at once and its block ends.  (us of the launch, 726 MB / 154 MB / 67 MB in four launches: blocks that stay, 1024 of
// them, each with a range of its own 170 / 30.3 / 52.0, piece by piece over all 160 / 29.5 / 49.8; a block for 1 piece a thread 120 / 29.0 / 49.5,
// 4 pieces 134 / 26.8 / 49.7, 16 pieces 118 / 26.3 / 48.3.)
constexpr int kFillEach = 16;
struct Fill {
  uint4 *to;
  int64_t pieces;
  int sorting;                                         // blocks that sort; those after them fill
  __device__ __forceinline__ bool take() const {       // whether this block fills, and if so, the filling
    const int64_t b = static_cast<int64_t>(blockIdx.x) - sorting;
    if (b < 0) return false;
    const int64_t first = b * (blockDim.x * kFillEach) + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kFillEach; ++k) {
      const int64_t i = first + k * blockDim.x;
      if (i < pieces) to[i] = make_uint4(0, 0, 0, 0);
    }
    return true;
  }
};

// Few tokens, one launch: a token's place is the number of tokens with a smaller id, or the same id and an earlier place.  A block
// ranks 64 tokens, one a lane; its sixteen waves share out the tokens compared with, whose ids are wave-uniform.
constexpr int kRankWaves = 16;
template <typename ID>
__global__ __launch_bounds__(64 * kRankWaves) void rank_kernel(const ID *__restrict__ ids, int32_t *__restrict__ key,
                                                               int32_t *__restrict__ pos, int32_t *__restrict__ shared_rows, int32_t T, int32_t V,
                                                               const Fill fill) {
  __shared__ int32_t count[kRankWaves][64];
  if (fill.take()) return;
  if (blockIdx.x == 0 && threadIdx.x == 0) *shared_rows = 0;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t t0 = blockIdx.x * 64, t = t0 + lane;
  const int32_t mine = t < T ? key_of(ids, t, V) : V;
  const int32_t per = ((T + kRankWaves - 1) / kRankWaves + 63) / 64 * 64;
  const int32_t first = wave * per, last = min(T, first + per);
  int32_t smaller = 0;
  for (int32_t j0 = first; j0 < last; j0 += 64) {
    const int32_t theirs = j0 + lane < last ? key_of(ids, j0 + lane, V) : 0x7fffffff;
    const int32_t below = j0 < t0 ? mine + 1 : mine;   // equal ids count where they come before
#pragma unroll
    for (int k = 0; k < 64; ++k) smaller += __builtin_amdgcn_readlane(theirs, k) < below ? 1 : 0;
    if (j0 == t0) {
#pragma unroll
      for (int k = 0; k < 64; ++k) smaller += __builtin_amdgcn_readlane(theirs, k) == mine && k < lane ? 1 : 0;
    }
  }
  count[wave][lane] = smaller;
  __syncthreads();
  if (wave == 0 && t < T) {
    int32_t place = 0;
#pragma unroll
    for (int w = 0; w < kRankWaves; ++w) place += count[w][lane];
    key[place] = mine;
    pos[place] = t;
  }
}

// Many tokens: by digits of the id, the lowest first.  A block has a range of `per` tokens; digit_count_kernel counts its digits,
// digit_place_kernel moves its tokens behind all of smaller digits and those of the same digit in earlier blocks.  (us, the ranks
// above / two passes of digits: 4096 tokens 10.6 / 17.2, 8192 17.6 / 20.5, 16384 31.4 / 23.2; 10^6 - / 136.)
constexpr int kDigitMost = 9, kDigits = 1 << kDigitMost, kSortBlocks = 64, kSortThreads = 512, kSortTile = 2048;

struct Unsorted {   // keys and places of a pass: from the ids (the first one) or from what the pass before left
  const void *ids;
  const int32_t *key, *pos;
  template <typename ID, bool FIRST>
  __device__ __forceinline__ int32_t at(int32_t i, int32_t V) const {
    if constexpr (FIRST) return key_of(static_cast<const ID *>(ids), i, V);
    return key[i];
  }
};

template <typename ID, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void digit_count_kernel(const Unsorted in, int32_t *__restrict__ counts, int32_t *__restrict__ shared_rows,
                                                                   int32_t T, int32_t V, int32_t per, int shift, int bits, const Fill fill) {
  __shared__ int32_t count[kDigits];
  if (fill.take()) return;
  if (blockIdx.x == 0 && threadIdx.x == 0) *shared_rows = 0;
  for (int d = threadIdx.x; d < kDigits; d += kSortThreads) count[d] = 0;
  __syncthreads();
  const int32_t first = blockIdx.x * per, last = min(T, first + per);
  for (int32_t i = first + threadIdx.x; i < last; i += kSortThreads)
    atomicAdd(&count[in.at<ID, FIRST>(i, V) >> shift & ((1 << bits) - 1)], 1);   // (whole numbers: any order)
  __syncthreads();
  for (int d = threadIdx.x; d < kDigits; d += kSortThreads) counts[blockIdx.x * kDigits + d] = count[d];
}

template <typename ID, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void digit_place_kernel(const Unsorted in, const int32_t *__restrict__ counts,
                                                                   int32_t *__restrict__ key, int32_t *__restrict__ pos, int32_t T, int32_t V,
                                                                   int32_t per, int shift, int bits, const Fill fill) {
  static_assert(kDigits == kSortThreads, "a thread for each digit");
  constexpr int WAVES = kSortThreads / 64, ROUNDS = kSortTile / kSortThreads;
  __shared__ int32_t next[kDigits], count[WAVES][kDigits], sums[WAVES];
  if (fill.take()) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  {
    // where this block's tokens of digit `tid` begin
    int32_t before = 0, all = 0;
    for (int b = 0; b < fill.sorting; ++b) {
      const int32_t c = counts[b * kDigits + tid];
      before += b < static_cast<int>(blockIdx.x) ? c : 0;
      all += c;
    }
    int32_t upto = all;                                // sum over the digits up to this one
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      const int32_t v = __shfl_up(upto, off, 64);
      upto += lane >= off ? v : 0;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += sums[w];
    next[tid] = upto - all + before;
  }
  const int32_t first = blockIdx.x * per, last = min(T, first + per);
  for (int32_t tile = first; tile < last; tile += kSortTile) {
#pragma unroll
    for (int w = 0; w < WAVES; ++w) count[w][tid] = 0;
    __syncthreads();
    // a wave takes neighbouring tokens, 64 at a time: a token's place among those of its digit in the wave
    int32_t k[ROUNDS], p[ROUNDS], place[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int32_t i = tile + wave * (64 * ROUNDS) + r * 64 + lane;
      const bool there = i < last;
      k[r] = there ? in.at<ID, FIRST>(i, V) : 0;
      p[r] = there ? (FIRST ? i : in.pos[i]) : -1;
      const int digit = k[r] >> shift & ((1 << bits) - 1);
      uint64_t same = __ballot(there);
#pragma unroll
      for (int b = 0; b < kDigitMost; ++b) {
        const bool one = digit >> b & 1;
        const uint64_t ones = __ballot(one);
        same &= one ? ones : ~ones;
      }
      const int lower = __popcll(same & ((uint64_t{1} << lane) - 1));
      place[r] = there ? count[wave][digit] + lower : 0;
      __builtin_amdgcn_wave_barrier();                 // (all of a wave's lanes have read before one of them writes)
      if (there && lower == 0) count[wave][digit] += __popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    {
      int32_t begin = next[tid];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const int32_t c = count[w][tid];
        count[w][tid] = begin;
        begin += c;
      }
      next[tid] = begin;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (p[r] < 0) continue;
      const int32_t to = count[wave][k[r] >> shift & ((1 << bits) - 1)] + place[r];
      key[to] = k[r];
      pos[to] = p[r];
    }
    __syncthreads();
  }
}

// Sums of `span` sorted tokens (a chunk), TX threads for a row's columns (grid.y: the pieces of VEC TX columns), one chunk per
// threadIdx.y.  A row whose tokens all lie in the chunk is written; of a row shared with other chunks the sum goes to
// part[chunk][0] where it continues from the chunk before, else (it begins here) to part[chunk][1].
template <typename IO, typename W, bool ACC>
__device__ __forceinline__ void embed_write(void *g_table, size_t elem, const float (&sum)[IO::kVec], float scale) {
  constexpr int VEC = IO::kVec;
  float v[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) v[e] = sum[e] * scale;
  if constexpr (ACC) {
    float old[VEC];
    load_as<W, VEC>(g_table, elem, old);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] += old[e];
  }
  store_as<W, VEC>(g_table, elem, v);
}
// N: the number of streams where it is four or less, else 0; the rows of four tokens are asked for together then.  A chunk in which a
// shared row begins joins the list of those.  Bound by reading g_x: 32768 tokens, n = 4, C = 4096, bf16 227 us, 4.7 TB/s.
template <typename IO, typename W, bool ACC, int N, bool ONCE>
__global__ __launch_bounds__(kBlock) void embed_sum_kernel(const int32_t *__restrict__ key, const int32_t *__restrict__ pos,
                                                           const void *__restrict__ g_x, void *__restrict__ g_table,
                                                           float *__restrict__ part, int32_t *__restrict__ shared_rows, int span, int n,
                                                           int C, int32_t T, int32_t V, float scale) {
  constexpr int VEC = IO::kVec, GROUP = N > 0 ? 4 : 1;
  const int32_t chunk = blockIdx.x * blockDim.y + threadIdx.y;
  const int64_t s = static_cast<int64_t>(chunk) * span;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  if (s >= T || c >= C) return;
  const int64_t end = min<int64_t>(s + span, T);
  float sum[VEC] = {};
  int32_t cur = key[s];
  if (cur >= V) return;                                 // (those come last)
  bool from_before = s > 0 && key[s - 1] == cur;
  for (int64_t k = s; k < end; k += GROUP) {
    int32_t id[GROUP];
    float own[GROUP][VEC];
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      id[j] = k + j < end ? key[k + j] : V;
      // (in place of what is not summed, the chunk's first token: without a branch the loads go out together)
      stream_sum<IO, N, ONCE>(g_x, pos[id[j] < V ? k + j : s], n, C, c, own[j]);
    }
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      if (id[j] >= V) break;
      if (id[j] != cur) {
        if (from_before) store_as<F32, VEC>(part, static_cast<size_t>(chunk) * 2 * C + c, sum);
        else embed_write<IO, W, ACC>(g_table, static_cast<size_t>(cur) * C + c, sum, scale);
        cur = id[j];
        from_before = false;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += own[j][e];
    }
  }
  const bool goes_on = end < T && key[end] == cur;
  if (!from_before && !goes_on) {
    embed_write<IO, W, ACC>(g_table, static_cast<size_t>(cur) * C + c, sum, scale);
    return;
  }
  store_as<F32, VEC>(part, (static_cast<size_t>(chunk) * 2 + (from_before ? 0 : 1)) * C + c, sum);
  if (!from_before && c == 0) shared_rows[1 + atomicAdd(shared_rows, 1)] = chunk;   // (their order changes nothing)
}

// The rows that lie in several chunks, 256 columns at a time: the last row of the chunk in which it begins and the first ones of the
// chunks after it, in order; four threads of a column take a range of them each.  The blocks share out the list that the sums have left
// (a block for every chunk and 64 columns instead, most of which end at once: 32768 tokens, C = 4096 458 us, all of it launch).
constexpr int kJoinRows = 4, kJoinBlocks = 2048;
template <typename W, bool ACC>
__global__ __launch_bounds__(64 * kJoinRows) void embed_join_kernel(const int32_t *__restrict__ key, const float *__restrict__ part,
                                                                    const int32_t *__restrict__ shared_rows, void *__restrict__ g_table,
                                                                    int span, int C, int32_t T, int32_t V, float scale) {
  __shared__ float4 red[kJoinRows][64];
  const int tiles = (C + 255) / 256;
  const int64_t items = static_cast<int64_t>(*shared_rows) * tiles;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t chunk = shared_rows[1 + item / tiles];
    const int c = static_cast<int>(item % tiles) * 256 + threadIdx.x * 4;
    const int64_t e = (chunk + 1) * span;
    const int32_t id = key[e - 1];
    // its last chunk: the one of the last token with this id
    int64_t lo = e, hi = T;                                               // key[lo] == id, key[hi] > id
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) / 2;
      if (key[mid] == id) lo = mid;
      else hi = mid;
    }
    const int64_t parts = lo / span - chunk;                            // after this chunk's
    const int64_t per = (parts + kJoinRows - 1) / kJoinRows;
    const int64_t k0 = threadIdx.y * per, k1 = min(parts, k0 + per);
    float sum[4] = {};
    if (c < C) {
      if (threadIdx.y == 0) F32::load(part, (chunk * 2 + 1) * C + c, sum);
#pragma unroll 8
      for (int64_t k = k0; k < k1; ++k) {
        float v[4];
        F32::load(part, (chunk + 1 + k) * 2 * C + c, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += v[i];
      }
    }
    red[threadIdx.y][threadIdx.x] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    if (threadIdx.y == 0 && c < C) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sum[i] = pairwise_sum<kJoinRows>([&](int k) { return reinterpret_cast<const float *>(&red[k][threadIdx.x])[i]; });
      embed_write<F32, W, ACC>(g_table, static_cast<size_t>(id) * C + c, sum, scale);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- norm of the streams' sum
// A token's row of C is held by L threads, CH pieces of 16 bytes each; a block has kTokens(L) tokens at a time.
constexpr int norm_tokens(int L) { return L >= 256 ? 1 : 256 / L; }

// sum over the L threads of a token, in each of them
template <int L>
__device__ __forceinline__ float row_sum(float v, float *red) {
  v = wave_sum(v);
  if constexpr (L > 64) {
    constexpr int waves = L / 64;
    __syncthreads();                       // (red may still be read from the sum before)
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = pairwise_sum<waves>([&](int k) { return red[k]; });
  }
  return v;
}

// h = gain s / sqrt(mean(s^2) + eps), s the sum of a token's streams in fp32; one pass, bound by memory: 32768 tokens, n = 4, C = 4096,
// bf16 219 us, 6.1 TB/s.  Streams that the last-level cache cannot hold are read past the caches (kept: 248).
template <typename IO, int N, int L, int CH, bool ONCE>
__global__ __launch_bounds__(L *norm_tokens(L)) void norm_kernel(const void *__restrict__ x, const float *__restrict__ gain,
                                                                 void *__restrict__ h, int n, int C, int64_t T, float eps) {
  constexpr int VEC = IO::kVec;
  __shared__ float red[16];
  const int lane = threadIdx.x % L;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * norm_tokens(L) + threadIdx.x / L;
  if (t >= T) return;                      // (whole waves; with more than a wave a token the block has one token)
  float s[CH][VEC], sq = 0.f;
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = (k * L + lane) * VEC;
    if (c < C) {
      stream_sum<IO, N, ONCE>(x, t, n, C, c, s[k]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) sq = fmaf(s[k][e], s[k][e], sq);
    }
  }
  const float r = rms_factor(row_sum<L>(sq, red), C, eps);
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = (k * L + lane) * VEC;
    if (c < C) {
      float g[VEC];
      load_as<F32, VEC>(gain, c, g);
#pragma unroll
      for (int e = 0; e < VEC; ++e) g[e] *= s[k][e] * r;
      IO::store(h, t * C + c, g);
    }
  }
}

// u = s r, g = g_h gain:  g_s = r (g - u mean(g u)), written to every stream; g_gain = sum_t g_h u.  A block takes every
// gridDim-th token and keeps its part of g_gain in registers.  Bound by memory: 32768 tokens,
// n = 4, C = 4096, bf16 449 us, 5.4 TB/s.
template <typename IO, int N, int L, int CH>
__global__ __launch_bounds__(L *norm_tokens(L)) void norm_bwd_kernel(const void *__restrict__ x, const float *__restrict__ gain,
                                                                     const void *__restrict__ g_h, void *__restrict__ g_x,
                                                                     float *__restrict__ part, int n, int C, int64_t T, float eps) {
  constexpr int VEC = IO::kVec, TOK = norm_tokens(L);
  __shared__ float red[16];
  const int lane = threadIdx.x % L, row = threadIdx.x / L;
  float acc[CH][VEC] = {};
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * TOK + row; t < T; t += static_cast<int64_t>(gridDim.x) * TOK) {
    float s[CH][VEC], g[CH][VEC], sq = 0.f, gs = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * L + lane) * VEC;
      if (c < C) {
        stream_sum<IO, N, false>(x, t, n, C, c, s[k]);
        float w[VEC];
        IO::load(g_h, t * C + c, g[k]);
        load_as<F32, VEC>(gain, c, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          sq = fmaf(s[k][e], s[k][e], sq);
          gs = fmaf(g[k][e] * w[e], s[k][e], gs);
        }
      }
    }
    const float r = rms_factor(row_sum<L>(sq, red), C, eps);
    const float m = row_sum<L>(gs, red) / static_cast<float>(C) * r * r;   // mean(g u) r
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * L + lane) * VEC;
      if (c < C) {
        float w[VEC], o[VEC];
        load_as<F32, VEC>(gain, c, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float u = s[k][e] * r;
          acc[k][e] = fmaf(g[k][e], u, acc[k][e]);
          o[e] = r * (g[k][e] * w[e]) - u * m;
        }
        for (int i = 0; i < n; ++i) IO::store(g_x, (t * n + i) * C + c, o);
      }
    }
  }
  // the tokens of a block that share it add up, in order
  if constexpr (TOK > 1) {
    __shared__ float sums[TOK][64 * VEC];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[row][e * 64 + lane] = acc[k][e];
      __syncthreads();
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[k][e] = pairwise_sum<TOK>([&](int j) { return sums[j][e * 64 + lane]; });
    }
  }
  if (row == 0) {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * L + lane) * VEC;
      if (c < C) store_as<F32, VEC>(part, static_cast<size_t>(blockIdx.x) * C + c, acc[k]);
    }
  }
}

// g_gain[c] = the sum of its column of `part`, in order: sixteen threads of a column take a range of the rows each
__global__ __launch_bounds__(1024) void gain_sum_kernel(const float *__restrict__ part, float *__restrict__ g_gain, int rows, int C) {
  __shared__ float red[16][64];
  const int c = blockIdx.x * 64 + threadIdx.x;
  const int per = (rows + 15) / 16, k0 = threadIdx.y * per, k1 = min(rows, k0 + per);
  float sum = 0.f;
  if (c < C) {
#pragma unroll 8
    for (int k = k0; k < k1; ++k) sum += part[static_cast<size_t>(k) * C + c];
  }
  red[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.y == 0 && c < C) g_gain[c] = pairwise_sum<16>([&](int k) { return red[k][threadIdx.x]; });
}

__global__ __launch_bounds__(kBlock) void zero_kernel(uint32_t *__restrict__ p, size_t words) {
  const size_t i = static_cast<size_t>(blockIdx.x) * kBlock + threadIdx.x;
  if (i < words) p[i] = 0;
}

inline unsigned blocks(int64_t items, int64_t each) { return static_cast<unsigned>((items + each - 1) / each); }

// f(first, count) for parts of `items` in turn, until one fails: a launch has to stay below 2^32 threads in x, and has at most half as
// many here (of `threads` for each item, a power of two).
constexpr int64_t kLaunchThreads = int64_t{1} << 31;
template <typename F>
hipError_t in_launches(int64_t items, int64_t threads, F &&f) {
  const int64_t most = kLaunchThreads / threads;
  hipError_t e = hipSuccess;
  for (int64_t at = 0; at < items && e == hipSuccess; at += most) e = f(at, items - at < most ? items - at : most);
  return e;
}

// threads for a row of `pieces` pieces, and for as many rows as a block then has threads for
inline dim3 row_block(int pieces) {
  int x = 1;
  while (x < kBlock && x < pieces) x *= 2;
  return dim3(x, kBlock / x);
}

template <typename F>
hipError_t dispatch_io_w(const mhcl_ends_desc &d, F &&f) {
  return dispatch_io(d.io_dtype, [&](auto io) {
    return dispatch_io(d.w_dtype, [&](auto w) { return f(io, w); });
  });
}

// L, CH of a row of `pieces` 16-byte pieces: few threads where a row is short, so that a block has several tokens; no more
// than two pieces a thread while the block can grow
template <typename F>
hipError_t dispatch_row(int pieces, F &&f) {
  const auto go = [&](auto l, auto ch) { return f(l, ch); };
  if (pieces <= 64) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  if (pieces <= 128) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
  if (pieces <= 256) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  if (pieces <= 512) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
  if (pieces <= 1024) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  if (pieces <= 2048) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 8>{});
}
// number of streams: known to the kernel up to four
template <typename F>
hipError_t dispatch_streams(int n, F &&f) {
  switch (n) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
  }
  return f(std::integral_constant<int, 0>{});
}

}  // namespace

// About a thousand chunks, for the chip, of 8 to 32 tokens: shorter ones leave more rows to be joined.  (us, sums and joins at 8 / 16 / 32, n = 4:
// 3001 tokens, C = 768, fp32 18.6 / 23.1 / 37.5; bf16 8000, 4096 69.6 / 64.7 / 70.9; 16384, 1024 40.7 / 41.7 / 51.7; 16384, 4096 141 / 131 / 125; 32768,
// 1024 72.5 / 65.6 / 71.5; 32768, 4096 284 / 262 / 246; 65536, 1024 144 / 128 / 119.  The rule knows the tokens alone; short rows have fewer threads
// at work and would take shorter chunks: 16384, 256 21.0 / 28.0 / 43.5, 32768, 256 31.0 / 30.3 / 46.2.)
int32_t EmbedBwdWs::embed_chunk(const mhcl_ends_desc &d) { return d.T < 16384 ? 8 : (d.T < 32768 ? 16 : 32); }

hipError_t launch_zero(void *p, size_t bytes, hipStream_t s) {
  return in_launches(static_cast<int64_t>(bytes / 4), 1, [&](int64_t at, int64_t words) {
    hipLaunchKernelGGL(zero_kernel, dim3(blocks(words, kBlock)), dim3(kBlock), 0, s, static_cast<uint32_t *>(p) + at, static_cast<size_t>(words));
    return hipGetLastError();
  });
}

hipError_t launch_embed(const mhcl_ends_desc &d, const void *table, const void *ids, void *x, hipStream_t s) {
  return dispatch_io_w(d, [&](auto io, auto w) {
    return dispatch_id(d.id_dtype, [&](auto id) {
      using IO = decltype(io);
      using ID = decltype(id);
      const dim3 block = row_block(d.C / IO::kVec);
      return in_launches(d.T, block.x, [&](int64_t t0, int64_t T) {
        hipLaunchKernelGGL((embed_kernel<IO, decltype(w), ID>), dim3(blocks(T, block.y), blocks(d.C / IO::kVec, block.x)), block, 0, s, table,
                           static_cast<const ID *>(ids) + t0, static_cast<char *>(x) + t0 * d.n * d.C * (16 / IO::kVec), d.n, d.C, T, d.V, d.scale);
        return hipGetLastError();
      });
    });
  });
}

// Gradients above the size of the L2s are read past them (us of the sums, kept / past them, n = 4, C = 1024, bf16: 17 MB 9.8 / 11.8,
// 34 MB 15.6 / 14.0, 67 MB 27.0 / 18.4, 134 MB 54.6 / 36.1; C = 4096, 1.07 GB 293 / 242).
constexpr int64_t kOnceBytes = int64_t{32} << 20;

// up to so many tokens by comparing each with each
constexpr int32_t kRankTokens = 8192;

// sorts the tokens and, if `zero` is there, fills it
static hipError_t sort_tokens(const mhcl_ends_desc &d, const void *ids, const EmbedBwdWs &w, void *zero, hipStream_t s) {
  const int32_t T = static_cast<int32_t>(d.T);
  const int64_t pieces = zero ? static_cast<int64_t>(d.V) * (static_cast<int64_t>(d.C) * dtype_bytes(d.w_dtype) / 16) : 0;
  // the part-th of `parts` parts of the filling, after `sorting` blocks
  const auto fill = [&](int part, int parts, unsigned sorting) {
    const int64_t from = pieces * part / parts, to = pieces * (part + 1) / parts;
    return Fill{static_cast<uint4 *>(zero) + from, to - from, static_cast<int>(sorting)};
  };
  const auto with = [](const Fill &f, int threads) { return dim3(f.sorting + blocks(f.pieces, threads * kFillEach)); };
  return dispatch_id(d.id_dtype, [&](auto id) {
    using ID = decltype(id);
    if (T <= kRankTokens) {
      const Fill f = fill(0, 1, blocks(T, 64));
      hipLaunchKernelGGL((rank_kernel<ID>), with(f, 64 * kRankWaves), dim3(64 * kRankWaves), 0, s, static_cast<const ID *>(ids), w.key,
                         w.pos, w.shared_rows, T, d.V, f);
      return hipGetLastError();
    }
    int bits = 1;
    while (d.V >> bits) ++bits;                          // ids are 0 .. V
    const int passes = (bits + kDigitMost - 1) / kDigitMost, each = (bits + passes - 1) / passes;
    const int32_t per = static_cast<int32_t>((T + int64_t{kSortBlocks} * kSortTile - 1) / (int64_t{kSortBlocks} * kSortTile) * kSortTile);
    const unsigned sorting = blocks(T, per);
    const dim3 block(kSortThreads);
    for (int p = 0; p < passes; ++p) {
      // the last pass leaves its result in key and pos, the ones before by turns there and in the other two
      const bool home = (passes - 1 - p) % 2 == 0;
      int32_t *key = home ? w.key : w.key2, *pos = home ? w.pos : w.pos2;
      const Unsorted in{ids, home ? w.key2 : w.key, home ? w.pos2 : w.pos};
      const auto pass = [&](auto first) {
        constexpr bool FIRST = decltype(first)::value;
        const Fill count = fill(2 * p, 2 * passes, sorting), place = fill(2 * p + 1, 2 * passes, sorting);
        hipLaunchKernelGGL((digit_count_kernel<ID, FIRST>), with(count, kSortThreads), block, 0, s, in, w.counts, w.shared_rows, T, d.V, per,
                           p * each, each, count);
        hipLaunchKernelGGL((digit_place_kernel<ID, FIRST>), with(place, kSortThreads), block, 0, s, in, w.counts, key, pos, T, d.V, per,
                           p * each, each, place);
      };
      if (p == 0) pass(std::true_type{});
      else pass(std::false_type{});
    }
    return hipGetLastError();
  });
}

hipError_t launch_embed_bwd(const mhcl_ends_desc &d, const void *ids, const void *g_x, void *g_table, bool accumulate,
                            const EmbedBwdWs &w, hipStream_t s) {
  const int32_t T = static_cast<int32_t>(d.T);
  const hipError_t e = sort_tokens(d, ids, w, accumulate ? nullptr : g_table, s);
  if (e != hipSuccess) return e;
  const unsigned chunks = static_cast<unsigned>(w.chunks);
  return dispatch_io_w(d, [&](auto io, auto wt) {
    using IO = decltype(io);
    using W = decltype(wt);
    const int pieces = d.C / IO::kVec;
    const dim3 block = row_block(pieces);
    const auto go = [&](auto acc) {
      constexpr bool ACC = decltype(acc)::value;
      return dispatch_streams(d.n, [&](auto nn) {
        constexpr int N = decltype(nn)::value;
        const bool once = d.T * d.n * d.C * static_cast<int64_t>(dtype_bytes(d.io_dtype)) > kOnceBytes;
        hipLaunchKernelGGL((once ? embed_sum_kernel<IO, W, ACC, N, true> : embed_sum_kernel<IO, W, ACC, N, false>), dim3(blocks(chunks, block.y), blocks(pieces, block.x)),
                           block, 0, s, w.key, w.pos, g_x, g_table, w.part, w.shared_rows, w.chunk, d.n, d.C, T, d.V, d.scale);
        const int64_t most = static_cast<int64_t>(chunks) * blocks(d.C, 256);
        hipLaunchKernelGGL((embed_join_kernel<W, ACC>), dim3(most < kJoinBlocks ? static_cast<unsigned>(most) : kJoinBlocks),
                           dim3(64, kJoinRows), 0, s, w.key, w.part, w.shared_rows, g_table, w.chunk, d.C, T, d.V, d.scale);
        return hipGetLastError();
      });
    };
    return accumulate ? go(std::true_type{}) : go(std::false_type{});
  });
}

hipError_t launch_streams_norm(const mhcl_ends_desc &d, const void *x, const float *gain, void *h, hipStream_t s) {
  return dispatch_io(d.io_dtype, [&](auto io) {
    using IO = decltype(io);
    return dispatch_row(d.C / IO::kVec, [&](auto l, auto ch) {
      return dispatch_streams(d.n, [&](auto nn) {
        constexpr int L = decltype(l)::value, CH = decltype(ch)::value, N = decltype(nn)::value;
        constexpr int ES = 16 / IO::kVec;
        const bool once = d.T * d.n * d.C * ES > kLastLevelCache;
        return in_launches(d.T, L, [&](int64_t t0, int64_t T) {
          hipLaunchKernelGGL((once ? norm_kernel<IO, N, L, CH, true> : norm_kernel<IO, N, L, CH, false>), dim3(blocks(T, norm_tokens(L))),
                             dim3(L * norm_tokens(L)), 0, s, static_cast<const char *>(x) + t0 * d.n * d.C * ES, gain,
                             static_cast<char *>(h) + t0 * d.C * ES, d.n, d.C, T, d.eps);
          return hipGetLastError();
        });
      });
    });
  });
}

hipError_t launch_streams_norm_bwd(const mhcl_ends_desc &d, const void *x, const float *gain, const void *g_h, void *g_x,
                                   float *g_gain, float *part, hipStream_t s) {
  return dispatch_io(d.io_dtype, [&](auto io) {
    using IO = decltype(io);
    return dispatch_row(d.C / IO::kVec, [&](auto l, auto ch) {
      return dispatch_streams(d.n, [&](auto nn) {
        constexpr int L = decltype(l)::value;
        const unsigned want = blocks(d.T, norm_tokens(L)), grid = want < kNormBwdBlocks ? want : kNormBwdBlocks;
        hipLaunchKernelGGL((norm_bwd_kernel<IO, decltype(nn)::value, L, decltype(ch)::value>), dim3(grid),
                           dim3(L * norm_tokens(L)), 0, s, x, gain, g_h, g_x, part, d.n, d.C, d.T, d.eps);
        hipLaunchKernelGGL(gain_sum_kernel, dim3(blocks(d.C, 64)), dim3(64, 16), 0, s, part, g_gain, static_cast<int>(grid), d.C);
        return hipGetLastError();
      });
    });
  });
}

}  // namespace mhcl
