// The gated feed-forward block and its gradients.
//
//   G = x Wg^T, U = x Wu^T          [T, H] each, Wg and Wu the halves of W_up [2 H, C]
//   a = silu(G) U,  silu(G) = G s,  s = 1 / (1 + exp(-G))
//   y = a Wd^T                      [T, C], Wd = W_down [C, H]
//
//   g_a = g_y Wd                    [T, H]  never in memory
//   g_U = g_a silu(G),  g_G = g_a U s (1 + G (1 - s))
//   g_x = [g_G g_U] W_up,  g_W_up = [g_G g_U]^T x,  g_W_down = g_y^T a
//
// Three products of 2 T C H operations forward, six backward.  The first one takes a row of Wg and the row of Wu that goes with it in
// one lane's sums, so that its epilogue has G and U in fp32 and leaves a; that of g_a reads G and U and leaves g_G, g_U and a again.
#include "../csrc_ends/mhcl_product.h"
#include "mhcl_ffn.h"

namespace mhcl {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + exp(-x)): by the instructions for bf16 operands, to 1.25 * 2^-22 + 1.22 * 2^-24 |x| of itself, the library's for fp32 ones.  (An ulp, 2^-23, each
// for the exponential and the reciprocal, half a one for the sum; in the exponent the product's 2^-24 and the constant's 2^-26.2 of |x|.)
template <bool WIDE>
__device__ __forceinline__ float sigmoid(float x) {
  if constexpr (WIDE) return 1.f / (1.f + expf(-x));
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x));
}

// Four numbers of a lane (r, q) at 16 i + 4 q and four at 16 (i + 1) + 4 q of row n of a matrix [rows][ld], rounded to its type: an exchange makes
// one 16-byte piece of bf16 ones
template <bool WIDE>
__device__ __forceinline__ void store_two(void *p, int64_t row, int64_t m, int q, const f32x4 &u, const f32x4 &v, bool here, int64_t end) {
  if constexpr (WIDE) {
    float *o = static_cast<float *>(p) + row + m + 4 * q;
    if (here && m + 4 * q < end) *reinterpret_cast<f32x4 *>(o) = u;
    if (here && m + 16 + 4 * q < end) *reinterpret_cast<f32x4 *>(o + 16) = v;
  } else {
    const uint4 eight = join_pairs(make_uint2(pack_bf16x2(u[0], u[1]), pack_bf16x2(u[2], u[3])),
                                   make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])));
    const int64_t at = m + 16 * (q & 1) + 8 * (q >> 1);
    if (here && at < end) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + row + at) = eight;
  }
}
template <bool WIDE>
__device__ __forceinline__ void store_one(void *p, int64_t row, int64_t m, int q, const f32x4 &u, bool here, int64_t end) {
  if (!here || m + 4 * q >= end) return;
  if constexpr (WIDE) *reinterpret_cast<f32x4 *>(static_cast<float *>(p) + row + m + 4 * q) = u;
  else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + row + m + 4 * q) = make_uint2(pack_bf16x2(u[0], u[1]), pack_bf16x2(u[2], u[3]));
}
__device__ __forceinline__ f32x4 load_four(const float *p, bool here) { return here ? *reinterpret_cast<const f32x4 *>(p) : f32x4{0.f, 0.f, 0.f, 0.f}; }

// m: pairs of rows of W_up, n: tokens.  a is formed of the sums and rounded once; KEEP: G and U for the backward, in fp32: rounded to bf16 they
// would put their error into every gradient besides that of the rounded g_G, g_U and a (off from 64 bits by 0.0034 of the 2-norm then, 0.0024 so).
// 16384 rows, C = 4096, H = 8192, with them 1883 us, 1.17 PFLOP/s: matrix units and their clock, and 1.3 GB of stores.
template <bool KEEP, bool WIDE>
struct GateEpilogue {
  static constexpr bool kWide = WIDE, kPaired = true, kEarly = false, kCounted = false;
  void *a;
  float *pre;
  int64_t H, T;
  template <int FM, int FN>
  __device__ __forceinline__ int hold(int64_t, int64_t) const { return 0; }
  template <int FM, int FN>
  static constexpr int stores() { return FN * ((WIDE || FM < 4 ? FM / 2 : FM / 4) + (KEEP ? FM : 0)); }
  __device__ __forceinline__ bool whole(int64_t m_end, int64_t n_end) const { return m_end / 2 <= H && n_end <= T; }
  template <int FM, int FN>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[FM][FN], int, int64_t m0, int64_t n0, int) const {
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    constexpr int HM = FM / 2;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t n = n0 + 16 * j + r;
      const bool here = n < T;
      f32x4 v[HM];
#pragma unroll
      for (int i = 0; i < HM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = acc[i][j][e] * sigmoid<WIDE>(acc[i][j][e]) * acc[HM + i][j][e];
#pragma unroll
      for (int i = 0; i < HM; i += 2) {
        const int64_t m = m0 / 2 + 16 * i;
        if constexpr (HM > 1) store_two<WIDE>(a, n * H, m, q, v[i], v[i + 1], here, H);
        else store_one<WIDE>(a, n * H, m, q, v[i], here, H);
      }
      if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < HM; ++i) {
          store_one<true>(pre, n * 2 * H, m0 / 2 + 16 * i, q, acc[i][j], here, H);
          store_one<true>(pre, n * 2 * H + H, m0 / 2 + 16 * i, q, acc[HM + i][j], here, H);
        }
      }
    }
  }
};

// m: H, n: tokens.  The sums are g_a; g_G, g_U and a of them and of G and U, each rounded once.  16384 rows, C = 4096, H = 8192 1220 us, 0.90 PFLOP/s;
// without the reads 1010, without the stores 998: 1.9 GB at the memory's rate between the main loops of 830 us in all.  (Reads two or three fragments ahead
// 1214 and 1228; half of the blocks half a tile later 1249; tiles of 128 x 128, two to a unit, 1366.)
// ACT: a too, which g_W_down alone reads (without it 1167 us where a trace has 1222 with it).
template <bool WIDE, bool ACT>
struct GateGradEpilogue {
  static constexpr bool kWide = WIDE, kPaired = false, kEarly = false, kCounted = false;
  const float *pre;
  void *a, *g_pre;
  int64_t H, T;
  template <int FM, int FN>
  __device__ __forceinline__ int hold(int64_t, int64_t) const { return 0; }
  template <int FM, int FN>
  static constexpr int stores() { return FN * (WIDE ? FM : FM / 2) * (ACT ? 3 : 2); }
  __device__ __forceinline__ bool whole(int64_t m_end, int64_t n_end) const { return m_end <= H && n_end <= T; }
  template <int FM, int FN>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[FM][FN], int, int64_t m0, int64_t n0, int) const {
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t n = n0 + 16 * j + r, row = n * 2 * H;
      const bool here = n < T;
#pragma unroll
      for (int i = 0; i < FM; i += 2) {
        const int64_t m = m0 + 16 * i;
        f32x4 G[2], U[2], v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bool there = here && m + 16 * k + 4 * q < H;
          G[k] = load_four(pre + row + m + 16 * k + 4 * q, there);
          U[k] = load_four(pre + row + H + m + 16 * k + 4 * q, there);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float g = G[k][e], u = U[k][e], ga = acc[i + k][j][e], s = sigmoid<WIDE>(g), silu = g * s;
            v[k][e] = silu * u;
            G[k][e] = ga * u * (s * (1.f + g * (1.f - s)));
            U[k][e] = ga * silu;
          }
        if constexpr (ACT) store_two<WIDE>(a, n * H, m, q, v[0], v[1], here, H);
        store_two<WIDE>(g_pre, row, m, q, G[0], G[1], here, H);
        store_two<WIDE>(g_pre, row + H, m, q, U[0], U[1], here, H);
      }
    }
  }
};

// a of G and U, where nothing but g_W_down is asked for: blocks take rows in turn.  Bound by memory: 16384 rows,
// H = 8192, bf16 240 us, 5.6 TB/s.
template <typename IO>
__global__ __launch_bounds__(kBlock) void gate_kernel(const float *__restrict__ pre, void *__restrict__ a, int64_t T, int64_t H) {
  constexpr bool WIDE = IO::kVec == 4;
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x)
    for (int64_t m = threadIdx.x * 4; m < H; m += kBlock * 4) {
      const f32x4 G = load_four(pre + t * 2 * H + m, true), U = load_four(pre + t * 2 * H + H + m, true);
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = G[e] * sigmoid<WIDE>(G[e]) * U[e];
      store_one<WIDE>(a, t * H + m, 0, 0, v, true, H);
    }
}

// ---------------------------------------------------------------- few rows
// y = W x for up to 64 rows of x, as in a step of decoding: W is read once, straight into the fragments of its 16 rows a block, and the waves
// of the block share the depth, each a run of steps of 32; their sums meet in LDS, in order.  Nothing else is shared, so that no wave waits for another
// until then.  GATE: 16 rows of Wg and the 16 of Wu that go with them; out is silu(G) U, and pre, if it is there, G and U.
// Bound by what a block reads, its rows of W and all of x: 16 rows of x, C = H = 2048, bf16 16.4 us for both products (tiles, their parts and the sum
// over those 18.0), fp32 23.2 (49.5); 32, C = 1024, H = 4096 20.6 (15.3) and 34.7 (33.3); 64, C = 520, H = 1000 10.9 (13.3) and 16.0 (24.2).
// (Other orders of the steps for each block and wave, so that rows a power of two apart do not meet in one channel: no faster.)
struct FewArgs {
  const void *W, *x;
  void *out;
  float *pre;
  int64_t M, K, T;      // GATE: M is H
};
constexpr int64_t kFewRows = 64, kOneRows = 2, kOneBytes = 64 << 10;     // rows of x; of them in one_kernel, and their bytes
// Which of the two there are for few rows, or (0) the tiles: by what a block of few_kernel reads in the second product, against tiles whose time goes
// with W's size for fp32 and hardly at all for bf16 (up to 32M weights).  One row, C = 4096, H = 8192: one_kernel 39.8 us and 77.4, tiles 49.8 and
// 128.5; two 42.6 and 81.9; four 52.2 and 91.8, where few_kernel takes 48.5 and 77.8.
enum class Few { kNone, kOne, kFew };
Few few_for(const mhcl_ffn_desc &d, bool wide) {
  if (d.T > kFewRows) return Few::kNone;
  if (d.T <= kOneRows && d.T * std::max(d.C, d.H) * (wide ? 4 : 2) <= kOneBytes) return Few::kOne;
  const int64_t reads = d.H * (16 + ceil_div(d.T, 16) * 16);
  return reads <= (wide ? 100000 + static_cast<int64_t>(d.C) * d.H / 64 : 90000) ? Few::kFew : Few::kNone;
}
template <bool WIDE>
struct FewFragment {
  u32x4 v[WIDE ? 2 : 1];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t p, uint32_t at) {
#pragma unroll
    for (int i = 0; i < (WIDE ? 2 : 1); ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b128(p, at + i * 16, 0, 0);
  }
  __device__ __forceinline__ Parts parts() const {
    return parts_of(Eight{{__builtin_bit_cast(f32x4, v[0]), __builtin_bit_cast(f32x4, v[WIDE ? 1 : 0])}});
  }
};
template <int FN, bool GATE, bool WIDE, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void few_kernel(const FewArgs a) {
  // steps whose loads are on their way together: what the registers hold (128 of a lane with sixteen waves) besides the sums and parts
  constexpr int HALVES = GATE ? 2 : 1, PARTS = WIDE ? 12 * (HALVES + 1) : 0, FIT = ((WAVES > 8 ? 104 : 128) - HALVES * FN * 4 - PARTS) / ((HALVES + FN) * (WIDE ? 8 : 4));
  constexpr int UNROLL = FIT >= 8 ? 8 : (FIT >= 4 ? 4 : (FIT >= 2 ? 2 : 1));
  __shared__ f32x4 sums[WAVES][HALVES][FN][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * 16;
  const int steps = static_cast<int>((a.K + 31) / 32), first = steps * wave / WAVES, last = steps * (wave + 1) / WAVES;
  // (loads past the depth ask for what is out of range, as rows of x that are not there do, and get zeros; rows past W's give results that nobody reads)
  constexpr int ES = WIDE ? 4 : 2;
  const auto range = [](int64_t bytes) { return static_cast<int>(bytes < 0x7fffffff ? bytes : 0x7fffffff); };
  const __amdgpu_buffer_rsrc_t in_w = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(static_cast<const char *>(a.W)) + m0 * a.K * ES, 0,
                                                                         range((HALVES * a.M - m0) * a.K * ES), 0x00020000);
  const __amdgpu_buffer_rsrc_t in_x = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(a.x), 0, range(a.T * a.K * ES), 0x00020000);
  const uint32_t row = static_cast<uint32_t>(r * a.K * ES), partner = static_cast<uint32_t>(a.M * a.K * ES), tile = static_cast<uint32_t>(16 * a.K * ES);
  f32x4 acc[HALVES][FN];
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[h][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = first; s < last; s += UNROLL) {
    FewFragment<WIDE> w[UNROLL][HALVES], x[UNROLL][FN];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int k = (s + u) * 32 + 8 * q;
      const uint32_t at = s + u < last && k < a.K ? row + k * ES : 0x80000000u;
#pragma unroll
      for (int h = 0; h < HALVES; ++h) w[u][h].load(in_w, at + h * partner);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int k = (s + u) * 32 + 8 * q;
      const uint32_t at = s + u < last && k < a.K ? row + k * ES : 0x80000000u;
#pragma unroll
      for (int j = 0; j < FN; ++j) x[u][j].load(in_x, at + j * tile);
    }
    __builtin_amdgcn_sched_barrier(0);     // (all of them before the products)
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if constexpr (WIDE) {
        constexpr int A[6] = {1, 0, 2, 0, 1, 0}, B[6] = {1, 2, 0, 1, 0, 0};
        Parts pw[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) pw[h] = w[u][h].parts();
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const Parts px = x[u][j].parts();
#pragma unroll
          for (int i = 0; i < 6; ++i)
#pragma unroll
            for (int h = 0; h < HALVES; ++h) acc[h][j] = mfma16(pw[h].p[A[i]], px.p[B[i]], acc[h][j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int h = 0; h < HALVES; ++h) acc[h][j] = mfma16(w[u][h].v[0], x[u][j].v[0], acc[h][j]);
      }
    }
  }
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int j = 0; j < FN; ++j) sums[wave][h][j][lane] = acc[h][j];
  __syncthreads();
  if (wave >= FN) return;
  f32x4 v[HALVES];
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    v[h] = sums[0][h][wave][lane];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v[h] += sums[i][h][wave][lane];
  }
  const int64_t n = 16 * wave + r;
  const bool here = n < a.T;
  if constexpr (GATE) {
    if (a.pre) {
      store_one<true>(a.pre, n * 2 * a.M, m0, q, v[0], here, a.M);
      store_one<true>(a.pre, n * 2 * a.M + a.M, m0, q, v[1], here, a.M);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[0][e] = v[0][e] * sigmoid<WIDE>(v[0][e]) * v[1][e];
  }
  store_one<WIDE>(a.out, n * a.M, m0, q, v[0], here, a.M);
}

// The same for one or two rows of x, which then lie in LDS: a wave takes ROWS rows of W (GATE: and their partners) over the whole depth, a
// kilobyte of each at a time, the next ones' loads under the products.  fp32 operands are multiplied as they are.  Bound by reading W: one row, C = 4096,
// H = 8192, bf16 22.1 and 12.6 us, 6.1 and 5.3 TB/s.
template <int TOKENS, bool GATE, bool WIDE>
__global__ __launch_bounds__(kBlock) void one_kernel(const FewArgs a) {
  constexpr int HALVES = GATE ? 2 : 1, ROWS = 2, UNROLL = 8 / HALVES, VEC = WIDE ? 4 : 8;
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  extern __shared__ u32x4 xs[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t m0 = (static_cast<int64_t>(blockIdx.x) * (kBlock / 64) + wave) * ROWS;
  const int pieces = static_cast<int>(a.K / VEC);        // of 16 bytes, of a row; loads past it get zeros
  const char *W = static_cast<const char *>(a.W);
  const auto row = [&](int i, int h) __attribute__((always_inline)) {
    const int64_t m = (m0 + i < a.M ? m0 + i : a.M - 1) + h * a.M;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(W) + m * pieces * 16, 0, pieces * 16, 0x00020000);
  };
  u32x4 next[UNROLL][ROWS][HALVES];
  const auto load = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int h = 0; h < HALVES; ++h) next[u][i][h] = __builtin_amdgcn_raw_buffer_load_b128(row(i, h), (p0 + u * 64 + lane) * 16, 0, 0);
    }
  };
  load(0);
  for (int p = threadIdx.x; p < TOKENS * pieces; p += kBlock) xs[p] = static_cast<const u32x4 *>(a.x)[p];
  float acc[ROWS][HALVES][TOKENS] = {};
  __syncthreads();
  for (int p0 = 0; p0 < pieces; p0 += UNROLL * 64) {
    u32x4 w[UNROLL][ROWS][HALVES];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int h = 0; h < HALVES; ++h) w[u][i][h] = next[u][i][h];
    load(p0 + UNROLL * 64);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int p = p0 + u * 64 + lane;
#pragma unroll
      for (int t = 0; t < TOKENS; ++t) {
        const u32x4 v = p < pieces ? xs[t * pieces + p] : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
          for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float &sum = acc[i][h][t];
              const uint32_t one = w[u][i][h][e], other = v[e];
              if constexpr (WIDE) sum = fmaf(__uint_as_float(one), __uint_as_float(other), sum);
              else sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, one), __builtin_bit_cast(bf16x2, other), sum, false);
            }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
#pragma unroll
      for (int h = 0; h < HALVES; ++h) acc[i][h][t] = wave_sum(acc[i][h][t]);
      const int64_t m = m0 + i;
      if (lane != i * TOKENS + t || m >= a.M) continue;
      float v = acc[i][0][t];
      if constexpr (GATE) {
        if (a.pre) {
          a.pre[t * 2 * a.M + m] = v;
          a.pre[t * 2 * a.M + a.M + m] = acc[i][1][t];
        }
        v = v * sigmoid<WIDE>(v) * acc[i][1][t];
      }
      if constexpr (WIDE) static_cast<float *>(a.out)[t * a.M + m] = v;
      else static_cast<uint16_t *>(a.out)[t * a.M + m] = f32_to_bf16(v);
    }
}
template <bool GATE, bool WIDE>
hipError_t launch_one(const FewArgs &a, hipStream_t s) {
  const unsigned count = blocks(a.M, 2 * (kBlock / 64)), bytes = static_cast<unsigned>(a.T * a.K * (WIDE ? 4 : 2));
  if (a.T == 1) hipLaunchKernelGGL((one_kernel<1, GATE, WIDE>), dim3(count), dim3(kBlock), bytes, s, a);
  else hipLaunchKernelGGL((one_kernel<2, GATE, WIDE>), dim3(count), dim3(kBlock), bytes, s, a);
  return hipGetLastError();
}

template <bool GATE, bool WIDE>
hipError_t launch_few(const FewArgs &a, hipStream_t s) {
  const unsigned count = blocks(a.M, 16);
  const auto go = [&](auto fn) {
    constexpr int FN = decltype(fn)::value;
    // (the waves of a unit: where it has one block, as many as it holds, which is so of all of bf16's first products: few_for takes up to 2812 rows of Wg)
    if constexpr (!GATE || WIDE) {
      if (count > kChipBlocks) {
        hipLaunchKernelGGL((few_kernel<FN, GATE, WIDE, 8>), dim3(count), dim3(512), 0, s, a);
        return hipGetLastError();
      }
    }
    hipLaunchKernelGGL((few_kernel<FN, GATE, WIDE, 16>), dim3(count), dim3(1024), 0, s, a);
    return hipGetLastError();
  };
  if (a.T <= 16) return go(std::integral_constant<int, 1>{});
  if (a.T <= 32) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}

// ---------------------------------------------------------------- the three last products of the backward in one launch
// None needs another's result; where they are small, each alone leaves units without work.  The blocks of the first product come first, then the
// second's and the third's.  us, the whole pass with three launches and
// their sums over slabs / with this: 333 rows, C = 520, H = 1000, bf16 51.0 / 37.8; 2048, 768, 2048, fp32 408 / 357.
struct TrioArgs {
  GemmArgs g[3];
  int blocks[2];        // of the first, of the first two
};
template <bool SLIM, bool WIDE>
__global__ __launch_bounds__(256, 2) void trio_kernel(const TrioArgs a, const StoreEpilogue<WIDE> to_gx, const StoreEpilogue<WIDE> to_gup,
                                                      const StoreEpilogue<WIDE> to_gdown) {
  constexpr int LEAST = SLIM ? kSharedPieces : 0;
  const int block = blockIdx.x;
  if (block < a.blocks[0])
    gemm_tiles<128, SLIM ? 32 : 128, SLIM ? 4 : 2, SLIM ? 1 : 2, SLIM ? 4 : 2, false, true, LEAST>(a.g[0], to_gx, block, a.blocks[0]);
  else if (block < a.blocks[1])
    gemm_tiles<128, 128, 2, 2, 2, false, false, LEAST>(a.g[1], to_gup, block - a.blocks[0], a.blocks[1] - a.blocks[0]);
  else
    gemm_tiles<128, 128, 2, 2, 2, false, false, LEAST>(a.g[2], to_gdown, block - a.blocks[1], gridDim.x - a.blocks[1]);
}
// the sums over slabs of up to three results in one launch
struct SlabSums {
  const float *in[3];
  void *out[3];
  int slabs[3];
  int64_t count[3], end[3];     // `end`: of its blocks
};
template <typename IO>
__global__ __launch_bounds__(kBlock) void slab_sums_kernel(const SlabSums a) {
  const int64_t block = blockIdx.x;
  const int p = block < a.end[0] ? 0 : (block < a.end[1] ? 1 : 2);
  const int64_t from = p == 0 ? 0 : a.end[p - 1], count = a.count[p], i = ((block - from) * kBlock + threadIdx.x) * 4;
  if (i >= count) return;
  const float *in = a.in[p] + i;
  f32x4 s = *reinterpret_cast<const f32x4 *>(in);
  const int slabs = a.slabs[p];
#pragma unroll 4
  for (int k = 1; k < slabs; ++k) s += *reinterpret_cast<const f32x4 *>(in + k * count);
  if constexpr (IO::kVec == 4) *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out[p]) + i) = s;
  else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out[p]) + i) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
}

// D[n][m] = sum over k, in `splits` slabs that are then joined, or at once
template <bool AK, bool BK, typename IO>
hipError_t product(const ProductTile &tile, const Operand &A, const Operand &B, int64_t M, int64_t N, int splits, float *slabs, void *out, hipStream_t s) {
  constexpr bool WIDE = IO::kVec == 4;
  const StoreEpilogue<WIDE> e{nullptr, splits > 1 ? slabs : (WIDE ? static_cast<float *>(out) : nullptr), static_cast<uint16_t *>(out), nullptr, M, N, M * N, nullptr, {}, false, nullptr};
  const hipError_t err = launch_gemm<AK, BK>(tile, A, B, M, N, splits, e, s);
  return err != hipSuccess || splits == 1 ? err : launch_slab_sum<IO>(slabs, out, splits, M * N, s);
}

template <typename IO>
hipError_t run_ffn(const mhcl_ffn_desc &d, const void *x, const void *W_up, const void *W_down, void *y, float *pre, const FfnWs &w, hipStream_t s) {
  constexpr bool WIDE = IO::kVec == 4;
  const FfnPlan &p = w.plan;
  const int64_t T = d.T, C = d.C, H = d.H;
  const Few few = few_for(d, WIDE);
  if (few != Few::kNone) {
    const FewArgs first{W_up, x, w.a, pre, H, C, T}, second{W_down, w.a, y, nullptr, C, H, T};
    const hipError_t e = few == Few::kOne ? launch_one<true, WIDE>(first, s) : launch_few<true, WIDE>(first, s);
    if (e != hipSuccess) return e;
    return few == Few::kOne ? launch_one<false, WIDE>(second, s) : launch_few<false, WIDE>(second, s);
  }
  const Operand Wu{W_up, C, 2 * H, C}, xk{x, C, T, C}, Wd{W_down, H, C, H}, ak{w.a, H, T, H};
  const hipError_t e = pre ? launch_gemm<true, true>(p.up, Wu, xk, 2 * H, T, 1, GateEpilogue<true, WIDE>{w.a, pre, H, T}, s)
                           : launch_gemm<true, true>(p.up, Wu, xk, 2 * H, T, 1, GateEpilogue<false, WIDE>{w.a, nullptr, H, T}, s);
  return e != hipSuccess ? e : product<true, true, IO>(p.down, Wd, ak, C, T, p.down_splits, w.slabs, y, s);
}

template <typename IO>
hipError_t run_ffn_grad(const mhcl_ffn_desc &d, const void *x, const void *W_up, const void *W_down, const float *pre, const void *g_y, void *g_x,
                        void *g_W_up, void *g_W_down, const FfnWs &w, hipStream_t s) {
  constexpr bool WIDE = IO::kVec == 4;
  const FfnPlan &p = w.plan;
  const int64_t T = d.T, C = d.C, H = d.H;
  const Operand Wd{W_down, H, H, C}, gk{g_y, C, T, C}, Wu{W_up, C, C, 2 * H}, pk{w.g_pre, 2 * H, T, 2 * H};
  const Operand xm{x, C, C, T}, pm{w.g_pre, 2 * H, 2 * H, T}, am{w.a, H, H, T}, gm{g_y, C, C, T};
  hipError_t e;
  if (!g_x && !g_W_up) {
    hipLaunchKernelGGL((gate_kernel<IO>), dim3(static_cast<unsigned>(std::min<int64_t>(T, 8 * kChipBlocks))), dim3(kBlock), 0, s, pre, w.a, T, H);
    e = hipGetLastError();
  } else if (g_W_down) {
    e = launch_gemm<false, true>(p.act, Wd, gk, H, T, 1, GateGradEpilogue<WIDE, true>{pre, w.a, w.g_pre, H, T}, s);
  } else {
    e = launch_gemm<false, true>(p.act, Wd, gk, H, T, 1, GateGradEpilogue<WIDE, false>{pre, nullptr, w.g_pre, H, T}, s);
  }
  if (e != hipSuccess) return e;
  void *const out[3] = {g_x, g_W_up, g_W_down};     // (as many parts of each whichever are asked for: the same bits)
  if (p.trio) {
    const auto to = [&](int splits, float *slabs, void *out, int64_t M, int64_t N) {
      return StoreEpilogue<WIDE>{nullptr, splits > 1 ? slabs : (WIDE ? static_cast<float *>(out) : nullptr), static_cast<uint16_t *>(out), nullptr, M, N, M * N, nullptr, {}, false, nullptr};
    };
    TrioArgs a{{gemm_args(p.gx, Wu, pk, C, T, p.gx_splits), gemm_args(p.gup, xm, pm, C, 2 * H, p.gup_splits), gemm_args(p.gdown, am, gm, H, C, p.gdown_splits)}, {}};
    const auto count = [&](int i) { return !out[i] ? 0 : a.g[i].tiles_m * a.g[i].tiles_n * a.g[i].splits; };
    a.blocks[0] = count(0);
    a.blocks[1] = count(0) + count(1);
    const dim3 grid(a.blocks[1] + count(2));
    const auto e0 = to(p.gx_splits, w.slabs, g_x, C, T), e1 = to(p.gup_splits, w.up_slabs, g_W_up, C, 2 * H),
               e2 = to(p.gdown_splits, w.down_slabs, g_W_down, H, C);
    if (p.gx.bn < 128) hipLaunchKernelGGL((trio_kernel<true, WIDE>), grid, dim3(256), 0, s, a, e0, e1, e2);
    else hipLaunchKernelGGL((trio_kernel<false, WIDE>), grid, dim3(256), 0, s, a, e0, e1, e2);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    SlabSums sums{{w.slabs, w.up_slabs, w.down_slabs}, {out[0], out[1], out[2]}, {p.gx_splits, p.gup_splits, p.gdown_splits}, {T * C, 2 * H * C, H * C}, {}};
    int64_t total = 0;
    for (int i = 0; i < 3; ++i) sums.end[i] = total += out[i] && sums.slabs[i] > 1 ? ceil_div(sums.count[i], kBlock * 4) : 0;
    if (total == 0) return hipSuccess;
    hipLaunchKernelGGL((slab_sums_kernel<IO>), dim3(static_cast<unsigned>(total)), dim3(kBlock), 0, s, sums);
    return hipGetLastError();
  }
  if (g_x && (e = product<false, true, IO>(p.gx, Wu, pk, C, T, p.gx_splits, w.slabs, g_x, s)) != hipSuccess) return e;
  if (g_W_up && (e = product<false, false, IO>(p.gup, xm, pm, C, 2 * H, p.gup_splits, w.slabs, g_W_up, s)) != hipSuccess) return e;
  return !g_W_down ? hipSuccess : product<false, false, IO>(p.gdown, am, gm, H, C, p.gdown_splits, w.slabs, g_W_down, s);
}

}  // namespace

FfnPlan::FfnPlan(const mhcl_ffn_desc &d, bool grad) {
  wide = d.io_dtype == MHCL_F32;
  const int64_t T = d.T, C = d.C, H = d.H, step = wide ? 32 : 64;
  up = tile_for(2 * H, T, 1, true, !wide);
  down = tile_for(C, T, std::max<int64_t>(1, ceil_div(H, step) / 8), true, !wide);
  act = tile_for(H, T, 1, true, !wide);
  gx = tile_for(C, T, std::max<int64_t>(1, ceil_div(2 * H, step) / 8), true, !wide);
  gup = tile_for(C, 2 * H, 1, false, !wide);
  gdown = tile_for(H, C, 1, false, !wide);
  down_splits = gx_splits = gup_splits = gdown_splits = 1;
  trio = false;
  if (T == 0) return;
  if (!grad) {
    down_splits = Split(down, C, T, H, wide).best();
    return;
  }
  const Split x(gx, C, T, 2 * H, wide), u(gup, C, 2 * H, T, wide), w(gdown, H, C, T, wide);
  trio = gx.bm < 256 && gup.bm < 256 && gdown.bm < 256;
  if (!trio) {
    gx_splits = x.best();
    gup_splits = u.best();
    gdown_splits = w.best();
    return;
  }
  // Parts of three products side by side (Split's model of a step): whatever is longest is split as long as the whole is expected to end sooner, which
  // is not before its longest part nor before all units have done their share.
  const Split *all[3] = {&x, &u, &w};
  int k[3] = {1, 1, 1};
  const auto slim = [&](int i) { return i == 0 && gx.bn < 128; };     // (half a step's time, a quarter of a slab's)
  const auto part = [&](int i) { return (ceil_div(all[i]->steps, k[i]) + 4) * (i == 0 && gx.bn < 128 ? 30 : 60); };
  int64_t best = INT64_MAX;
  for (;;) {
    int64_t longest = 0, work = 0, parts = 0, slabs = 0;
    int which = 0;
    for (int i = 0; i < 3; ++i) {
      const int64_t count = all[i]->tiles * k[i];
      if (part(i) > longest) longest = part(i), which = i;
      work += count * part(i);
      parts += count;
      slabs += k[i] > 1 ? count / (slim(i) ? 4 : 1) : 0;
    }
    const int64_t alone = parts <= kChipBlocks ? alone_time(wide) : 60;
    const int64_t time = std::max(longest * alone / 60, work / (2 * kChipBlocks)) + slabs + (slabs > 0 ? kSumTime : 0);
    if (time < best) {
      best = time;
      gx_splits = k[0];
      gup_splits = k[1];
      gdown_splits = k[2];
    }
    if (++k[which] > 64 || k[which] > all[which]->steps / 8) break;
  }
}

FfnWs::FfnWs(const mhcl_ffn_desc &d, bool grad, void *ws) : plan(d, grad) {
  WsCursor c(ws);
  const size_t T = static_cast<size_t>(d.T), C = static_cast<size_t>(d.C), H = static_cast<size_t>(d.H), es = plan.wide ? 4 : 2;
  a = c.take<char>(T * H * es);
  g_pre = grad ? c.take<char>(T * 2 * H * es) : nullptr;
  const auto parts = [](int splits) { return static_cast<size_t>(splits > 1 ? splits : 0); };
  const size_t x = std::max(parts(plan.down_splits), parts(plan.gx_splits)) * T * C, up = parts(plan.gup_splits) * 2 * H * C,
               down = parts(plan.gdown_splits) * H * C;
  slabs = c.take<float>(plan.trio ? x : std::max({x, up, down}));
  up_slabs = plan.trio ? c.take<float>(up) : slabs;
  down_slabs = plan.trio ? c.take<float>(down) : slabs;
  bytes = c.off;
}

hipError_t launch_ffn(const mhcl_ffn_desc &d, const void *x, const void *W_up, const void *W_down, void *y, float *pre, const FfnWs &w, hipStream_t s) {
  return dispatch_io(d.io_dtype, [&](auto io) { return run_ffn<decltype(io)>(d, x, W_up, W_down, y, pre, w, s); });
}

hipError_t launch_ffn_grad(const mhcl_ffn_desc &d, const void *x, const void *W_up, const void *W_down, const float *pre, const void *g_y, void *g_x,
                           void *g_W_up, void *g_W_down, const FfnWs &w, hipStream_t s) {
  return dispatch_io(d.io_dtype, [&](auto io) { return run_ffn_grad<decltype(io)>(d, x, W_up, W_down, pre, g_y, g_x, g_W_up, g_W_down, w, s); });
}

}  // namespace mhcl
