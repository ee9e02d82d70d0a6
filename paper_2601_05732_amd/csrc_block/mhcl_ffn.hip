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

// 1 / (1 + exp(-x)): by the instructions for bf16 operands, to 2^-22 + 2^-24 |x| of itself, the library's for fp32 ones
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
template <bool KEEP, bool WIDE>
struct GateEpilogue {
  static constexpr bool kWide = WIDE, kPaired = true;
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

// m: H, n: tokens.  The sums are g_a; g_G, g_U and a of them and of G and U, each rounded once.
template <bool WIDE>
struct GateGradEpilogue {
  static constexpr bool kWide = WIDE, kPaired = false;
  const float *pre;
  void *a, *g_pre;
  int64_t H, T;
  template <int FM, int FN>
  __device__ __forceinline__ int hold(int64_t, int64_t) const { return 0; }
  template <int FM, int FN>
  static constexpr int stores() { return FN * (WIDE ? FM : FM / 2) * 3; }
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
        store_two<WIDE>(a, n * H, m, q, v[0], v[1], here, H);
        store_two<WIDE>(g_pre, row, m, q, G[0], G[1], here, H);
        store_two<WIDE>(g_pre, row + H, m, q, U[0], U[1], here, H);
      }
    }
  }
};

// D[n][m] = sum over k, in `splits` slabs that are then joined, or at once
template <bool AK, bool BK, typename IO>
hipError_t product(const ProductTile &tile, const Operand &A, const Operand &B, int64_t M, int64_t N, int splits, float *slabs, void *out, hipStream_t s) {
  constexpr bool WIDE = IO::kVec == 4;
  const StoreEpilogue<WIDE> e{nullptr, splits > 1 ? slabs : (WIDE ? static_cast<float *>(out) : nullptr), static_cast<uint16_t *>(out), nullptr, M, N, M * N};
  const hipError_t err = launch_gemm<AK, BK>(tile, A, B, M, N, splits, e, s);
  return err != hipSuccess || splits == 1 ? err : launch_slab_sum<IO>(slabs, out, splits, M * N, s);
}

template <typename IO>
hipError_t run_ffn(const mhcl_ffn_desc &d, const void *x, const void *W_up, const void *W_down, void *y, float *pre, const FfnWs &w, hipStream_t s) {
  constexpr bool WIDE = IO::kVec == 4;
  const FfnPlan &p = w.plan;
  const int64_t T = d.T, C = d.C, H = d.H;
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
  if ((e = launch_gemm<false, true>(p.act, Wd, gk, H, T, 1, GateGradEpilogue<WIDE>{pre, w.a, w.g_pre, H, T}, s)) != hipSuccess) return e;
  if ((e = product<false, true, IO>(p.gx, Wu, pk, C, T, p.gx_splits, w.slabs, g_x, s)) != hipSuccess) return e;
  if ((e = product<false, false, IO>(p.gup, xm, pm, C, 2 * H, p.gup_splits, w.slabs, g_W_up, s)) != hipSuccess) return e;
  return product<false, false, IO>(p.gdown, am, gm, H, C, p.gdown_splits, w.slabs, g_W_down, s);
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
  if (T == 0) return;
  if (!grad) {
    down_splits = Split(down, C, T, H, wide).best();
  } else {
    gx_splits = Split(gx, C, T, 2 * H, wide).best();
    gup_splits = Split(gup, C, 2 * H, T, wide).best();
    gdown_splits = Split(gdown, H, C, T, wide).best();
  }
}

FfnWs::FfnWs(const mhcl_ffn_desc &d, bool grad, void *ws) : plan(d, grad) {
  WsCursor c(ws);
  const size_t T = static_cast<size_t>(d.T), C = static_cast<size_t>(d.C), H = static_cast<size_t>(d.H), es = plan.wide ? 4 : 2;
  a = c.take<char>(T * H * es);
  g_pre = grad ? c.take<char>(T * 2 * H * es) : nullptr;
  const auto parts = [](int splits) { return static_cast<size_t>(splits > 1 ? splits : 0); };
  slabs = c.take<float>(std::max({parts(plan.down_splits) * T * C, parts(plan.gx_splits) * T * C, parts(plan.gup_splits) * 2 * H * C,
                                  parts(plan.gdown_splits) * H * C}));
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
