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

#include "../csrc/mhcl_common.h"
#include "mhcl_head.h"
#include "../csrc/mhcl_mfma.h"

namespace mhcl {
namespace {

constexpr int kBlock = 256;
constexpr float kLog2e = 1.4426950408889634f;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

// ---------------------------------------------------------------- products
// D[m][n] = sum_k A[m][k] B[n][k].  An operand lies in memory with k innermost (KINNER: row m or n starts at p + m ld), or with m or n
// innermost (row k starts at p + k ld).  rows: its extent in m or n; depth: in k.  Elements are bf16, or fp32 (WIDE), which the
// fragments in registers split into three bf16 parts of 8 significant bits each; six of the nine products of parts are added, small ones
// first, the other three being below 2^-23 of the whole.  (The fp32 matrix instruction does a sixteenth of the bf16 one's operations a
// cycle, and six products are more exact.)
struct Operand {
  const void *p;
  int64_t ld;
  int64_t rows, depth;
};

struct GemmArgs {
  Operand A, B;
  int tiles_m, tiles_n, splits;
};

// One operand's tile of R rows by 128 bytes in LDS, in 16-byte pieces, as the loads that go straight to LDS leave it (piece i at
// 16 i), so that a piece's place is chosen by which piece of memory a thread asks for.
//  KINNER: piece (row, c) of a row's eight at 8 row + (c ^ (row / 2 % 8)): the 16 rows that a fragment reads at one c lie in
//   all 64 banks once.
//  else, bf16: row k holds R / 8 pieces; the pairs of pieces (16 numbers, what a transposing read takes of a row) are exchanged
//   by k: pair m16 of row k at m16 ^ (k % 4 + 4 (k / 8 % 2)), so that the eight rows that half a wave reads lie in all banks.
//  else, fp32: row k holds R / 4 pieces; its units of four (16 numbers) are exchanged: unit m16 of row k at m16 ^ (k / 4 % 4), so that
//   the four rows that a read takes lie in all banks.
// A thread's pieces lie the same distance apart; the loads' own range check gives zeros past the operand's end.  (Rows of m or n
// outside of the operand give results that nobody reads.)
template <int R, int NT, bool KINNER, bool WIDE>
struct TileLoader {
  static constexpr int PER = R * 8 / NT, ES = WIDE ? 4 : 2, DEPTH = 128 / ES, PPR = R * ES / 16;
  static constexpr int kRows = KINNER ? NT / 8 : NT / PPR;   // rows of memory from one piece to the next
  static_assert(PER == 1 || (KINNER || !WIDE ? kRows % 16 == 0 : kRows == 8), "how the exchange of pieces goes on from one to the next");
  const char *base;         // of the tile and the next step
  int64_t rest;             // bytes from there to the operand's end
  int step, apart;          // bytes from one step to the next; from one piece to the next (a tile's are less than 2^31: the host sees to it)
  uint32_t at, from;        // bytes from `base` to the thread's first piece; the same, or out of range, for this step
  uint32_t unit;            // fp32, not KINNER: its unit's bytes, which the pieces exchange
  int depth;                // KINNER: k of the thread's pieces within the tile
  __device__ __forceinline__ void init(const Operand &o, int64_t row0) {
    const int tid = threadIdx.x;
    const int64_t skip = row0 * (KINNER ? o.ld : 1) * ES;
    step = static_cast<int>((KINNER ? DEPTH : DEPTH * o.ld) * ES);
    apart = static_cast<int>(kRows * o.ld * ES);
    base = static_cast<const char *>(o.p) + skip;
    rest = (KINNER ? o.rows : o.depth) * o.ld * ES - skip;
    depth = 0;
    unit = 0;
    if constexpr (KINNER) {
      const int c = (tid & 7) ^ ((tid >> 4) & 7);
      depth = c * (16 / ES);
      at = static_cast<uint32_t>((tid >> 3) * o.ld * ES + c * 16);
    } else if constexpr (WIDE) {
      const int slot = tid % PPR;
      unit = ((slot >> 2) ^ (tid / PPR >> 2 & 3)) << 6;
      at = static_cast<uint32_t>(tid / PPR * o.ld * ES + (slot & 3) * 16);
    } else {
      const int kr = tid / PPR, slot = tid % PPR;
      const int m = (((slot >> 1) ^ ((kr & 3) | ((kr >> 3) & 1) << 2)) * 2 + (slot & 1)) * 8;
      at = static_cast<uint32_t>((kr * o.ld + m) * ES);
    }
  }
  __device__ __forceinline__ void skip(int64_t bytes) { base += bytes, rest -= bytes; }
  // left: depth that is left of the operand from this step on, 0 or less for a tile of zeros
  __device__ __forceinline__ void aim(int left) { from = depth < left ? at : 0x80000000u; }
  __device__ __forceinline__ void piece(uint4 *tile, int wave, int i) const {
    const int range = rest <= 0 ? 0 : (rest > 0x7fffffff ? 0x7fffffff : static_cast<int>(rest));
    uint32_t offset = from + i * apart;
    if constexpr (!KINNER && WIDE) offset += unit ^ (i & 1) << 7;   // (eight rows on: k / 4 is two more)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, range, 0x00020000),
                                             (lds_void *)(tile + i * NT + wave * 64), 16, offset, 0, 0, 0);
  }
};

// Fragments of 16 rows, k = 32 s + 8 q .. + 7 for lane (r, q); fp32: k = 4 q .. + 3 and 16 + 4 q .. + 3, in both operands alike, so that
// a lane's first read is the one of bf16.  lane_at: the lane's place in fragment 0 at s = 0, in bytes.
template <int R, bool KINNER, bool WIDE>
__device__ __forceinline__ int lane_at() {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  if constexpr (KINNER) return r * 128 | (q ^ ((r >> 1) & 7)) << 4;
  if constexpr (WIDE) return q * 4 * (R * 4) | q << 6 | r << 2;
  // 16 lanes read rows k .. k + 3, 32 bytes of each, and get a column of four each
  return (q * 8 + (r >> 2)) * (R * 2) | ((r >> 2) | (q & 1) << 2) << 5 | (r & 3) << 3;
}
// the same for the fragments from the first-th on (a power of two of them, first a multiple of it)
template <int R, bool KINNER, bool WIDE>
__device__ __forceinline__ int lane_at(int first) {
  if constexpr (KINNER) return lane_at<R, KINNER, WIDE>() + first * 2048;
  return lane_at<R, KINNER, WIDE>() ^ first << (WIDE ? 6 : 5);
}
template <int R, bool KINNER>
__device__ __forceinline__ u32x4 fragment(const uint4 *tile, int at, int f, int s) {
  const char *p = reinterpret_cast<const char *>(tile);
  if constexpr (KINNER) {
    return *reinterpret_cast<const u32x4 *>(p + (at ^ s << 6) + f * 2048);
  } else {
    const char *from = p + (at ^ f << 5) + s * (32 * R * 2);
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)from);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(from + 4 * R * 2));
    const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
    return u32x4{l[0], l[1], h[0], h[1]};
  }
}
// fp32: eight numbers, and their parts
struct Eight {
  f32x4 v[2];
};
template <int R, bool KINNER>
__device__ __forceinline__ Eight wide_fragment(const uint4 *tile, int at, int f) {
  const char *p = reinterpret_cast<const char *>(tile);
  Eight e;
  if constexpr (KINNER) {
    e.v[0] = *reinterpret_cast<const f32x4 *>(p + at + f * 2048);
    e.v[1] = *reinterpret_cast<const f32x4 *>(p + (at ^ 64) + f * 2048);
  } else {
    const char *from = p + (at ^ f << 6);
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i / 4][i % 4] = *reinterpret_cast<const float *>(from + (i / 4 * 16 + i % 4) * (R * 4));
  }
  return e;
}
struct Parts {
  u32x4 p[3];
};
// The rest after a part is a product of the pair of parts with (-1, 0) or (0, -1) added to the number: one instruction, and exact, since the
// rest is one of the fp32 numbers.  (An infinity's rest is NaN and its neighbour's too: both meet in the same sums.)
__device__ __forceinline__ Parts parts_of(const Eight &e) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  uint32_t first = 0x0000bf80u, second = 0xbf800000u;
  asm("" : "+s"(first));      // (as a constant in the instruction it would stand for both halves)
  asm("" : "+s"(second));
  Parts r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo = e.v[i / 2][i % 2 * 2], hi = e.v[i / 2][i % 2 * 2 + 1];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint32_t two = cvt_pk_bf16(lo, hi);
      r.p[k][i] = two;
      const bf16x2 pair = __builtin_bit_cast(bf16x2, two);
      lo = __builtin_amdgcn_fdot2_f32_bf16(pair, __builtin_bit_cast(bf16x2, first), lo, false);
      hi = __builtin_amdgcn_fdot2_f32_bf16(pair, __builtin_bit_cast(bf16x2, second), hi, false);
    }
  }
  return r;
}

// (the addresses of exchanged pieces take an instruction each; kept from step to step they would take a register each)
template <bool KINNER>
__device__ __forceinline__ int formed_here(int at) {
  if constexpr (!KINNER) asm volatile("" : "+v"(at));
  return at;
}
template <int LOADS>
__device__ __forceinline__ void wait_all_but() {   // the last LOADS loads
  static_assert(LOADS < 64, "what the counter holds");
  __builtin_amdgcn_s_waitcnt(0x0070 | (LOADS & 15) | (LOADS >> 4) << 14);
}
__device__ __forceinline__ void wait_all() { __builtin_amdgcn_s_waitcnt(0x0070); }   // vmcnt(0) lgkmcnt(0)
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The b-th tile (tm, tn, split), b being a block's number and then every gridDim.x-th: blocks of one XCD (every eighth) take
// neighbouring tiles, in strips of eight tiles of m
__device__ __forceinline__ void tile_of(const GemmArgs &g, int b, int &tm, int &tn, int &split) {
  const int total = g.tiles_m * g.tiles_n * g.splits;
  const int each = total / 8, more = total % 8, xcd = b % 8;
  int i = xcd * each + min(xcd, more) + b / 8;
  const int per = g.tiles_m * g.tiles_n;
  split = i / per;
  i -= split * per;
  constexpr int STRIP = 8;
  const int strip = i / (STRIP * g.tiles_n), m0 = strip * STRIP, width = min(STRIP, g.tiles_m - m0);
  i -= strip * STRIP * g.tiles_n;
  tm = m0 + i % width;
  tn = i / width;
}

// A block of WM x WN waves computes BM x BN tiles; wave (wm, wn) rows wm BM / WM of one and columns wn BN / WN on.
// The epilogue gets acc[fm][fn]: lane (r, q) holds m = 16 fm + 4 q + 0..3 of the wave's rows, n = 16 fn + r of its columns.
// The next tile's first loads are on their way during the epilogue, and the epilogue's stores during the next tile's first step.
// STAGES steps' tiles are in LDS or on their way there: two where products hide the way, four of the smallest tile, whose products are few
// (us, 333 tokens, C = 520, 1003 rows, logits / g_h: two 11.0 / 7.6, four 8.1 / 6.4; four of the middle tile are none the faster
// where there are few blocks, g_W 9.1 / 10.4).
// 256 x 256 tiles of eight waves, bound by the matrix units and the clock that they leave the chip (busy 64 to 68 % of the cycles at
// 1.87 GHz on one card, 62 to 66 % at 1.95 on another): 16384 tokens, C = 4096, 65536 rows, bf16, logits / g_h / g_W 7.0 / 6.7 / 7.0 ms
// there, 6.7 / 6.4 / 6.8 here, 1.25 to 1.37 PFLOP/s (a wave of 128 x 128 and four of them, raised wave priorities, barriers in the middle of a step, strips of 4 or 16 tiles: no faster).
// 128 x 128 of four waves: fp32, 2048 tokens, C = 768, 50257 rows 0.93 / 0.81 / 0.92 ms and 0.88 / 0.77 / 0.89, 1.0 to 1.2 PFLOP/s of bf16 products;
// matrix units busy for 49 % of the cycles, the vector ones, which take the parts, for 36 %.
// 128 x 32: one token, C = 4096, 50257 rows 70 to 80 us from card to card, W at 5.1 to 5.9 TB/s.
// block, blocks: its number of how many.
template <int BM, int BN, int WM, int WN, int STAGES, bool AK, bool BK, typename Epilogue>
__device__ __forceinline__ void gemm_tiles(const GemmArgs &g, const Epilogue &epilogue, int block, int blocks) {
  constexpr bool WIDE = Epilogue::kWide;
  constexpr int NT = WM * WN * 64, FM = BM / WM / 16, FN = BN / WN / 16;
  static_assert(STAGES == 2 || STAGES == 4, "the loop over steps");
  // A's and B's tile of a stage.  Four stages' lie in an array each: of more arrays the compiler does not keep apart which loads fill which, and
  // waits for all of them.  (Two stages' in one array each: 1 % slower, 16384 tokens, C = 4096, 65536 rows.)
  constexpr int TA = BM * 8, TB = BN * 8;
  constexpr bool FOUR = STAGES == 4;
  __shared__ uint4 m0[FOUR ? TA + TB : TA], m1[FOUR ? TA + TB : TA], m2[FOUR ? TA + TB : 1], m3[FOUR ? TA + TB : 1];
  __shared__ uint4 n0[FOUR ? 1 : TB], n1[FOUR ? 1 : TB];
  struct Stage {
    uint4 *a, *b;
  };
  const Stage s0{m0, FOUR ? m0 + TA : n0}, s1{m1, FOUR ? m1 + TA : n1}, s2{m2, m2 + TA}, s3{m3, m3 + TA};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
  TileLoader<BM, NT, AK, WIDE> la;
  TileLoader<BN, NT, BK, WIDE> lb;
  const int64_t depth = g.A.depth < g.B.depth ? g.B.depth : g.A.depth;
  const int steps = static_cast<int>((depth + la.DEPTH - 1) / la.DEPTH);
  const int tiles = g.tiles_m * g.tiles_n * g.splits;
  int tile = block, tm, tn, split;
  int at, to_load, to_do;         // step of the next load; steps to load, and to multiply
  const auto begin = [&]() __attribute__((always_inline)) {
    tile_of(g, tile, tm, tn, split);
    at = static_cast<int>(static_cast<int64_t>(steps) * split / g.splits);
    to_load = to_do = static_cast<int>(static_cast<int64_t>(steps) * (split + 1) / g.splits) - at;
    la.init(g.A, static_cast<int64_t>(tm) * BM);
    lb.init(g.B, static_cast<int64_t>(tn) * BN);
    la.skip(static_cast<int64_t>(at) * la.step);
    lb.skip(static_cast<int64_t>(at) * lb.step);
  };
  f32x4 acc[FM][FN];
  const auto aim = [&]() __attribute__((always_inline)) {
    const int done = to_load-- > 0 ? at * la.DEPTH : 0x7fffffff;   // past the last step: zeros
    la.aim(static_cast<int>(g.A.depth) - done);
    lb.aim(static_cast<int>(g.B.depth) - done);
  };
  const auto next = [&]() __attribute__((always_inline)) {
    ++at;
    la.skip(la.step);
    lb.skip(lb.step);
  };
  constexpr int HM = FM / 2;
  const int at_a = lane_at<BM, AK, WIDE>(wm * FM), at_b = lane_at<BN, BK, WIDE>(wn * FN);
  const auto piece_of = [&](const Stage &st, int p) __attribute__((always_inline)) {
    if (p < la.PER) la.piece(st.a, wave, p);
    else if (p < la.PER + lb.PER) lb.piece(st.b, wave, p - la.PER);
  };
  // The oldest of STAGES stages has arrived, whatever has been asked for since.
  constexpr int PER = la.PER + lb.PER;
  const auto wait_stage = [&]() __attribute__((always_inline)) { wait_all_but<(STAGES - 2) * PER>(); };
  // A step is four groups of products, (k half s, half hm of the rows), whose fragments are read one group ahead.  Once the last
  // group's have arrived the stage is free and the next one's tiles are needed: there the waves meet, and
  // the next step's first fragments are on their way while the last group multiplies.
  u32x4 fa[2][HM], fb[2][FN];
  const auto read_a = [&](const Stage &st, int s, int hm) __attribute__((always_inline)) {
    const int here = formed_here<AK>(at_a);
#pragma unroll
    for (int i = 0; i < HM; ++i) fa[hm][i] = fragment<BM, AK>(st.a, here, hm * HM + i, s);
  };
  const auto read_b = [&](const Stage &st, int s) __attribute__((always_inline)) {
    const int here = formed_here<BK>(at_b);
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[s][j] = fragment<BN, BK>(st.b, here, j, s);
  };
  // one row of fragments after the other, `between(i)` after row i
  const auto products = [&](int s, int hm, auto between) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < HM; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[hm * HM + i][j] = mfma16(fa[hm][i], fb[s][j], acc[hm * HM + i][j]);
      __builtin_amdgcn_sched_barrier(0);
      between(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto nothing = [](int) {};
  const auto step = [&](const Stage &st, const Stage &st_next) __attribute__((always_inline)) {
    read_a(st, 0, 1);
    products(0, 0, nothing);
    read_b(st, 1);
    read_a(st, 1, 0);
    products(0, 1, nothing);
    read_a(st, 1, 1);
    products(1, 0, nothing);
    wait_stage();
    barrier();
    read_a(st_next, 0, 0);
    read_b(st_next, 0);
    aim();
    // the tiles after the next take this step's place
    products(1, 1, [&](int i) __attribute__((always_inline)) {
      constexpr int EACH = (PER + HM - 1) / HM;
#pragma unroll
      for (int p = i * EACH; p < (i + 1) * EACH; ++p) piece_of(st, p);
    });
    next();
  };
  // fp32: two groups, (half hm of the rows), six products of parts each; the second one's numbers are read under the first one's products and the next
  // step's under the second one's.
  Eight ea[HM], eb[FN];
  Parts pa[HM], pb[FN];
  const auto read_wide_a = [&](const Stage &st, int hm) __attribute__((always_inline)) {
    const int here = formed_here<AK>(at_a);
#pragma unroll
    for (int i = 0; i < HM; ++i) ea[i] = wide_fragment<BM, AK>(st.a, here, hm * HM + i);
  };
  const auto read_wide_b = [&](const Stage &st) __attribute__((always_inline)) {
    const int here = formed_here<BK>(at_b);
#pragma unroll
    for (int j = 0; j < FN; ++j) eb[j] = wide_fragment<BN, BK>(st.b, here, j);
  };
  const auto wide_products = [&](int hm, auto between) __attribute__((always_inline)) {
    constexpr int A[6] = {1, 0, 2, 0, 1, 0}, B[6] = {1, 2, 0, 1, 0, 0};
#pragma unroll
    for (int k = 0; k < 6; ++k) {
#pragma unroll
      for (int i = 0; i < HM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[hm * HM + i][j] = mfma16(pa[i].p[A[k]], pb[j].p[B[k]], acc[hm * HM + i][j]);
      between(k);
    }
  };
  const auto wide_step = [&](const Stage &st, const Stage &st_next) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < FN; ++j) pb[j] = parts_of(eb[j]);
#pragma unroll
    for (int i = 0; i < HM; ++i) pa[i] = parts_of(ea[i]);
    read_wide_a(st, 1);
    wide_products(0, nothing);
#pragma unroll
    for (int i = 0; i < HM; ++i) pa[i] = parts_of(ea[i]);
    __builtin_amdgcn_sched_barrier(0);
    wait_stage();
    barrier();
    read_wide_a(st_next, 0);
    read_wide_b(st_next);
    aim();
    wide_products(1, [&](int k) __attribute__((always_inline)) {
      constexpr int EACH = (PER + 5) / 6;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = k * EACH; p < (k + 1) * EACH; ++p) piece_of(st, p);
      __builtin_amdgcn_sched_barrier(0);
    });
    next();
  };
  const auto load = [&](const Stage &st) __attribute__((always_inline)) {
    aim();
#pragma unroll
    for (int p = 0; p < PER; ++p) piece_of(st, p);
    next();
  };
  const auto fill = [&]() __attribute__((always_inline)) {
    begin();
    load(s0);
    load(s1);
    if constexpr (STAGES == 4) {
      load(s2);
      load(s3);
    }
  };
  const auto any_step = [&](const Stage &st, const Stage &st_next) __attribute__((always_inline)) {
    if constexpr (WIDE) wide_step(st, st_next);
    else step(st, st_next);
  };
  fill();
  bool stored = false;            // whether every wave's stores of the last epilogue were what stores<>() says at least
  for (;;) {
    if (stored) wait_all_but<(STAGES - 1) * PER + Epilogue::template stores<FM, FN>()>();
    else wait_all_but<(STAGES - 1) * PER>();
    barrier();
    if constexpr (WIDE) {
      read_wide_a(s0, 0);
      read_wide_b(s0);
    } else {
      read_a(s0, 0, 0);
      read_b(s0, 0);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (a stage's place is known where it is read: the steps of two stages in pairs, after an odd last one a step of zeros)
    if constexpr (STAGES == 2) {
      for (int left = to_do; left > 0; left -= 2) {
        any_step(s0, s1);
        any_step(s1, s0);
      }
    } else {
      // (the last ones after the loop: left from its middle, it would wait for all loads at its head)
      int left = to_do;
      for (; left >= 4; left -= 4) {
        any_step(s0, s1);
        any_step(s1, s2);
        any_step(s2, s3);
        any_step(s3, s0);
      }
      if (left > 0) any_step(s0, s1);
      if (left > 1) any_step(s1, s2);
      if (left > 2) any_step(s2, s3);
    }
    const int64_t first_m = static_cast<int64_t>(tm) * BM + wm * (FM * 16), first_n = static_cast<int64_t>(tn) * BN + wn * (FN * 16);
    const int this_split = split;
    const auto held = epilogue.template hold<FN>(first_n);
    // the stages are free once the last loads (of zeros) have arrived and every wave has read its fragments
    wait_all();
    barrier();
    stored = epilogue.whole(static_cast<int64_t>(tm + 1) * BM, static_cast<int64_t>(tn + 1) * BN);
    tile += blocks;
    const bool more = tile < tiles;
    if (more) fill();
    epilogue.template operator()<FM, FN>(acc, held, first_m, first_n, this_split);
    if (!more) break;
  }
}

template <int BM, int BN, int WM, int WN, int STAGES, bool AK, bool BK, typename Epilogue>
__global__ __launch_bounds__(WM *WN * 64, 2) void gemm_kernel(const GemmArgs g, const Epilogue epilogue) {
  gemm_tiles<BM, BN, WM, WN, STAGES, AK, BK>(g, epilogue, blockIdx.x, gridDim.x);
}

// The two gradients' products in one launch, where both have few parts: neither needs the other's result.  The first first_blocks blocks
// take g_h, the others g_W, a part each.  Up to two blocks for a compute unit, though one is there at a time (more than that loses: 7043 tokens,
// C = 560, 955 rows 79.2 / 90.1).  (us of the whole call with gradients, two launches / one: 333 tokens,
// C = 520, 1003 rows, bf16 28.4 / 23.1; 8, 256, 600 21.7 / 16.1; 1000, 512, 1000 35.0 / 27.5; 2000, 256, 600, fp32 64.7 / 50.5.)
template <bool SLIM, typename Epilogue>
__global__ __launch_bounds__(256, 1) void gemm_pair_kernel(const GemmArgs gh, const Epilogue to_gh, const GemmArgs gw, const Epilogue to_gw, int first_blocks) {
  const int block = blockIdx.x;
  if (block < first_blocks) gemm_tiles<128, SLIM ? 32 : 128, SLIM ? 4 : 2, SLIM ? 1 : 2, SLIM ? 4 : 2, false, true>(gh, to_gh, block, first_blocks);
  else gemm_tiles<128, 128, 2, 2, 2, false, false>(gw, to_gw, block - first_blocks, gridDim.x - first_blocks);
}

// Four 16-bit results of a lane (r, q) at 16 i + 4 q and as many at 16 (i + 1) + 4 q become eight, for one 16-byte store, at 16 (i + q % 2) +
// 8 (q / 2): the lanes of odd q exchange the former for the latter of the lanes sixteen before.  (A store of 8 bytes writes 32 bytes
// of each of 16 rows: 16384 tokens, 65536 rows, 64 deep, us: 8 bytes 1166, whole rows by way of LDS 1064.)
__device__ __forceinline__ uint4 join_pairs(uint2 lower, uint2 upper) {
  const auto x = __builtin_amdgcn_permlane16_swap(lower.x, upper.x, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(lower.y, upper.y, false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}

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
  static constexpr bool kWide = WIDE;
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

// out[n][m], m innermost, times *scale: fp32 slabs of splits (out32 != null), added to `add` if that is there; else rounded to bf16
template <bool WIDE>
struct StoreEpilogue {
  static constexpr bool kWide = WIDE;
  const float *scale;
  float *out32;
  uint16_t *out16;
  const float *add;
  int64_t M, N, slab;     // elements of a split's slab
  template <int FN>
  __device__ __forceinline__ float hold(int64_t) const { return *scale; }
  template <int FM, int FN>
  static constexpr int stores() { return FN * (WIDE ? FM : FM / 2); }   // (into fp32 slabs twice as many)
  __device__ __forceinline__ bool whole(int64_t m_end, int64_t n_end) const { return m_end <= M && n_end <= N; }
  template <int FM, int FN>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[FM][FN], float factor, int64_t m0, int64_t n0, int split) const {
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t n = n0 + 16 * j + r;
#pragma unroll
      for (int i = 0; i < FM; i += 2) {
        uint2 part[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int64_t m = m0 + 16 * (i + k) + 4 * q, elem = n * M + m;      // (M is a multiple of 8)
          const bool there = n < N && m < M;
          f32x4 v = acc[i + k][j] * factor;
          if (add && there) v += *reinterpret_cast<const f32x4 *>(add + elem);
          if (out32 && there) *reinterpret_cast<f32x4 *>(out32 + split * slab + elem) = v;
          part[k] = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
        if (!out32) {
          const uint4 eight = join_pairs(part[0], part[1]);
          const int64_t m = m0 + 16 * (i + (q & 1)) + 8 * (q >> 1);
          if (n < N && m < M) *reinterpret_cast<uint4 *>(out16 + n * M + m) = eight;
        }
      }
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

// out = the sum of `slabs` slabs of `count` floats (a multiple of 4), in order
template <typename IO>
__global__ __launch_bounds__(kBlock) void slab_sum_kernel(const float *__restrict__ in, void *__restrict__ out, int slabs, int64_t count) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * 4;
  if (i >= count) return;
  f32x4 s = *reinterpret_cast<const f32x4 *>(in + i);
#pragma unroll 4
  for (int k = 1; k < slabs; ++k) s += *reinterpret_cast<const f32x4 *>(in + k * count + i);
  if constexpr (IO::kVec == 4) *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + i) = s;
  else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + i) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
}

constexpr int64_t kChipBlocks = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
unsigned blocks(int64_t items, int64_t each) { return static_cast<unsigned>(ceil_div(items, each)); }

template <typename F>
hipError_t dispatch_id(int id_dtype, F &&f) {
  if (id_dtype == MHCL_I64) return f(int64_t{});
  return f(int32_t{});
}

GemmArgs gemm_args(const HeadTile &tile, const Operand &A, const Operand &B, int64_t M, int64_t N, int splits) {
  return {A, B, static_cast<int>(ceil_div(M, tile.bm)), static_cast<int>(ceil_div(N, tile.bn)), splits};
}

template <bool AK, bool BK, typename Epilogue>
hipError_t launch_gemm(const HeadTile &tile, const Operand &A, const Operand &B, int64_t M, int64_t N, int splits, const Epilogue &e, hipStream_t s) {
  const GemmArgs g = gemm_args(tile, A, B, M, N, splits);
  // as many blocks as the chip holds (of the smallest tile, which waits for memory, one for every tile)
  const unsigned tiles = static_cast<unsigned>(g.tiles_m * g.tiles_n * splits), most = tile.bm == 256 ? kChipBlocks : 2 * kChipBlocks;
  const dim3 grid(tile.bn < 128 || tiles < most ? tiles : most);
  if (tile.bm == 256) {
    if constexpr (!Epilogue::kWide) hipLaunchKernelGGL((gemm_kernel<256, 256, 2, 4, 2, AK, BK, Epilogue>), grid, dim3(512), 0, s, g, e);
    else return hipErrorInvalidValue;
  } else if (tile.bn == 128) {
    hipLaunchKernelGGL((gemm_kernel<128, 128, 2, 2, 2, AK, BK, Epilogue>), grid, dim3(256), 0, s, g, e);
  } else {
    if constexpr (BK) hipLaunchKernelGGL((gemm_kernel<128, 32, 4, 1, 4, AK, BK, Epilogue>), grid, dim3(256), 0, s, g, e);
    else return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename IO>
hipError_t launch_slab_sum(const float *slabs, void *out, int count, int64_t elems, hipStream_t s) {
  hipLaunchKernelGGL((slab_sum_kernel<IO>), dim3(blocks(elems, kBlock * 4)), dim3(kBlock), 0, s, slabs, out, count, elems);
  return hipGetLastError();
}

// the largest tile of which there are enough for the chip (of fp32 operands the middle one: the largest one's registers do not hold their
// numbers and parts besides the sums)
// The smallest one for the few tokens of a step of decoding, or where the middle one leaves a quarter of the chip without work; `parts`: into
// how many the depth can be split.  (us, middle / smallest.  Logits and g_h of 333 tokens, C = 520, 1003 rows, bf16 16.4, 12.4 / 11.0, 7.8.  The
// loss alone, bf16: 1000 tokens, C = 1024, 2000 rows, 128 tiles 22.1 / 17.5; 300, 2048, 8000, 189 tiles 30.5 / 29.5; 600, 256, 5000, 200
// tiles 13.1 / 14.3; 140, 512, 16000, 250 tiles 14.0 / 15.5; 120, 1024, 30000, 235 tiles 22.7 / 24.3, but 158, 3776, 12304, 194 tiles 47.3 /
// 36.2.  fp32: 300, 1024, 6000, 141 tiles 54.3 / 39.2.)
HeadTile tile_for(int64_t M, int64_t N, int64_t parts, bool slim, bool big) {
  if (slim && (N <= 64 || ceil_div(M, 128) * ceil_div(N, 128) * parts < kChipBlocks * 3 / 4)) return kTileSlim;
  return big && ceil_div(M, 256) * ceil_div(N, 256) >= kChipBlocks ? kTileBig : kTileMid;
}

// Into how many parts the depth of a product of few tiles is split, each a slab of fp32 sums of its own: the number that is expected to end
// first, in sixtieths of a step of two blocks on a compute unit.  A block alone there takes 0.7 of that for a step (fp32: 0.55), a part the like of
// four steps for its first loads and its epilogue, a tile of a slab a sixtieth for being written and read again by every 256 units,
// and the sum over slabs is a launch, kSumTime.  Parts of fewer than eight steps, or more than 64, are not taken.
// (us, one part / this many.  g_W of 7043 tokens, C = 560, 955 rows, bf16, 40 tiles, 6: 83.7 / 25.0; of 7621 tokens, C = 3768, 1317 rows, fp32, 330
// tiles, 3: 674 / 522.  g_h of 1000 tokens, C = 1024, 20000 rows, bf16, 64 tiles, 4 / 8: 69.1 / 52.9.)
constexpr int64_t kSumTime = 240;
struct Split {
  int64_t tiles, steps;
  bool alone, wide;      // alone: a block of the tile fills a compute unit
  Split(const HeadTile &tile, int64_t M, int64_t N, int64_t depth, bool w)
      : tiles(ceil_div(M, tile.bm) * ceil_div(N, tile.bn)), steps(ceil_div(depth, w ? 32 : 64)), alone(tile.bm == 256), wide(w) {}
  int64_t time(int k) const {   // without the sum
    const int64_t parts = tiles * k, rest = parts % (2 * kChipBlocks);
    const int64_t step = alone ? ceil_div(parts, kChipBlocks) * 60
                               : parts / (2 * kChipBlocks) * 60 + (rest == 0 ? 0 : rest > kChipBlocks ? 60 : wide ? 33 : 42);
    return step * (ceil_div(steps, k) + 4) + (k > 1 ? parts : 0);
  }
  int best() const {
    int k_best = 1;
    for (int k = 2; k <= 64 && k <= steps / 8; ++k)
      if (time(k) + kSumTime < time(k_best) + (k_best > 1 ? kSumTime : 0)) k_best = k;
    return k_best;
  }
};

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
