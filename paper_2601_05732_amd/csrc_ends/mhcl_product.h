// Matrix products on the bf16 matrix units with a caller's epilogue, for the kernels around the layers: device code, the host's
// choice of tiles and parts, launches.
#pragma once
#include <algorithm>
#include <type_traits>

#include "../csrc/mhcl_common.h"
#include "../csrc/mhcl_mfma.h"
#include "mhcl_tiles.h"

namespace mhcl {
namespace {

constexpr int kBlock = 256;

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

// The time of a product of few tiles whose depth is split into parts, in sixtieths of a step of two blocks on a compute unit: `each` steps of a
// part, whose first loads and epilogue are the like of four more, `parts` of them at once.  filling: a block of the tile fills a compute unit; alone: a step's time
// of one that does not and has a unit for itself.  (Split on the host, TokenCount on the device.)
constexpr int64_t kChipBlocks = 256, kSumTime = 240;      // the sum over slabs, a launch
constexpr int alone_time(bool wide) { return wide ? 33 : 42; }
template <typename I>
__host__ __device__ constexpr I parts_time(I parts, I each, bool filling, I alone) {
  constexpr I UNITS = static_cast<I>(kChipBlocks);
  const I rest = parts % (2 * UNITS);
  const I step = filling ? (parts + UNITS - 1) / UNITS * 60 : parts / (2 * UNITS) * 60 + (rest == 0 ? 0 : (rest > UNITS ? 60 : alone));
  return step * (each + 4);
}

// How many tokens there are is known to the device alone: `count` of them less those of blocks before (`first`), at most as many as the host has sized the
// product for.  They are D's rows n, or (deep) its depth.
struct TokenCount {
  const int32_t *count;
  int64_t first;
  __device__ __forceinline__ int64_t of(int64_t most) const {
    const int64_t n = static_cast<int64_t>(*count) - first;
    return n < 0 ? 0 : (n < most ? n : most);
  }
  // Parts of the depth of a product over n, up to `most_parts` (0: as the host says): the number that ends first, of tiles_m tiles for
  // every bn tokens (a slab of the largest tile counting four times).  (us, 8192 tokens, of which 5700 count, C = 4096, 65536 rows, pairs, the whole call: one part 8471,
  // so 7840; all 8192 count 10600 and 10730.)
  int tiles_m, bn, steps, alone, most_parts;
  __device__ __forceinline__ int parts(int64_t rows) const {
    const int tiles = tiles_m * static_cast<int>((rows + bn - 1) / bn), slab = bn >= 256 ? 4 : 1;
    int best = 1, least = 0x7fffffff;
    for (int k = 1; k <= most_parts; ++k) {
      const int time = parts_time(tiles * k, (steps + k - 1) / k, bn >= 256, alone) + (k > 1 ? tiles * k * slab + static_cast<int>(kSumTime) : 0);
      if (time < least) least = time, best = k;
    }
    return best;
  }
};
struct GemmArgs {
  Operand A, B;
  int tiles_m, tiles_n, splits;
  TokenCount tokens;      // read with epilogues that are kCounted
  bool deep;
};
template <int BN, typename Epilogue>
__device__ __forceinline__ std::conditional_t<Epilogue::kCounted, GemmArgs, const GemmArgs &> counted(const GemmArgs &given) {
  if constexpr (Epilogue::kCounted) {
    GemmArgs g = given;
    if (g.deep) {
      g.A.depth = g.B.depth = g.tokens.of(given.A.depth);
    } else {
      g.B.rows = g.tokens.of(given.B.rows);
      g.tiles_n = static_cast<int>((g.B.rows + BN - 1) / BN);
      if (g.tokens.most_parts > 1) g.splits = g.tokens.parts(g.B.rows);
    }
    return g;
  } else {
    return given;
  }
}

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

// The same of an operand (KINNER) of two halves of rows / 2 rows, whose rows meet in a lane: the tile's rows are, for each wave, HALF of the first half
// and the HALF of the second that go with them, so that the fragments FM / 2 on are the former ones' partners.  (Rows past the first half are
// the second's first ones; they give results that nobody reads.)
template <int R, int NT, int HALF, bool WIDE>
struct PairedLoader {
  static constexpr int PER = R * 8 / NT, ES = WIDE ? 4 : 2, DEPTH = 128 / ES, kRows = NT / 8;
  static_assert(HALF == kRows || HALF * 2 == kRows, "a piece is of one half, or has both");
  const char *base;
  int64_t rest;
  int step, apart;
  uint32_t at, from;
  uint32_t second;          // bytes from a row to its partner (less than 2^31: the host sees to it)
  int depth;
  __device__ __forceinline__ void init(const Operand &o, int64_t row0) {
    const int tid = threadIdx.x, row = tid >> 3, c = (tid & 7) ^ ((tid >> 4) & 7);
    const int64_t skip = row0 / 2 * o.ld * ES;
    step = DEPTH * ES;
    apart = static_cast<int>(HALF * o.ld * ES);
    base = static_cast<const char *>(o.p) + skip;
    rest = o.rows * o.ld * ES - skip;
    second = static_cast<uint32_t>(o.rows / 2 * o.ld * ES);
    depth = c * (16 / ES);
    at = static_cast<uint32_t>(row % HALF * o.ld * ES + c * 16) + (row >= HALF ? second : 0u);
  }
  __device__ __forceinline__ void skip(int64_t bytes) { base += bytes, rest -= bytes; }
  __device__ __forceinline__ void aim(int left) { from = depth < left ? at : 0x80000000u; }
  __device__ __forceinline__ void piece(uint4 *tile, int wave, int i) const {
    const int range = rest <= 0 ? 0 : (rest > 0x7fffffff ? 0x7fffffff : static_cast<int>(rest));
    const uint32_t offset = HALF == kRows ? from + i / 2 * apart + (i % 2 ? second : 0u) : from + i * apart;
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

// The I-th array of N 16-byte pieces of LDS: one and the same for every product of a kernel that asks for it
template <int N, int I>
__device__ __forceinline__ uint4 *lds_array() {
  __shared__ uint4 a[N];
  return a;
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
// What an epilogue reads ahead it asks for after the last step, or (Epilogue::kEarly) before the first.
// Epilogue::kPaired: A's rows are two halves (PairedLoader).  block, blocks: its number of how many.  LEAST: of the pieces of an array in LDS, where a
// kernel has products of several tiles.
template <int BM, int BN, int WM, int WN, int STAGES, bool AK, bool BK, int LEAST, typename Epilogue>
__device__ __forceinline__ void gemm_tiles(const GemmArgs &given, const Epilogue &epilogue, int block, int blocks) {
  constexpr bool WIDE = Epilogue::kWide;
  const std::conditional_t<Epilogue::kCounted, GemmArgs, const GemmArgs &> g = counted<BN, Epilogue>(given);
  constexpr int NT = WM * WN * 64, FM = BM / WM / 16, FN = BN / WN / 16;
  static_assert(STAGES == 2 || STAGES == 4, "the loop over steps");
  // A's and B's tile of a stage.  Four stages' lie in an array each: of more arrays the compiler does not keep apart which loads fill which, and
  // waits for all of them.  (Two stages' in one array each: 1 % slower, 16384 tokens, C = 4096, 65536 rows.)
  constexpr int TA = BM * 8, TB = BN * 8;
  constexpr bool FOUR = STAGES == 4;
  constexpr int LM = std::max(FOUR ? TA + TB : TA, LEAST), LN = std::max(FOUR ? TA + TB : TB, LEAST);
  struct Stage {
    uint4 *a, *b;
  };
  uint4 *const m0 = lds_array<LM, 0>(), *const m1 = lds_array<LM, 1>(), *const m2 = lds_array<LN, 2>(), *const m3 = lds_array<LN, 3>();
  const Stage s0{m0, FOUR ? m0 + TA : m2}, s1{m1, FOUR ? m1 + TA : m3}, s2{m2, m2 + TA}, s3{m3, m3 + TA};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
  std::conditional_t<Epilogue::kPaired, PairedLoader<BM, NT, FM * 8, WIDE>, TileLoader<BM, NT, AK, WIDE>> la;
  static_assert(AK || !Epilogue::kPaired, "halves of rows");
  TileLoader<BN, NT, BK, WIDE> lb;
  const int64_t depth = g.A.depth < g.B.depth ? g.B.depth : g.A.depth;
  const int steps = static_cast<int>((depth + la.DEPTH - 1) / la.DEPTH);
  const int tiles = g.tiles_m * g.tiles_n * g.splits;
  if (Epilogue::kCounted && block >= tiles) return;
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
    decltype(epilogue.template hold<FM, FN>(0, 0)) held;
    if constexpr (Epilogue::kEarly)
      held = epilogue.template hold<FM, FN>(static_cast<int64_t>(tm) * BM + wm * (FM * 16), static_cast<int64_t>(tn) * BN + wn * (FN * 16));
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
    if constexpr (!Epilogue::kEarly) held = epilogue.template hold<FM, FN>(first_m, first_n);
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
  gemm_tiles<BM, BN, WM, WN, STAGES, AK, BK, 0>(g, epilogue, blockIdx.x, gridDim.x);
}

// The two gradients' products in one launch, where both have few parts: neither needs the other's result.  The first first_blocks blocks
// take g_h, the others g_W, a part each.  Up to two blocks for a compute unit (more than that loses: 7043 tokens,
// C = 560, 955 rows 79.2 / 90.1).  (us of the whole call with gradients, two launches / one: 333 tokens,
// C = 520, 1003 rows, bf16 28.4 / 23.1; 8, 256, 600 21.7 / 16.1; 1000, 512, 1000 35.0 / 27.5; 2000, 256, 600, fp32 64.7 / 50.5.)
constexpr int kSharedPieces = 128 * 8 + 32 * 8;   // of the smallest tile's arrays, which are the larger
template <bool SLIM, typename Epilogue>
__global__ __launch_bounds__(256, 2) void gemm_pair_kernel(const GemmArgs gh, const Epilogue to_gh, const GemmArgs gw, const Epilogue to_gw, int first_blocks) {
  constexpr int LEAST = SLIM ? kSharedPieces : 0;
  const int block = blockIdx.x;
  if (block < first_blocks) gemm_tiles<128, SLIM ? 32 : 128, SLIM ? 4 : 2, SLIM ? 1 : 2, SLIM ? 4 : 2, false, true, LEAST>(gh, to_gh, block, first_blocks);
  else gemm_tiles<128, 128, 2, 2, 2, false, false, LEAST>(gw, to_gw, block - first_blocks, gridDim.x - first_blocks);
}

// Four 16-bit results of a lane (r, q) at 16 i + 4 q and as many at 16 (i + 1) + 4 q become eight, for one 16-byte store, at 16 (i + q % 2) +
// 8 (q / 2): the lanes of odd q exchange the former for the latter of the lanes sixteen before.  (A store of 8 bytes writes 32 bytes
// of each of 16 rows: 16384 tokens, 65536 rows, 64 deep, us: 8 bytes 1166, whole rows by way of LDS 1064.)
__device__ __forceinline__ uint4 join_pairs(uint2 lower, uint2 upper) {
  const auto x = __builtin_amdgcn_permlane16_swap(lower.x, upper.x, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(lower.y, upper.y, false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}

// out[n][m], m innermost, times *scale (null: 1): fp32 slabs of splits (out32 != null), added to `add` if that is there; else rounded to bf16.
// COUNTED: row n goes to row[n] (null: n), and `tokens` bounds them.
template <bool WIDE, bool COUNTED = false>
struct StoreEpilogue {
  static constexpr bool kWide = WIDE, kPaired = false, kEarly = false, kCounted = COUNTED;
  const float *scale;
  float *out32;
  uint16_t *out16;
  const float *add;
  int64_t M, N, slab;     // elements of a split's slab
  const int32_t *row;
  TokenCount tokens;
  bool deep;
  float *slabs;           // COUNTED: of several parts, in rows as they are; one part goes where the rest says
  __device__ __forceinline__ int64_t rows() const {
    if constexpr (COUNTED) return deep ? N : tokens.of(N);
    return N;
  }
  template <int FM, int FN>
  __device__ __forceinline__ float hold(int64_t, int64_t) const { return scale ? *scale : 1.f; }
  template <int FM, int FN>
  static constexpr int stores() { return FN * (WIDE ? FM : FM / 2); }   // (into fp32 slabs twice as many)
  __device__ __forceinline__ bool whole(int64_t m_end, int64_t n_end) const { return m_end <= M && n_end <= rows(); }
  template <int FM, int FN>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[FM][FN], float factor, int64_t m0, int64_t n0, int split) const {
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int64_t end = rows();
    float *to32 = out32;
    const int32_t *map = row;
    if constexpr (COUNTED) {
      if (slabs && tokens.parts(end) > 1) to32 = slabs, map = nullptr;
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t n = n0 + 16 * j + r;
      int64_t to = n;
      if constexpr (COUNTED) {
        if (map && n < end) to = map[n];
      }
#pragma unroll
      for (int i = 0; i < FM; i += 2) {
        uint2 part[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int64_t m = m0 + 16 * (i + k) + 4 * q, elem = to * M + m;      // (M is a multiple of 8)
          const bool there = n < end && m < M;
          f32x4 v = acc[i + k][j] * factor;
          if (add && there) v += *reinterpret_cast<const f32x4 *>(add + elem);
          if (to32 && there) *reinterpret_cast<f32x4 *>(to32 + split * slab + elem) = v;
          part[k] = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
        if (!to32) {
          const uint4 eight = join_pairs(part[0], part[1]);
          const int64_t m = m0 + 16 * (i + (q & 1)) + 8 * (q >> 1);
          if (n < end && m < M) *reinterpret_cast<uint4 *>(out16 + to * M + m) = eight;
        }
      }
    }
  }
};

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

// The same of rows of M numbers, row n to row[n], as many as there are tokens, and parts where there are several
template <typename IO>
__global__ __launch_bounds__(kBlock) void slab_sum_rows_kernel(const float *__restrict__ in, void *__restrict__ out, int64_t N, int64_t M,
                                                               const int32_t *__restrict__ row, TokenCount tokens) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * 4, n = i / M, count = N * M, rows = tokens.of(N);
  if (n >= rows) return;
  const int slabs = tokens.parts(rows);
  if (slabs == 1) return;
  f32x4 s = *reinterpret_cast<const f32x4 *>(in + i);
#pragma unroll 4
  for (int k = 1; k < slabs; ++k) s += *reinterpret_cast<const f32x4 *>(in + k * count + i);
  const int64_t to = row[n] * M + i % M;
  if constexpr (IO::kVec == 4) *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + to) = s;
  else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + to) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
unsigned blocks(int64_t items, int64_t each) { return static_cast<unsigned>(ceil_div(items, each)); }

GemmArgs gemm_args(const ProductTile &tile, const Operand &A, const Operand &B, int64_t M, int64_t N, int splits, TokenCount tokens = {}, bool deep = false) {
  return {A, B, static_cast<int>(ceil_div(M, tile.bm)), static_cast<int>(ceil_div(N, tile.bn)), splits, tokens, deep};
}

template <bool AK, bool BK, typename Epilogue>
hipError_t launch_gemm(const ProductTile &tile, const Operand &A, const Operand &B, int64_t M, int64_t N, int splits, const Epilogue &e, hipStream_t s,
                       TokenCount tokens = {}, bool deep = false) {
  const GemmArgs g = gemm_args(tile, A, B, M, N, splits, tokens, deep);
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
ProductTile tile_for(int64_t M, int64_t N, int64_t parts, bool slim, bool big) {
  if (slim && (N <= 64 || ceil_div(M, 128) * ceil_div(N, 128) * parts < kChipBlocks * 3 / 4)) return kTileSlim;
  return big && ceil_div(M, 256) * ceil_div(N, 256) >= kChipBlocks ? kTileBig : kTileMid;
}

// Into how many parts the depth of a product of few tiles is split, each a slab of fp32 sums of its own: the number that is expected to end
// first, by parts_time (a block alone on a compute unit takes 0.7 of a step of two, fp32 0.55), a tile of a slab taking a sixtieth of a step for being
// written and read again by every 256 units, and the sum over slabs being a launch, kSumTime.  Parts of fewer than eight steps, or more than 64, are not taken.
// (us, one part / this many.  g_W of 7043 tokens, C = 560, 955 rows, bf16, 40 tiles, 6: 83.7 / 25.0; of 7621 tokens, C = 3768, 1317 rows, fp32, 330
// tiles, 3: 674 / 522.  g_h of 1000 tokens, C = 1024, 20000 rows, bf16, 64 tiles, 4 / 8: 69.1 / 52.9.)
struct Split {
  int64_t tiles, steps;
  bool alone, wide;      // alone: a block of the tile fills a compute unit
  Split(const ProductTile &tile, int64_t M, int64_t N, int64_t depth, bool w)
      : tiles(ceil_div(M, tile.bm) * ceil_div(N, tile.bn)), steps(ceil_div(depth, w ? 32 : 64)), alone(tile.bm == 256), wide(w) {}
  int64_t time(int k) const {   // without the sum
    return parts_time<int64_t>(tiles * k, ceil_div(steps, k), alone, alone_time(wide)) + (k > 1 ? tiles * k : 0);
  }
  int best() const {
    int k_best = 1;
    for (int k = 2; k <= 64 && k <= steps / 8; ++k)
      if (time(k) + kSumTime < time(k_best) + (k_best > 1 ? kSumTime : 0)) k_best = k;
    return k_best;
  }
};

}  // namespace
}  // namespace mhcl
