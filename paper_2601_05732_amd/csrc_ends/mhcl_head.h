// Host-side declarations of the head's losses: cross entropy and pairs of sequences (mhcl_head.hip), a teacher's top logits (mhcl_distill.hip).
#pragma once
#include "mhcl_ends.h"
#include "mhcl_tiles.h"

namespace mhcl {

constexpr int32_t kHeadMostRows = (1 << 22) - 256;   // of the vocabulary

struct HeadPlan {
  bool wide;            // fp32 operands
  ProductTile logits, gh, gw;
  int64_t tokens;       // of a block
  int64_t ld;           // row of the softmax's numerators: V, filled up to whole tiles
  int64_t granules;     // partial sums of a row
  int gh_splits, gw_splits;   // parts of the vocabulary in the product for g_h, of the tokens in that for g_W
  bool pair;            // the products for g_h and g_W in one launch
  HeadPlan(const mhcl_ends_desc &d, bool grad, bool ordered);   // ordered: tokens are left out, how many the host does not know (TokenOrder)
};

struct HeadWs {
  HeadPlan plan;
  char *hp;             // [tokens][C]: h, zeros where a token does not count
  char *E;              // [tokens][ld] numerators in 16 bits, then g in bf16 in their place; fp32: 32 bits each
  float2 *stat;         // [tokens][granules] maximum and sum
  float *zt;            // [tokens] the targets' logits
  float *common;        // [2] what all weights are multiples of, in g_h and in g_W
  float *slabs;         // [gh_splits][tokens][C]
  float *gw_slabs;      // [gw_splits][V][C]
  float *gW;            // [V][C] sums over blocks of tokens
  size_t bytes;
  HeadWs(const mhcl_ends_desc &d, bool grad, void *ws, bool ordered = false);
};

// g_h, g_W null: the loss alone.  weight null: that of the mean.  unrounded: g_h and g_W are fp32, whatever the operands.
hipError_t launch_head(const mhcl_ends_desc &d, const void *h, const void *W, const void *targets, const float *weight,
                       float *loss, float *lse, void *g_h, void *g_W, bool unrounded, const HeadWs &w, hipStream_t s);

// targets null: all count
hipError_t launch_head_total(const mhcl_ends_desc &d, const void *targets, const float *loss, const float *weight, float *total,
                             hipStream_t s);
// Tokens in an order of their own, those that count first (mhcl_head_rows.h), for products that are large enough that what the others cost is more than
// the order.  (us, pairs, without / with; bf16, 1024 tokens, C = 1024, 16384 rows, all count 155 / 167, 70 % 134 / 135, 40 % 130 / 118; 2048, 768, 32768
// 372 / 389, 363 / 308, 350 / 232, and the loss alone 97 / 111, 101 / 90, 101 / 66; fp32, 1024, 1024, 16384 581 / 600, 556 / 482, 540 / 315.  Distillation, which
// needs all logits: bf16, 4096, 1024, 32768 904 / 908, 95 % 901 / 897, 70 % 886 / 787.)
struct TokenOrder {
  int32_t *row = nullptr;       // [T] the order
  int32_t *count = nullptr;     // [1] how many count
  int32_t *counts = nullptr;    // [T / 4096] of a block of threads
  char *hp = nullptr;           // [tokens of a block][C] h's rows in this order
  // (multiplications of a product, of which fp32 operands' are six)
  static bool pays(const mhcl_ends_desc &d, double least) {
    return static_cast<double>(d.T) * d.C * d.V * (d.io_dtype == MHCL_F32 ? 4 : 1) >= least;
  }
  void take(WsCursor &c, const mhcl_ends_desc &d, const HeadWs &head) {
    row = c.take<int32_t>(static_cast<size_t>(d.T));
    count = c.take<int32_t>(1);
    counts = c.take<int32_t>(static_cast<size_t>(d.T) / 4096 + 1);
    const size_t rows = static_cast<size_t>(head.plan.tokens) * d.C * (head.plan.wide ? 4 : 2);
    hp = head.hp ? head.hp : c.take<char>(rows);
  }
};
constexpr double kOrderPairs = 0x1p35, kOrderDistill = 0x1p37;

// A loss of pairs of sequences
constexpr int32_t kMostPairs = 1 << 22;   // a block of threads each
struct PairArgs {
  const float *reference;   // [2 pairs], may be null
  const float *weight;      // [pairs], null: that of the mean
  float *loss, *logp;       // [pairs], [2 pairs]
  int64_t T;
  int32_t pairs;
  float beta, smoothing;
  const float *ce;          // [T] cross entropies
  float *token_weight;      // [T], null: the loss alone
};
struct PreferenceWs {
  HeadWs head;
  float *ce, *lse, *token_weight;   // [T]
  TokenOrder order;
  bool ordered;
  size_t bytes;
  PreferenceWs(const mhcl_ends_desc &d, bool grad, void *ws) : head(d, grad, ws, TokenOrder::pays(d, kOrderPairs)) {
    WsCursor c(ws ? static_cast<char *>(ws) + head.bytes : nullptr);
    ce = c.take<float>(static_cast<size_t>(d.T));
    lse = c.take<float>(static_cast<size_t>(d.T));
    token_weight = grad ? c.take<float>(static_cast<size_t>(d.T)) : nullptr;
    ordered = TokenOrder::pays(d, kOrderPairs);
    if (ordered) order.take(c, d, head);
    bytes = head.bytes + c.off;
  }
};
hipError_t launch_preference(const mhcl_ends_desc &d, const void *h, const void *W, const void *targets, const void *offsets, int offset_dtype,
                             PairArgs a, void *g_h, void *g_W, bool unrounded, const PreferenceWs &w, hipStream_t s);

constexpr int kMostSlots = 256;   // of a token's teacher
struct DistillWs {
  HeadWs head;
  int32_t *mark;        // [T] negative where the teacher says nothing, 1 where it is a mistake (a row past the vocabulary, NaN, infinity), else 0
  // of a block of tokens: a token's ids in order, its teacher's probability and the logarithm of it for each, the student's logit, how many there
  // are; which of them lie in each granule
  int32_t *id;          // [tokens][K]
  float2 *p;            // [tokens][K]
  float *z;             // [tokens][K]
  int32_t *listed;      // [tokens]
  uint32_t *table;      // [tokens][granules]
  TokenOrder order;
  bool ordered;
  size_t bytes;
  DistillWs(const mhcl_ends_desc &d, int32_t K, bool grad, void *ws) : head(d, grad, ws, grad && TokenOrder::pays(d, kOrderDistill)) {
    WsCursor c(ws ? static_cast<char *>(ws) + head.bytes : nullptr);
    const size_t T = static_cast<size_t>(head.plan.tokens), slots = T * static_cast<size_t>(K);
    mark = c.take<int32_t>(static_cast<size_t>(d.T));
    id = c.take<int32_t>(slots);
    p = c.take<float2>(slots);
    z = c.take<float>(slots);
    listed = c.take<int32_t>(T);
    table = c.take<uint32_t>(T * static_cast<size_t>(head.plan.granules));
    ordered = grad && TokenOrder::pays(d, kOrderDistill);
    if (ordered) order.take(c, d, head);
    bytes = head.bytes + c.off;
  }
};
// total may be null; g_h, g_W null: the loss alone
hipError_t launch_distill(const mhcl_ends_desc &d, int32_t K, float temperature, const void *h, const void *W, const void *ids, const float *logits,
                          const float *weight, float *loss, float *lse, float *total, void *g_h, void *g_W, bool unrounded, const DistillWs &w,
                          hipStream_t s);

hipError_t launch_scale(void *p, int dtype, int64_t count, const float *factor, hipStream_t s);
hipError_t launch_scale_to(const float *in, void *out, int dtype, int64_t count, const float *factor, hipStream_t s);

}  // namespace mhcl
