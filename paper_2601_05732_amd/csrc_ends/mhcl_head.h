// Host-side declarations of the head's softmax cross entropy (mhcl_head.hip).
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
  HeadPlan(const mhcl_ends_desc &d, bool grad);
};

struct HeadWs {
  HeadPlan plan;
  char *hp;             // [tokens][C]: h, zeros where a token does not count
  char *E;              // [tokens][ld] numerators in 16 bits, then g in bf16 in their place; fp32: 32 bits each
  float2 *stat;         // [tokens][granules] maximum and sum
  float *zt;            // [tokens] the targets' logits
  float *common;        // [1] what all weights are multiples of
  float *slabs;         // [gh_splits][tokens][C]
  float *gw_slabs;      // [gw_splits][V][C]
  float *gW;            // [V][C] sums over blocks of tokens
  size_t bytes;
  HeadWs(const mhcl_ends_desc &d, bool grad, void *ws);
};

// g_h, g_W null: the loss alone.  weight null: that of the mean.  unrounded: g_h and g_W are fp32, whatever the operands.
hipError_t launch_head(const mhcl_ends_desc &d, const void *h, const void *W, const void *targets, const float *weight,
                       float *loss, float *lse, void *g_h, void *g_W, bool unrounded, const HeadWs &w, hipStream_t s);

hipError_t launch_head_total(const mhcl_ends_desc &d, const void *targets, const float *loss, const float *weight, float *total,
                             hipStream_t s);
hipError_t launch_scale(void *p, int dtype, int64_t count, const float *factor, hipStream_t s);
hipError_t launch_scale_to(const float *in, void *out, int dtype, int64_t count, const float *factor, hipStream_t s);

}  // namespace mhcl
