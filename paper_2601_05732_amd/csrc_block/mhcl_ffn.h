// Host-side declarations of the gated feed-forward block (mhcl_ffn.hip).
#pragma once
#include "../csrc/mhcl_internal.h"
#include "../csrc_ends/mhcl_tiles.h"

namespace mhcl {

constexpr int64_t kFfnMostWeights = int64_t{1} << 28;   // H C: the halves of W_up lie less than 2^31 bytes apart

struct FfnPlan {
  bool wide;                                  // fp32 operands
  ProductTile up, down, act, gx, gup, gdown;
  int down_splits, gx_splits, gup_splits, gdown_splits;
  bool trio;                                  // the backward's three last products in one launch
  FfnPlan(const mhcl_ffn_desc &d, bool grad);
};

struct FfnWs {
  FfnPlan plan;
  char *a;              // [T][H] silu(gate) * up
  char *g_pre;          // [T][2 H] gradients on gate | up
  float *slabs, *up_slabs, *down_slabs;   // parts of the sums of y and g_x, g_W_up, g_W_down; one and the same where they come one after the other
  size_t bytes;
  FfnWs(const mhcl_ffn_desc &d, bool grad, void *ws);
};

// pre [T][2 H], may be null: gate | up
hipError_t launch_ffn(const mhcl_ffn_desc &d, const void *x, const void *W_up, const void *W_down, void *y, float *pre, const FfnWs &w, hipStream_t s);
// g_x, g_W_up, g_W_down: those that are null are not formed
hipError_t launch_ffn_grad(const mhcl_ffn_desc &d, const void *x, const void *W_up, const void *W_down, const float *pre, const void *g_y, void *g_x,
                           void *g_W_up, void *g_W_down, const FfnWs &w, hipStream_t s);

}  // namespace mhcl
