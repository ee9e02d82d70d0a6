// C ABI of the two ends of a language model: validation, workspaces, dispatch.  See include/mhcl.h.
#include <math.h>

#include "mhcl_ends.h"
#include "mhcl_head.h"

using namespace mhcl;

namespace {

bool dtype_ok(int dtype) { return dtype == MHCL_BF16 || dtype == MHCL_F32; }

bool aligned(const void *p, size_t a) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % a == 0; }
template <typename... P>
bool all16(P... p) {
  return (aligned(p, 16) && ...);
}
bool ids_ok(const mhcl_ends_desc &d, const void *ids) { return aligned(ids, d.id_dtype == MHCL_I64 ? 8 : 4); }

enum class End { kEmbed, kNorm, kHead };

int check_ends(const mhcl_ends_desc *d, End end) {
  if (!d) return MHCL_ERR_INVALID_ARG;
  if (d->C < 8 || d->C % 8 != 0 || d->T < 0 || !dtype_ok(d->io_dtype)) return MHCL_ERR_INVALID_ARG;
  if (end != End::kHead && (d->n < 1 || d->n > 8)) return MHCL_ERR_INVALID_ARG;
  if (end != End::kNorm) {
    if (d->V < 1 || !dtype_ok(d->w_dtype)) return MHCL_ERR_INVALID_ARG;
    if (d->id_dtype != MHCL_I64 && d->id_dtype != MHCL_I32) return MHCL_ERR_INVALID_ARG;
  }
  if (end == End::kEmbed && !isfinite(d->scale)) return MHCL_ERR_INVALID_ARG;
  if (end == End::kNorm && !(d->eps >= 0.f)) return MHCL_ERR_INVALID_ARG;
  if (end == End::kHead && d->w_dtype != d->io_dtype) return MHCL_ERR_UNSUPPORTED;
  // index arithmetic: tokens and rows of the vocabulary in 32 bits, with room for a sentinel; at most 2^31 - 1 blocks a launch
  if (d->C > 32768 || d->T > (1 << 30)) return MHCL_ERR_UNSUPPORTED;
  if (end != End::kNorm && d->V > (1 << 30)) return MHCL_ERR_UNSUPPORTED;
  // (the head's products reach over 256 rows of numerators, 128 of fp32, by 31-bit offsets in bytes)
  if (end == End::kHead && d->V > kHeadMostRows) return MHCL_ERR_UNSUPPORTED;
  if (d->T * (d->C / 4) / 256 > (int64_t{1} << 31) - 1) return MHCL_ERR_UNSUPPORTED;
  return MHCL_OK;
}

#define MHCL_HIP(expr)                              \
  do {                                              \
    if ((expr) != hipSuccess) return MHCL_ERR_HIP;  \
  } while (0)

// mhcl_head_loss_grad and its unrounded form
int head_loss_grad(const mhcl_ends_desc *desc, const void *h, const void *W, const void *targets, const float *weight, float *loss,
                   float *lse, void *g_h, void *g_W, bool unrounded, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_ends(desc, End::kHead)) return e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!all16(g_W)) return MHCL_ERR_INVALID_ARG;
  if (desc->T == 0) {
    MHCL_HIP(launch_zero(g_W, static_cast<size_t>(desc->V) * desc->C * (unrounded ? 4 : dtype_bytes(desc->w_dtype)), s));
    return MHCL_OK;
  }
  if (!all16(h, W, (const void *)g_h) || !ids_ok(*desc, targets) || !aligned(loss, 4) || !aligned(lse, 4) ||
      (weight && !aligned(weight, 4)))
    return MHCL_ERR_INVALID_ARG;
  if (!all16(ws) || ws_bytes < mhcl_ends_workspace_bytes(desc, MHCL_OP_HEAD_LOSS_GRAD)) return MHCL_ERR_WORKSPACE;
  MHCL_HIP(launch_head(*desc, h, W, targets, weight, loss, lse, g_h, g_W, unrounded, HeadWs(*desc, true, ws), s));
  return MHCL_OK;
}

}  // namespace

extern "C" {

size_t mhcl_ends_workspace_bytes(const mhcl_ends_desc *desc, int op) {
  switch (op) {
    case MHCL_OP_EMBED_BWD:
      return check_ends(desc, End::kEmbed) ? 0 : align_up(EmbedBwdWs(*desc, nullptr).bytes + 1);
    case MHCL_OP_STREAMS_NORM_BWD:
      return check_ends(desc, End::kNorm) ? 0 : norm_bwd_ws_bytes(*desc);
    case MHCL_OP_HEAD_LOSS:
    case MHCL_OP_HEAD_LOSS_GRAD:
      return check_ends(desc, End::kHead) ? 0 : align_up(HeadWs(*desc, op == MHCL_OP_HEAD_LOSS_GRAD, nullptr).bytes + 1);
  }
  return 0;
}

int mhcl_embed(const mhcl_ends_desc *desc, const void *table, const void *ids, void *x, void *stream) {
  if (int e = check_ends(desc, End::kEmbed)) return e;
  if (desc->T == 0) return MHCL_OK;   // per-token tensors may then be null
  if (!all16(table, x) || !ids_ok(*desc, ids)) return MHCL_ERR_INVALID_ARG;
  MHCL_HIP(launch_embed(*desc, table, ids, x, static_cast<hipStream_t>(stream)));
  return MHCL_OK;
}

int mhcl_embed_bwd(const mhcl_ends_desc *desc, const void *ids, const void *g_x, void *g_table, int accumulate, void *ws,
                   size_t ws_bytes, void *stream) {
  if (int e = check_ends(desc, End::kEmbed)) return e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!all16(g_table)) return MHCL_ERR_INVALID_ARG;
  if (desc->T == 0) {
    if (!accumulate) MHCL_HIP(launch_zero(g_table, static_cast<size_t>(desc->V) * desc->C * dtype_bytes(desc->w_dtype), s));
    return MHCL_OK;
  }
  if (!all16(g_x) || !ids_ok(*desc, ids)) return MHCL_ERR_INVALID_ARG;
  if (!all16(ws) || ws_bytes < mhcl_ends_workspace_bytes(desc, MHCL_OP_EMBED_BWD)) return MHCL_ERR_WORKSPACE;
  MHCL_HIP(launch_embed_bwd(*desc, ids, g_x, g_table, accumulate != 0, EmbedBwdWs(*desc, ws), s));
  return MHCL_OK;
}

int mhcl_streams_norm(const mhcl_ends_desc *desc, const void *x, const float *gain, void *h, void *stream) {
  if (int e = check_ends(desc, End::kNorm)) return e;
  if (desc->T == 0) return MHCL_OK;
  if (!all16(x, (const void *)gain, h)) return MHCL_ERR_INVALID_ARG;
  MHCL_HIP(launch_streams_norm(*desc, x, gain, h, static_cast<hipStream_t>(stream)));
  return MHCL_OK;
}

int mhcl_streams_norm_bwd(const mhcl_ends_desc *desc, const void *x, const float *gain, const void *g_h, void *g_x,
                          float *g_gain, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_ends(desc, End::kNorm)) return e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!all16((const void *)g_gain)) return MHCL_ERR_INVALID_ARG;
  if (desc->T == 0) {
    MHCL_HIP(launch_zero(g_gain, static_cast<size_t>(desc->C) * 4, s));
    return MHCL_OK;
  }
  if (!all16(x, (const void *)gain, g_h, g_x)) return MHCL_ERR_INVALID_ARG;
  if (!all16(ws) || ws_bytes < mhcl_ends_workspace_bytes(desc, MHCL_OP_STREAMS_NORM_BWD)) return MHCL_ERR_WORKSPACE;
  MHCL_HIP(launch_streams_norm_bwd(*desc, x, gain, g_h, g_x, g_gain, static_cast<float *>(ws), s));
  return MHCL_OK;
}

int mhcl_head_loss(const mhcl_ends_desc *desc, const void *h, const void *W, const void *targets, float *loss, float *lse,
                   void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_ends(desc, End::kHead)) return e;
  if (desc->T == 0) return MHCL_OK;
  if (!all16(h, W) || !ids_ok(*desc, targets) || !aligned(loss, 4) || !aligned(lse, 4)) return MHCL_ERR_INVALID_ARG;
  if (!all16(ws) || ws_bytes < mhcl_ends_workspace_bytes(desc, MHCL_OP_HEAD_LOSS)) return MHCL_ERR_WORKSPACE;
  MHCL_HIP(launch_head(*desc, h, W, targets, nullptr, loss, lse, nullptr, nullptr, false, HeadWs(*desc, false, ws),
                       static_cast<hipStream_t>(stream)));
  return MHCL_OK;
}

int mhcl_head_loss_grad(const mhcl_ends_desc *desc, const void *h, const void *W, const void *targets, const float *weight,
                        float *loss, float *lse, void *g_h, void *g_W, void *ws, size_t ws_bytes, void *stream) {
  return head_loss_grad(desc, h, W, targets, weight, loss, lse, g_h, g_W, false, ws, ws_bytes, stream);
}

int mhcl_head_loss_grad_unrounded(const mhcl_ends_desc *desc, const void *h, const void *W, const void *targets, const float *weight,
                                  float *loss, float *lse, float *g_h, float *g_W, void *ws, size_t ws_bytes, void *stream) {
  return head_loss_grad(desc, h, W, targets, weight, loss, lse, g_h, g_W, true, ws, ws_bytes, stream);
}

int mhcl_head_total(const mhcl_ends_desc *desc, const void *targets, const float *loss, const float *weight, float *total,
                    void *stream) {
  if (int e = check_ends(desc, End::kHead)) return e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!aligned(total, 4)) return MHCL_ERR_INVALID_ARG;
  if (desc->T == 0) {
    MHCL_HIP(launch_zero(total, 4, s));
    return MHCL_OK;
  }
  if (!ids_ok(*desc, targets) || !aligned(loss, 4) || (weight && !aligned(weight, 4))) return MHCL_ERR_INVALID_ARG;
  MHCL_HIP(launch_head_total(*desc, targets, loss, weight, total, s));
  return MHCL_OK;
}

size_t mhcl_head_distill_workspace_bytes(const mhcl_ends_desc *desc, int32_t K, int grad) {
  if (K < 1 || K > kMostSlots || check_ends(desc, End::kHead)) return 0;
  return align_up(DistillWs(*desc, K, grad != 0, nullptr).bytes + 1);
}

int mhcl_head_distill(const mhcl_ends_desc *desc, int32_t K, float temperature, const void *h, const void *W, const void *ids, const float *logits,
                      const float *weight, float *loss, float *lse, float *total, void *g_h, void *g_W, int unrounded, void *ws, size_t ws_bytes,
                      void *stream) {
  if (int e = check_ends(desc, End::kHead)) return e;
  if (K < 1 || !(temperature >= 1e-6f && temperature <= 1e6f)) return MHCL_ERR_INVALID_ARG;
  if (K > kMostSlots) return MHCL_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool grad = g_W != nullptr;
  if ((grad && !all16((const void *)g_W)) || (total && !aligned(total, 4))) return MHCL_ERR_INVALID_ARG;
  if (desc->T == 0) {
    if (g_h && !grad) return MHCL_ERR_INVALID_ARG;
    if (grad) MHCL_HIP(launch_zero(g_W, static_cast<size_t>(desc->V) * desc->C * (unrounded ? 4 : dtype_bytes(desc->w_dtype)), s));
    if (total) MHCL_HIP(launch_zero(total, 4, s));
    return MHCL_OK;
  }
  if (!all16(h, W) || !ids_ok(*desc, ids) || !aligned(logits, 4) || !aligned(loss, 4) || !aligned(lse, 4) || (weight && !aligned(weight, 4)) ||
      (g_h != nullptr) != grad || (grad && !all16((const void *)g_h)))
    return MHCL_ERR_INVALID_ARG;
  if (!all16(ws) || ws_bytes < mhcl_head_distill_workspace_bytes(desc, K, grad)) return MHCL_ERR_WORKSPACE;
  MHCL_HIP(launch_distill(*desc, K, temperature, h, W, ids, logits, weight, loss, lse, total, g_h, g_W, unrounded != 0, DistillWs(*desc, K, grad, ws), s));
  return MHCL_OK;
}

size_t mhcl_head_preference_workspace_bytes(const mhcl_ends_desc *desc, int grad) {
  return check_ends(desc, End::kHead) ? 0 : align_up(PreferenceWs(*desc, grad != 0, nullptr).bytes + 1);
}

int mhcl_head_preference(const mhcl_ends_desc *desc, int32_t pairs, float beta, float smoothing, const void *h, const void *W, const void *targets,
                         const void *offsets, int offset_dtype, const float *reference, const float *weight, float *loss, float *logp, float *total,
                         void *g_h, void *g_W, int unrounded, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_ends(desc, End::kHead)) return e;
  if (pairs < 0 || !isfinite(beta) || !(smoothing >= 0.f && smoothing <= 1.f)) return MHCL_ERR_INVALID_ARG;
  if (offset_dtype != MHCL_I64 && offset_dtype != MHCL_I32) return MHCL_ERR_INVALID_ARG;
  if (pairs > kMostPairs) return MHCL_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool grad = g_W != nullptr;
  if ((grad && !all16((const void *)g_W)) || (total && !aligned(total, 4)) || (g_h && !grad) || (weight && !aligned(weight, 4))) return MHCL_ERR_INVALID_ARG;
  if (pairs > 0 && (!aligned(offsets, offset_dtype == MHCL_I64 ? 8 : 4) || !aligned(loss, 4) || !aligned(logp, 4) || (reference && !aligned(reference, 4))))
    return MHCL_ERR_INVALID_ARG;
  if (desc->T > 0) {
    if (!all16(h, W) || !ids_ok(*desc, targets) || (grad && !all16((const void *)g_h))) return MHCL_ERR_INVALID_ARG;
    if (!all16(ws) || ws_bytes < mhcl_head_preference_workspace_bytes(desc, grad)) return MHCL_ERR_WORKSPACE;
  } else if (grad) {
    MHCL_HIP(launch_zero(g_W, static_cast<size_t>(desc->V) * desc->C * (unrounded ? 4 : dtype_bytes(desc->w_dtype)), s));
  }
  PairArgs a{};
  a.reference = reference;
  a.weight = weight;
  a.loss = loss;
  a.logp = logp;
  a.T = desc->T;
  a.pairs = pairs;
  a.beta = beta;
  a.smoothing = smoothing;
  MHCL_HIP(launch_preference(*desc, h, W, targets, offsets, offset_dtype, a, g_h, g_W, unrounded != 0, PreferenceWs(*desc, grad, ws), s));
  if (!total) return MHCL_OK;
  if (pairs == 0) {
    MHCL_HIP(launch_zero(total, 4, s));
    return MHCL_OK;
  }
  mhcl_ends_desc all = *desc;
  all.T = pairs;
  MHCL_HIP(launch_head_total(all, nullptr, loss, weight, total, s));
  return MHCL_OK;
}

int mhcl_scale(void *p, int dtype, int64_t count, const float *factor, void *stream) {
  if (!dtype_ok(dtype) || count < 0 || !aligned(factor, 4)) return MHCL_ERR_INVALID_ARG;
  if (count == 0) return MHCL_OK;
  if (!all16(p)) return MHCL_ERR_INVALID_ARG;
  MHCL_HIP(launch_scale(p, dtype, count, factor, static_cast<hipStream_t>(stream)));
  return MHCL_OK;
}

int mhcl_scale_to(const float *in, void *out, int dtype, int64_t count, const float *factor, void *stream) {
  if (!dtype_ok(dtype) || count < 0 || !aligned(factor, 4)) return MHCL_ERR_INVALID_ARG;
  if (count == 0) return MHCL_OK;
  if (!all16((const void *)in, out)) return MHCL_ERR_INVALID_ARG;
  MHCL_HIP(launch_scale_to(in, out, dtype, count, factor, static_cast<hipStream_t>(stream)));
  return MHCL_OK;
}

}  // extern "C"
