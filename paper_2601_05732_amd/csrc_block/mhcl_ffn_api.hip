// C ABI of the gated feed-forward block: validation, workspaces, dispatch.  See include/mhcl.h.
#include "../csrc_ends/mhcl_ends.h"
#include "mhcl_ffn.h"

using namespace mhcl;

namespace {

int check_ffn(const mhcl_ffn_desc *d) {
  if (!d) return MHCL_ERR_INVALID_ARG;
  if (d->C < 8 || d->C % 8 != 0 || d->H < 8 || d->H % 8 != 0 || d->T < 0) return MHCL_ERR_INVALID_ARG;
  if (d->io_dtype != MHCL_BF16 && d->io_dtype != MHCL_F32) return MHCL_ERR_INVALID_ARG;
  // a tile's rows reach over less than 2^31 bytes, and so does a row of W_up from its partner; tiles and 256-number pieces in 31 bits
  if (d->C > 32768 || d->H > 131072 || static_cast<int64_t>(d->H) * d->C > kFfnMostWeights || d->T > (int64_t{1} << 30)) return MHCL_ERR_UNSUPPORTED;
  const int64_t widest = d->C > d->H ? d->C : d->H;
  if (d->T * (widest / 4) / 256 > (int64_t{1} << 31) - 1) return MHCL_ERR_UNSUPPORTED;
  return MHCL_OK;
}
template <typename... P>
bool all16(P... p) {
  return ((p != nullptr && reinterpret_cast<uintptr_t>(p) % 16 == 0) && ...);
}

bool none_or16(const void *p) { return p == nullptr || all16(p); }

#define MHCL_HIP(expr)                              \
  do {                                              \
    if ((expr) != hipSuccess) return MHCL_ERR_HIP;  \
  } while (0)

// mhcl_ffn_grad and mhcl_ffn_grad_of, which has seen to it that of g_x, g_W_up and g_W_down those are there that have to be
int ffn_grad(const mhcl_ffn_desc *desc, const void *x, const void *W_up, const void *W_down, const float *pre, const void *g_y, void *g_x,
             void *g_W_up, void *g_W_down, void *ws, size_t ws_bytes, hipStream_t s) {
  if (desc->T == 0) {
    const size_t half = static_cast<size_t>(desc->H) * desc->C * dtype_bytes(desc->io_dtype);
    if (g_W_up) MHCL_HIP(launch_zero(g_W_up, 2 * half, s));
    if (g_W_down) MHCL_HIP(launch_zero(g_W_down, half, s));
    return MHCL_OK;
  }
  if (!all16(x, W_up, W_down, (const void *)pre, g_y)) return MHCL_ERR_INVALID_ARG;
  if (!all16(ws) || ws_bytes < mhcl_ffn_workspace_bytes(desc, MHCL_OP_FFN_GRAD)) return MHCL_ERR_WORKSPACE;
  MHCL_HIP(launch_ffn_grad(*desc, x, W_up, W_down, pre, g_y, g_x, g_W_up, g_W_down, FfnWs(*desc, true, ws), s));
  return MHCL_OK;
}

}  // namespace

extern "C" {

size_t mhcl_ffn_workspace_bytes(const mhcl_ffn_desc *desc, int op) {
  if (op != MHCL_OP_FFN && op != MHCL_OP_FFN_GRAD) return 0;
  return check_ffn(desc) ? 0 : align_up(FfnWs(*desc, op == MHCL_OP_FFN_GRAD, nullptr).bytes + 1);
}

int mhcl_ffn(const mhcl_ffn_desc *desc, const void *x, const void *W_up, const void *W_down, void *y, float *pre, void *ws, size_t ws_bytes,
             void *stream) {
  if (int e = check_ffn(desc)) return e;
  if (desc->T == 0) return MHCL_OK;
  if (!all16(x, W_up, W_down, (const void *)y) || (pre && !all16((const void *)pre))) return MHCL_ERR_INVALID_ARG;
  if (!all16(ws) || ws_bytes < mhcl_ffn_workspace_bytes(desc, MHCL_OP_FFN)) return MHCL_ERR_WORKSPACE;
  MHCL_HIP(launch_ffn(*desc, x, W_up, W_down, y, pre, FfnWs(*desc, false, ws), static_cast<hipStream_t>(stream)));
  return MHCL_OK;
}

int mhcl_ffn_grad(const mhcl_ffn_desc *desc, const void *x, const void *W_up, const void *W_down, const float *pre, const void *g_y, void *g_x,
                  void *g_W_up, void *g_W_down, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_ffn(desc)) return e;
  if (!all16(g_W_up, g_W_down) || (desc->T > 0 && !all16((const void *)g_x))) return MHCL_ERR_INVALID_ARG;
  return ffn_grad(desc, x, W_up, W_down, pre, g_y, g_x, g_W_up, g_W_down, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

int mhcl_ffn_grad_of(const mhcl_ffn_desc *desc, const void *x, const void *W_up, const void *W_down, const float *pre, const void *g_y, void *g_x,
                     void *g_W_up, void *g_W_down, void *ws, size_t ws_bytes, void *stream) {
  if (int e = check_ffn(desc)) return e;
  if (!none_or16(g_x) || !none_or16(g_W_up) || !none_or16(g_W_down) || (desc->T > 0 && !g_x && !g_W_up && !g_W_down))
    return MHCL_ERR_INVALID_ARG;
  return ffn_grad(desc, x, W_up, W_down, pre, g_y, g_x, g_W_up, g_W_down, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

}  // extern "C"
