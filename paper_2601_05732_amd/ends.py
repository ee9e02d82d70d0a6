"""The two ends of a language model around a stack of hyper-connection layers: token embedding into the streams, the norm of
the streams' sum, and the head's softmax cross entropy, each with its gradients.

The functions here allocate the results and make one call into ``libmhcl.so`` (``mhcl_embed`` and so on; include/mhcl.h has
the formulas), which computes everything.  Tensors may be strided or at any address: what the library cannot read as it is
gets copied first.
"""
from __future__ import annotations

import torch

from . import binding as mhcl
from .layer import PHASE_G_X, PHASE_X, empty_stream


def _dense(t: torch.Tensor) -> torch.Tensor:
    """`t` contiguous and 16-byte aligned, as the kernels read it."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _same_device(*tensors):
    """The calls run on the current device's stream: the tensors have to lie on that device."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and (not t.is_cuda or t.device.index != device):
            raise ValueError(f"tensors must lie on the current GPU (cuda:{device}), got {t.device}")


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def embed_tokens(table: torch.Tensor, ids: torch.Tensor, n: int, scale: float = 1.0, dtype=None) -> torch.Tensor:
    """``x [T, n, C]`` with ``x[t, i] = scale * table[ids[t]]`` for every stream i, in `dtype` (default: the table's);
    zeros where ``ids[t]`` is negative, NaN where it is V or more.  table [V, C], ids [T] int64 or int32."""
    _same_device(table, ids)
    _need(table.dim() == 2 and ids.dim() == 1, f"table [V, C] and ids [T], got {tuple(table.shape)} and {tuple(ids.shape)}")
    V, C = table.shape
    T = ids.shape[0]
    d = mhcl.EndsDesc(C, T, n, V, dtype or table.dtype, table.dtype, ids.dtype, scale)
    x = empty_stream((T, n, C), d.io, table.device, PHASE_X)
    mhcl.mhcl_embed(d, _dense(table), ids.contiguous(), x)
    return x


def embed_tokens_grad(ids: torch.Tensor, g_x: torch.Tensor, V: int, scale: float = 1.0, dtype=None, into=None) -> torch.Tensor:
    """The gradient [V, C] on `embed_tokens`' table, in `dtype` (default: that of g_x [T, n, C]).  into: a tensor [V, C] that
    it is added to (and that is returned) instead."""
    _same_device(ids, g_x, into)
    _need(g_x.dim() == 3 and ids.shape == g_x.shape[:1], f"ids [T] and g_x [T, n, C], got {tuple(ids.shape)} and {tuple(g_x.shape)}")
    T, n, C = g_x.shape
    w = into.dtype if into is not None else dtype or g_x.dtype
    d = mhcl.EndsDesc(C, T, n, V, g_x.dtype, w, ids.dtype, scale)
    g_table = into if into is not None else torch.empty(V, C, device=g_x.device, dtype=w)
    ws = mhcl.new_ends_workspace(d, mhcl.OP_EMBED_BWD, g_x.device)
    mhcl.mhcl_embed_bwd(d, ids.contiguous(), _dense(g_x), g_table, into is not None, ws)
    return g_table


def _norm_desc(x, gain, eps):
    _need(x.dim() == 3 and gain.shape == x.shape[2:], f"x [T, n, C] and gain [C], got {tuple(x.shape)} and {tuple(gain.shape)}")
    T, n, C = x.shape
    return mhcl.EndsDesc(C, T, n, io=x.dtype, eps=eps)


def streams_norm(x: torch.Tensor, gain: torch.Tensor, eps: float = 1e-6) -> torch.Tensor:
    """``h [T, C] = gain * s / sqrt(mean(s^2) + eps)`` of the sum s of the streams of x [T, n, C]; gain [C] fp32."""
    _same_device(x, gain)
    d = _norm_desc(x, gain, eps)
    h = torch.empty(d.T, d.C, device=x.device, dtype=x.dtype)
    mhcl.mhcl_streams_norm(d, _dense(x), _dense(gain), h)
    return h


def streams_norm_grad(x: torch.Tensor, gain: torch.Tensor, g_h: torch.Tensor, eps: float = 1e-6):
    """``g_x [T, n, C], g_gain [C]`` of `streams_norm` for the gradient g_h [T, C] on its result."""
    _same_device(x, gain, g_h)
    d = _norm_desc(x, gain, eps)
    g_x = empty_stream(x.shape, x.dtype, x.device, PHASE_G_X)
    g_gain = torch.empty(d.C, device=x.device, dtype=torch.float32)
    ws = mhcl.new_ends_workspace(d, mhcl.OP_STREAMS_NORM_BWD, x.device)
    mhcl.mhcl_streams_norm_bwd(d, _dense(x), _dense(gain), _dense(g_h), g_x, g_gain, ws)
    return g_x, g_gain


def _head_desc(h, W, targets):
    _need(h.dim() == 2 and W.dim() == 2 and W.shape[1] == h.shape[1] and targets.shape == h.shape[:1],
          f"h [T, C], W [V, C] and targets [T], got {tuple(h.shape)}, {tuple(W.shape)} and {tuple(targets.shape)}")
    return mhcl.EndsDesc(h.shape[1], h.shape[0], 1, W.shape[0], h.dtype, W.dtype, targets.dtype)


def head_loss(h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor):
    """``loss [T], lse [T]`` (fp32): the softmax cross entropy of the logits h W^T with the targets, 0 where a target is negative,
    and the logits' log-sum-exp.  h [T, C], W [V, C] of one type."""
    _same_device(h, W, targets)
    d = _head_desc(h, W, targets)
    loss, lse = (torch.empty(d.T, device=h.device, dtype=torch.float32) for _ in range(2))
    ws = mhcl.new_ends_workspace(d, mhcl.OP_HEAD_LOSS, h.device)
    mhcl.mhcl_head_loss(d, _dense(h), _dense(W), targets.contiguous(), loss, lse, ws)
    return loss, lse


def head_loss_grad(h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, weight=None):
    """``loss [T], lse [T], g_h [T, C], g_W [V, C]``: `head_loss` and the gradients of ``sum(weight * loss)``; weight [T] fp32,
    or None for the mean over the targets that are not negative."""
    _same_device(h, W, targets, weight)
    d = _head_desc(h, W, targets)
    loss, lse = (torch.empty(d.T, device=h.device, dtype=torch.float32) for _ in range(2))
    g_h, g_W = torch.empty_like(h, memory_format=torch.contiguous_format), torch.empty_like(W, memory_format=torch.contiguous_format)
    ws = mhcl.new_ends_workspace(d, mhcl.OP_HEAD_LOSS_GRAD, h.device)
    mhcl.mhcl_head_loss_grad(d, _dense(h), _dense(W), targets.contiguous(), None if weight is None else weight.contiguous(),
                             loss, lse, g_h, g_W, ws)
    return loss, lse, g_h, g_W
