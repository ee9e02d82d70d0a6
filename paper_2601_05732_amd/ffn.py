"""The gated feed-forward block between the layers, ``y = (silu(x Wg^T) * (x Wu^T)) W_down^T``, with its gradients.

As in :mod:`.ends`: the functions allocate the results and make one call into ``libmhcl.so`` (``mhcl_ffn``, ``mhcl_ffn_grad_of``; include/mhcl.h
has the formulas), through the extension in C++ where the library can read the tensors as they are; others are copied first.
:class:`GatedFeedForward` is the same under ``torch.autograd``: first derivatives; second ones and forward-mode tangents are refused.
"""
from __future__ import annotations

import functools

import torch

from . import binding as mhcl
from .autograd import _native, first_only
from .ends import _dense, _need, _same_device


def _desc(x, W_up, W_down):
    _need(x.dim() == 2 and W_up.dim() == 2 and W_down.dim() == 2 and W_down.shape[0] == x.shape[1]
          and W_up.shape == (2 * W_down.shape[1], x.shape[1]),
          f"x [T, C], W_up [2 H, C] and W_down [C, H], got {tuple(x.shape)}, {tuple(W_up.shape)} and {tuple(W_down.shape)}")
    return mhcl.FfnDesc(x.shape[1], W_down.shape[1], x.shape[0], x.dtype)


def gated_ffn(x: torch.Tensor, W_up: torch.Tensor, W_down: torch.Tensor, keep: bool = False):
    """``y [T, C] = (silu(x Wg^T) * (x Wu^T)) W_down^T`` of x [T, C], W_up [2 H, C] (Wg is its first half of rows, Wu the other) and
    W_down [C, H], all of one type.  keep: ``y, kept`` with what `gated_ffn_grad` needs besides the operands, x W_up^T [T, 2 H] in
    fp32."""
    native = _native()
    if native is not None and (out := native.ffn(x, W_up, W_down, keep)) is not None:
        return out if keep else out[0]
    _same_device(x, W_up, W_down)
    d = _desc(x, W_up, W_down)
    y = torch.empty(d.T, d.C, device=x.device, dtype=x.dtype)
    kept = torch.empty(d.T, 2 * d.H, device=x.device, dtype=torch.float32) if keep else None
    ws = mhcl.new_ffn_workspace(d, mhcl.OP_FFN, x.device)
    mhcl.mhcl_ffn(d, _dense(x), _dense(W_up), _dense(W_down), y, kept, ws)
    return (y, kept) if keep else y


def gated_ffn_grad(x: torch.Tensor, W_up: torch.Tensor, W_down: torch.Tensor, kept: torch.Tensor, g_y: torch.Tensor, wanted=(True, True, True)):
    """``g_x [T, C], g_W_up [2 H, C], g_W_down [C, H]`` of `gated_ffn` for the gradient g_y [T, C] on its result; `kept` as it gave it.
    wanted: which of the three (one at least); those that are not wanted are None, and their products are left out."""
    wanted = tuple(bool(w) for w in wanted)
    _need(len(wanted) == 3 and any(wanted), f"wanted: which of the three gradients, got {wanted}")
    native = _native()
    if native is not None and (g := native.ffn_grad(x, W_up, W_down, kept, g_y, *wanted)) is not None:
        return g
    _same_device(x, W_up, W_down, kept, g_y)
    d = _desc(x, W_up, W_down)
    g_x, g_W_up, g_W_down = (torch.empty(t.shape, device=t.device, dtype=t.dtype) if w else None for t, w in zip((x, W_up, W_down), wanted))
    ws = mhcl.new_ffn_workspace(d, mhcl.OP_FFN_GRAD, x.device)
    mhcl.mhcl_ffn_grad_of(d, _dense(x), _dense(W_up), _dense(W_down), _dense(kept), _dense(g_y), g_x, g_W_up, g_W_down, ws)
    return g_x, g_W_up, g_W_down


@functools.lru_cache(maxsize=64)
def takes(C: int, H: int, dtype) -> bool:
    """Whether the block's kernels take these widths and this type."""
    return dtype in (torch.bfloat16, torch.float32) and mhcl.ffn_workspace_bytes(mhcl.FfnDesc(C, H, 1, dtype), mhcl.OP_FFN) > 0


class _Ffn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W_up, W_down, record):
        if not (record and any(ctx.needs_input_grad)):
            return gated_ffn(x, W_up, W_down)
        y, kept = gated_ffn(x, W_up, W_down, keep=True)
        ctx.save_for_backward(x, W_up, W_down, kept)
        return y

    @staticmethod
    def backward(ctx, g_y):
        x, W_up, W_down, kept = ctx.saved_tensors
        grads = gated_ffn_grad(x, W_up, W_down, kept, g_y, ctx.needs_input_grad[:3])      # (frozen weights need no products)
        return *first_only("the feed-forward block", grads, x, W_up, W_down, g_y), None


def apply_gated_ffn(x, W_up, W_down):
    """`gated_ffn` of rows x [..., C] under autograd."""
    y = _Ffn.apply(x.reshape(-1, x.shape[-1]), W_up, W_down, torch.is_grad_enabled())
    return y.view(x.shape)


class GatedFeedForward(torch.nn.Module):
    """Rows x [..., C] to rows of the same shape through H hidden numbers; W_up [2 H, C], W_down [C, H]."""

    def __init__(self, C: int, hidden: int, dtype=torch.bfloat16, std: float = 0.02, device="cuda"):
        super().__init__()
        self.W_up = torch.nn.Parameter(torch.empty(2 * hidden, C, device=device, dtype=dtype).normal_(0.0, std))
        self.W_down = torch.nn.Parameter(torch.empty(C, hidden, device=device, dtype=dtype).normal_(0.0, std))

    def forward(self, x):
        return apply_gated_ffn(x, self.W_up, self.W_down)
