"""The two ends of a language model around a stack of hyper-connection layers: token embedding into the streams, the norm of
the streams' sum, and the head's softmax cross entropy, each with its gradients; and what the head learns from besides next tokens, a teacher's
likeliest ones and pairs of sequences.

The functions here allocate the results and make one call into ``libmhcl.so`` (``mhcl_embed`` and so on; include/mhcl.h has
the formulas), which computes everything.  Tensors may be strided or at any address: what the library cannot read as it is
gets copied first.  Calls with tensors that it can read go through the extension in C++ (``torch_ext/ends.cpp``: the same at less
than half of the host time), where that is built.

:class:`TokenEmbedding`, :class:`StreamsNorm` and :class:`Head` are the same under ``torch.autograd``: first derivatives; second ones and
forward-mode tangents are refused.
"""
from __future__ import annotations

import torch

from . import binding as mhcl
from .autograd import _native, first_only
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
    native = _native()
    if native is not None and (x := native.embed(table, ids, n, scale, dtype or table.dtype)) is not None:
        return x
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
    native = _native()
    if native is not None and (g := native.embed_grad(ids, g_x, V, scale, dtype or g_x.dtype, into)) is not None:
        return g
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
    native = _native()
    if native is not None and (h := native.norm(x, gain, eps)) is not None:
        return h
    _same_device(x, gain)
    d = _norm_desc(x, gain, eps)
    h = torch.empty(d.T, d.C, device=x.device, dtype=x.dtype)
    mhcl.mhcl_streams_norm(d, _dense(x), _dense(gain), h)
    return h


def streams_norm_grad(x: torch.Tensor, gain: torch.Tensor, g_h: torch.Tensor, eps: float = 1e-6):
    """``g_x [T, n, C], g_gain [C]`` of `streams_norm` for the gradient g_h [T, C] on its result."""
    native = _native()
    if native is not None and (g := native.norm_grad(x, gain, g_h, eps)) is not None:
        return g
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
    native = _native()
    if native is not None and (out := native.head(h, W, targets)) is not None:
        return out
    _same_device(h, W, targets)
    d = _head_desc(h, W, targets)
    loss, lse = (torch.empty(d.T, device=h.device, dtype=torch.float32) for _ in range(2))
    ws = mhcl.new_ends_workspace(d, mhcl.OP_HEAD_LOSS, h.device)
    mhcl.mhcl_head_loss(d, _dense(h), _dense(W), targets.contiguous(), loss, lse, ws)
    return loss, lse


def head_loss_grad(h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, weight=None, dtype=None):
    """``loss [T], lse [T], g_h [T, C], g_W [V, C]``: `head_loss` and the gradients of ``sum(weight * loss)``; weight [T] fp32,
    or None for the mean over the targets that are not negative.  The gradients are of `dtype`: h's and W's type (the default), or
    float32, which holds their sums as they are."""
    dtype = dtype or h.dtype
    native = _native()
    if native is not None and (out := native.head_grad(h, W, targets, weight, dtype)) is not None:
        return out
    _same_device(h, W, targets, weight)
    d = _head_desc(h, W, targets)
    loss, lse = (torch.empty(d.T, device=h.device, dtype=torch.float32) for _ in range(2))
    _need(dtype in (h.dtype, torch.float32), f"gradients of {dtype}: {h.dtype} or float32")
    g_h, g_W = (torch.empty(t.shape, device=h.device, dtype=dtype if dtype is not h.dtype else t.dtype) for t in (h, W))
    ws = mhcl.new_ends_workspace(d, mhcl.OP_HEAD_LOSS_GRAD, h.device)
    mhcl.mhcl_head_loss_grad(d, _dense(h), _dense(W), targets.contiguous(), None if weight is None else weight.contiguous(),
                             loss, lse, g_h, g_W, ws)
    return loss, lse, g_h, g_W


def _constant(**tensors):
    """The losses below take these as they are: a gradient that somebody waits for on them would be missing."""
    for name, t in tensors.items():
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} is a constant of this loss: detach it")


def _distill(h, W, ids, logits, weight, temperature, dtype, grad, total):
    """``loss, lse, g_h, g_W, total``, with None for what is not asked for."""
    logits = logits.float() if logits.dtype in (torch.bfloat16, torch.float16) else logits
    native = _native()
    if native is not None and (out := native.distill(h, W, ids, logits, weight, temperature, dtype if grad else None, total)) is not None:
        return out
    _same_device(h, W, ids, logits, weight)
    _need(h.dim() == 2 and W.dim() == 2 and W.shape[1] == h.shape[1] and ids.dim() == 2 and ids.shape[0] == h.shape[0] and ids.shape == logits.shape,
          f"h [T, C], W [V, C], ids [T, K] and logits [T, K], got {tuple(h.shape)}, {tuple(W.shape)}, {tuple(ids.shape)} and {tuple(logits.shape)}")
    d = mhcl.EndsDesc(h.shape[1], h.shape[0], 1, W.shape[0], h.dtype, W.dtype, ids.dtype)
    loss, lse = (torch.empty(d.T, device=h.device, dtype=torch.float32) for _ in range(2))
    g_h, g_W = _head_grad_buffers(h, W, dtype, grad)
    sum_ = torch.empty(1, device=h.device, dtype=torch.float32) if total else None
    ws = torch.empty(mhcl.head_distill_workspace_bytes(d, ids.shape[1], grad), dtype=torch.uint8, device=h.device)
    mhcl.mhcl_head_distill(d, temperature, _dense(h), _dense(W), ids.contiguous(), logits.contiguous(), None if weight is None else weight.contiguous(),
                           loss, lse, sum_, g_h, g_W, ws)
    return loss, lse, g_h, g_W, sum_


def _head_grad_buffers(h, W, dtype, grad):
    if not grad:
        return None, None
    _need(dtype in (h.dtype, torch.float32), f"gradients of {dtype}: {h.dtype} or float32")
    return tuple(torch.empty(t.shape, device=h.device, dtype=dtype) for t in (h, W))


def head_distill(h: torch.Tensor, W: torch.Tensor, ids: torch.Tensor, logits: torch.Tensor, temperature: float = 1.0):
    """``loss [T], lse [T]`` (fp32): the head against a teacher's likeliest rows, the divergence sum_k p_k (log p_k - log q[ids[t, k]]) of q, the
    softmax of the logits h W^T / temperature, from p, that of the teacher's logits [T, K] / temperature over a token's slots; and the log-sum-exp of
    the former.  A slot is empty where ids [T, K] (int64 or int32) is negative or the logit -inf; a token without any does not count: its
    loss is 0.  h [T, C], W [V, C] of one type; the teacher's logits fp32, or of 16 bits (copied then); at most 256 slots."""
    return _distill(h, W, ids, logits, None, temperature, None, False, False)[:2]


def head_distill_grad(h: torch.Tensor, W: torch.Tensor, ids: torch.Tensor, logits: torch.Tensor, weight=None, temperature: float = 1.0, dtype=None):
    """``loss [T], lse [T], g_h [T, C], g_W [V, C]``: `head_distill` and the gradients of ``sum(weight * loss)``; weight [T] fp32, or None for the
    mean over the tokens that count.  dtype as in `head_loss_grad`."""
    return _distill(h, W, ids, logits, weight, temperature, dtype or h.dtype, True, False)[:4]


def _preference(h, W, targets, offsets, reference, weight, beta, smoothing, dtype, grad, total):
    """``loss, logp, g_h, g_W, total``, with None for what is not asked for."""
    native = _native()
    if native is not None and (out := native.preference(h, W, targets, offsets, reference, weight, beta, smoothing, dtype if grad else None,
                                                        total)) is not None:
        return out
    _same_device(h, W, targets, offsets, reference, weight)
    d = _head_desc(h, W, targets)
    _need(offsets.dim() == 1 and offsets.shape[0] % 2 == 1, f"offsets [2 P + 1] of P pairs, got {tuple(offsets.shape)}")
    pairs = offsets.shape[0] // 2
    loss, logp = (torch.empty(n, device=h.device, dtype=torch.float32) for n in (pairs, 2 * pairs))
    g_h, g_W = _head_grad_buffers(h, W, dtype, grad)
    sum_ = torch.empty(1, device=h.device, dtype=torch.float32) if total else None
    ws = torch.empty(mhcl.head_preference_workspace_bytes(d, grad), dtype=torch.uint8, device=h.device)
    mhcl.mhcl_head_preference(d, pairs, beta, smoothing, _dense(h), _dense(W), targets.contiguous(), offsets.contiguous(),
                              *(None if t is None else t.contiguous() for t in (reference, weight)), loss, logp, sum_, g_h, g_W, ws)
    return loss, logp, g_h, g_W, sum_


def head_preference(h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, offsets: torch.Tensor, reference=None, beta: float = 0.1,
                    smoothing: float = 0.0):
    """``loss [P], logp [2 P]`` (fp32) of P pairs of packed sequences, tokens offsets[s] to offsets[s + 1] - 1 being sequence s, the chosen ones
    even and the rejected ones odd: logp[s] is the sum of the log probabilities of its targets that are not negative, and

        loss[p] = (1 - smoothing) log(1 + exp(-m)) + smoothing log(1 + exp(m)),  m = beta ((logp - reference)[2 p] - (logp - reference)[2 p + 1])

    reference [2 P] fp32: those of a reference model (what this returns for it), or None for zeros.  offsets [2 P + 1] int64 or int32, ascending
    within 0..T (a pair whose are not has a loss of NaN); tokens outside of them add nothing.  h [T, C], W [V, C] of one type."""
    return _preference(h, W, targets, offsets, reference, None, beta, smoothing, None, False, False)[:2]


def head_preference_grad(h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, offsets: torch.Tensor, reference=None, weight=None,
                         beta: float = 0.1, smoothing: float = 0.0, dtype=None):
    """``loss [P], logp [2 P], g_h [T, C], g_W [V, C]``: `head_preference` and the gradients of ``sum(weight * loss)``; weight [P] fp32, or None for
    the mean over the pairs.  dtype as in `head_loss_grad`."""
    return _preference(h, W, targets, offsets, reference, weight, beta, smoothing, dtype or h.dtype, True, False)[:4]


# ---- under torch.autograd --------------------------------------------------------------------


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, n, scale, dtype):
        ctx.save_for_backward(ids)
        ctx.V, ctx.scale, ctx.dtype = table.shape[0], scale, table.dtype
        return embed_tokens(table, ids, n, scale, dtype)

    @staticmethod
    def backward(ctx, g_x):
        ids, = ctx.saved_tensors
        return *first_only("the embedding", (embed_tokens_grad(ids, g_x, ctx.V, ctx.scale, ctx.dtype),), g_x), None, None, None, None


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, eps):
        ctx.save_for_backward(x, gain)
        ctx.eps = eps
        return streams_norm(x, gain, eps)

    @staticmethod
    def backward(ctx, g_h):
        x, gain = ctx.saved_tensors
        return *first_only("the norm of the streams", streams_norm_grad(x, gain, g_h, ctx.eps), x, gain, g_h), None


class _HeadTotal(torch.autograd.Function):
    """The gradients are taken with the loss, for a gradient of 1 on it: the softmax's numerators, which both need, are formed
    once.  The backward multiplies them by what it gets.  Those of bf16 operands are kept as fp32 sums until then, so that a factor on the
    loss is in them before they are rounded (bf16 gradients times a factor that is no power of two are rounded twice); those of fp32
    operands are multiplied where they are, unless the factor is 1 (the device looks).  (us, forward and backward, 16384 tokens, C = 4096,
    65536 rows, with bf16 gradients kept and multiplied / this: 20800 / 21500; 333, 520, 1003 75 / 81.)"""

    @staticmethod
    def forward(ctx, h, W, targets, weight, record):
        if record and (ctx.needs_input_grad[0] or ctx.needs_input_grad[1]):
            loss, _, *grads = head_loss_grad(h, W, targets, weight, torch.float32)
        else:
            loss, grads = head_loss(h, W, targets)[0], [None, None]
        total = _total(h, W, targets, loss, weight)
        _keep_grads(ctx, h, W, weight, *grads, loss, record and ctx.needs_input_grad[3])
        return total

    @staticmethod
    def backward(ctx, g):
        g_h, g_W, g_weight = _kept_grads(ctx, g, "the head's loss")
        return g_h, g_W, None, g_weight, None


class _DistillTotal(torch.autograd.Function):
    """As _HeadTotal, of the loss against a teacher."""

    @staticmethod
    def forward(ctx, h, W, weight, ids, logits, temperature, record):
        grad = record and (ctx.needs_input_grad[0] or ctx.needs_input_grad[1])
        loss, _, g_h, g_W, total = _distill(h, W, ids, logits, weight, temperature, torch.float32, grad, True)
        _keep_grads(ctx, h, W, weight, g_h, g_W, loss, record and ctx.needs_input_grad[2])
        return total[0]

    @staticmethod
    def backward(ctx, g):
        return *_kept_grads(ctx, g, "the head's loss against a teacher", 2), None, None, None, None


class _PreferenceTotal(torch.autograd.Function):
    """As _HeadTotal, of the loss of pairs; and the sequences' log probabilities, as numbers."""

    @staticmethod
    def forward(ctx, h, W, weight, targets, offsets, reference, beta, smoothing, record):
        grad = record and (ctx.needs_input_grad[0] or ctx.needs_input_grad[1])
        loss, logp, g_h, g_W, total = _preference(h, W, targets, offsets, reference, weight, beta, smoothing, torch.float32, grad, True)
        _keep_grads(ctx, h, W, weight, g_h, g_W, loss, record and ctx.needs_input_grad[2])
        ctx.mark_non_differentiable(logp)
        return total[0], logp

    @staticmethod
    def backward(ctx, g, _):
        return *_kept_grads(ctx, g, "the head's loss of pairs", 2), None, None, None, None, None, None


def _keep_grads(ctx, h, W, weight, g_h, g_W, loss, weighed):
    """What _kept_grads multiplies: the gradients for a factor of 1."""
    ctx.save_for_backward(h, W, weight)     # (read by a recorded backward alone)
    # (a place of weight 0 adds nothing, whatever it holds)
    g_weight = loss.masked_fill((weight == 0) & ~loss.isfinite(), 0.0) if weighed else None
    ctx.grads, ctx.dtypes = [g_h, g_W, g_weight], (h.dtype, W.dtype, torch.float32)


def _kept_grads(ctx, g, what, weight_at=3):
    """g_h, g_W and g_weight of a loss whose gradients were taken with it, for the gradient g on it."""
    if ctx.grads is None:
        raise RuntimeError("the head's gradients went out with its first backward: run the head again for another one")
    grads, ctx.grads = ctx.grads, None
    needed = (*ctx.needs_input_grad[:2], ctx.needs_input_grad[weight_at])
    grads = tuple(_times(t, g, dtype) if need else None for t, dtype, need in zip(grads, ctx.dtypes, needed))
    if torch.is_grad_enabled():
        grads = first_only(what, grads, *ctx.saved_tensors, g)
    return grads


def _times(t, factor, dtype):
    """t (fp32, nobody else's) times a factor on the GPU, of `dtype`."""
    if dtype is torch.float32:
        mhcl.mhcl_scale(t, factor)
        return t
    out = torch.empty(t.shape, device=t.device, dtype=dtype)
    mhcl.mhcl_scale_to(t, factor, out)
    return out


def _total(h, W, targets, loss, weight):
    d = _head_desc(h, W, targets)
    total = torch.empty(1, device=h.device, dtype=torch.float32)
    mhcl.mhcl_head_total(d, targets.contiguous(), loss, None if weight is None else weight.contiguous(), total)
    return total[0]


class TokenEmbedding(torch.nn.Module):
    """Token ids [T] to the streams x [T, n, C] of the first layer; negative ids hold no token."""

    def __init__(self, V: int, C: int, n: int, scale: float = 1.0, dtype=torch.bfloat16, table_dtype=torch.float32,
                 std: float = 0.02, device="cuda"):
        super().__init__()
        self.n, self.scale, self.dtype = n, scale, dtype
        self.table = torch.nn.Parameter(torch.empty(V, C, device=device, dtype=table_dtype).normal_(0.0, std))

    def forward(self, ids):
        return _Embed.apply(self.table, ids, self.n, self.scale, self.dtype)


class StreamsNorm(torch.nn.Module):
    """RMS norm of the sum of the streams x [T, n, C], or of one row h [T, C], with a gain; [T, C]."""

    def __init__(self, C: int, eps: float = 1e-6, device="cuda"):
        super().__init__()
        self.eps = eps
        self.gain = torch.nn.Parameter(torch.ones(C, device=device))

    def forward(self, x):
        return _Norm.apply(x if x.dim() == 3 else x.unsqueeze(1), self.gain, self.eps)


class Head(torch.nn.Module):
    """The mean of the softmax cross entropy of h W^T with the next tokens [T] over those that are not negative, or, with weight [T],
    the sum of weight times it, whose gradient on weight[t] is the token's cross entropy.  W [V, C] is of h's type; `table`: the parameter of an embedding of that type, shared."""

    def __init__(self, V: int, C: int, dtype=torch.bfloat16, std: float = 0.02, device="cuda", table=None):
        super().__init__()
        if table is not None and (table.shape != (V, C) or table.dtype is not dtype):
            raise ValueError(f"table must be [{V}, {C}] of {dtype}, got {tuple(table.shape)} of {table.dtype}")
        self.W = table if table is not None else torch.nn.Parameter(torch.empty(V, C, device=device, dtype=dtype).normal_(0.0, std))

    def forward(self, h, targets, weight=None):
        # (also where no gradient is asked for: a forward-mode tangent is refused there)
        return _HeadTotal.apply(h, self.W, targets, weight, torch.is_grad_enabled())

    def distill(self, h, ids, logits, weight=None, temperature: float = 1.0):
        """The mean of `head_distill`'s loss over the tokens that count, or, with weight [T], the sum of weight times it."""
        _constant(logits=logits)
        return _DistillTotal.apply(h, self.W, weight, ids, logits, temperature, torch.is_grad_enabled())

    def prefer(self, h, targets, offsets, reference=None, weight=None, beta: float = 0.1, smoothing: float = 0.0):
        """The mean of `head_preference`'s loss over the pairs, or, with weight [P], the sum of weight times it; and logp [2 P], as numbers."""
        _constant(reference=reference)
        return _PreferenceTotal.apply(h, self.W, weight, targets, offsets, reference, beta, smoothing, torch.is_grad_enabled())

    @torch.no_grad()
    def score(self, h, targets):
        """``loss [T], lse [T]`` of each token."""
        return head_loss(h, self.W, targets)
