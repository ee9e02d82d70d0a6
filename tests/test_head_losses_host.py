"""Host side of the head's losses against a teacher and of pairs (no GPU needed): refusals and workspaces of the C ABI."""
import ctypes
import math

import pytest
import torch

import paper_2601_05732_amd as mhcl
from paper_2601_05732_amd import binding, ends

OK = 4096      # an aligned, never dereferenced address: validation fails first


def _desc(**kw):
    base = dict(n=1, C=64, T=16, V=100, io_dtype=mhcl.BF16, w_dtype=mhcl.BF16, id_dtype=mhcl.I64, scale=1.0, eps=0.0)
    base.update(kw)
    return binding._CEndsDesc(*[base[k] for k, _ in binding._CEndsDesc._fields_])


def _distill(d, K=4, tau=1.0, ws=None, bytes_=0, **kw):
    p = dict(h=OK, W=OK, ids=OK, logits=OK, weight=None, loss=OK, lse=OK, total=None, g_h=OK, g_W=OK)
    p.update(kw)
    return mhcl.lib().mhcl_head_distill(ctypes.byref(d), K, tau, *p.values(), 0, ws, bytes_, None)


def _prefer(d, pairs=2, beta=0.1, smoothing=0.0, offset_dtype=mhcl.I64, ws=None, bytes_=0, **kw):
    p = dict(h=OK, W=OK, targets=OK, offsets=OK)
    q = dict(reference=None, weight=None, loss=OK, logp=OK, total=None, g_h=OK, g_W=OK)
    for k, v in kw.items():
        (p if k in p else q)[k] = v
    return mhcl.lib().mhcl_head_preference(ctypes.byref(d), pairs, beta, smoothing, *p.values(), offset_dtype, *q.values(), 0, ws, bytes_, None)


@pytest.mark.parametrize("kw,status", [
    (dict(C=0), 1), (dict(C=12), 1), (dict(T=-1), 1), (dict(io_dtype=5), 1), (dict(V=0), 1), (dict(w_dtype=2), 1), (dict(id_dtype=7), 1),
    (dict(C=32776), 2), (dict(T=2 ** 30 + 1), 2), (dict(V=2 ** 22 - 255), 2), (dict(w_dtype=mhcl.F32), 2),
])
def test_descriptors_that_are_refused(kw, status):
    d = _desc(**kw)
    assert _distill(d) == status and _prefer(d) == status
    for grad in (0, 1):
        assert mhcl.lib().mhcl_head_distill_workspace_bytes(ctypes.byref(d), 4, grad) == 0
        assert mhcl.lib().mhcl_head_preference_workspace_bytes(ctypes.byref(d), grad) == 0


def test_numbers_that_are_refused():
    d = _desc()
    for tau in (0.0, -1.0, math.nan, math.inf, 1e-7, 1e7):
        assert _distill(d, tau=tau) == 1
    assert _distill(d, K=0) == 1 and _distill(d, K=-1) == 1 and _distill(d, K=257) == 2 and _distill(d, K=256) == 3
    for K in (0, 257):
        assert mhcl.lib().mhcl_head_distill_workspace_bytes(ctypes.byref(d), K, 0) == 0
    for kw in (dict(beta=math.nan), dict(beta=math.inf), dict(smoothing=-0.1), dict(smoothing=1.5), dict(smoothing=math.nan), dict(pairs=-1),
               dict(offset_dtype=2)):
        assert _prefer(d, **kw) == 1, kw
    assert _prefer(d, pairs=2 ** 22 + 1) == 2


@pytest.mark.parametrize("call", [_distill, _prefer])
def test_pointers(call):
    d = _desc()
    assert call(d) == 3                                               # no workspace
    names = dict(h=8, W=8, loss=2, g_h=8, g_W=8)
    names.update(dict(ids=4, logits=2, lse=2) if call is _distill else dict(targets=4, offsets=4, logp=2))
    for name, off in names.items():
        assert call(d, **{name: None}) == 1, name
        assert call(d, **{name: OK + off}) == 1, name
    for name in ("weight", "total") + (("reference",) if call is _prefer else ()):
        assert call(d, **{name: OK + 2}) == 1 and call(d, **{name: OK + 4}) == 3, name
    assert call(d, g_h=None, g_W=None) == 3                           # the loss alone
    grad_bytes = (mhcl.lib().mhcl_head_distill_workspace_bytes(ctypes.byref(d), 4, 1) if call is _distill
                  else mhcl.lib().mhcl_head_preference_workspace_bytes(ctypes.byref(d), 1))
    assert call(d, ws=OK, bytes_=grad_bytes - 1) == 3 and call(d, ws=OK + 8, bytes_=2 * grad_bytes) == 3
    assert call(_desc(id_dtype=mhcl.I32), **({"ids": OK + 4} if call is _distill else {"targets": OK + 4})) == 3


def test_workspaces_hold_a_block_of_tokens():
    d, more = _desc(T=16384, C=1024, V=50257), _desc(T=2 ** 20, C=1024, V=50257)
    for f in (lambda d: mhcl.lib().mhcl_head_distill_workspace_bytes(ctypes.byref(d), 256, 1),
              lambda d: mhcl.lib().mhcl_head_preference_workspace_bytes(ctypes.byref(d), 1)):
        assert 16384 * 50257 * 2 < f(d) < f(more) < 6 * 2 ** 30


def test_tensors_of_the_cpu_are_refused():
    h, W, ids = torch.ones(6, 64), torch.ones(10, 64), torch.zeros(6, dtype=torch.int64)
    offsets = torch.tensor([0, 3, 6])
    for call in (lambda: mhcl.head_distill(h, W, ids[:, None], h[:, :1]), lambda: mhcl.head_distill_grad(h, W, ids[:, None], h[:, :1]),
                 lambda: mhcl.head_preference(h, W, ids, offsets), lambda: mhcl.head_preference_grad(h, W, ids, offsets)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            call()


def test_constants_that_ask_for_a_gradient_are_refused():
    head = ends.Head(10, 64, device="cpu")
    h, ids = torch.ones(6, 64, dtype=torch.bfloat16), torch.zeros(6, 1, dtype=torch.int64)
    with pytest.raises(ValueError, match="logits is a constant"):
        head.distill(h, ids, torch.ones(6, 1, requires_grad=True))
    with pytest.raises(ValueError, match="reference is a constant"):
        head.prefer(h, ids[:, 0], torch.tensor([0, 3, 6]), torch.zeros(2, requires_grad=True))
