"""Host side of the gated feed-forward block (no GPU needed): descriptors, workspaces and refusals."""
import ctypes
import itertools

import pytest
import torch

import paper_2601_05732_amd as mhcl
from paper_2601_05732_amd import binding, ffn

OK = 4096      # an aligned, never dereferenced address: validation fails first


def _desc(**kw):
    base = dict(C=64, H=128, T=16, io_dtype=mhcl.BF16)
    base.update(kw)
    return binding._CFfnDesc(*[base[k] for k, _ in binding._CFfnDesc._fields_])


def _bytes(d, op):
    return mhcl.lib().mhcl_ffn_workspace_bytes(ctypes.byref(d), op)


def _forward(d, *args, ws=None, bytes_=0):
    return mhcl.lib().mhcl_ffn(ctypes.byref(d), *(args or (OK, OK, OK, OK, None)), ws, bytes_, None)


def _grad(d, *args, ws=None, bytes_=0):
    return mhcl.lib().mhcl_ffn_grad(ctypes.byref(d), *(args or (OK,) * 8), ws, bytes_, None)


@pytest.mark.parametrize("kw,status", [
    (dict(C=0), 1), (dict(C=12), 1), (dict(C=-8), 1), (dict(H=0), 1), (dict(H=20), 1), (dict(T=-1), 1), (dict(io_dtype=2), 1),
    (dict(C=32776), 2), (dict(H=131080), 2), (dict(C=16384, H=16392), 2), (dict(T=2 ** 30 + 1), 2), (dict(T=2 ** 30, H=4096), 2),
])
def test_descriptors_that_are_refused(kw, status):
    d = _desc(**kw)
    assert _forward(d) == status and _grad(d) == status
    assert _bytes(d, mhcl.OP_FFN) == 0 and _bytes(d, mhcl.OP_FFN_GRAD) == 0


def test_pointers_and_workspaces():
    d = _desc()
    assert mhcl.lib().mhcl_ffn(None, OK, OK, OK, OK, None, None, 0, None) == 1
    assert _forward(d) == 3 and _grad(d) == 3                                 # no workspace
    assert _forward(d, ws=OK, bytes_=_bytes(d, mhcl.OP_FFN) - 1) == 3
    assert _grad(d, ws=OK, bytes_=_bytes(d, mhcl.OP_FFN_GRAD) - 1) == 3
    for i in range(5):
        args = [OK, OK, OK, OK, OK]
        args[i] += 8
        assert _forward(d, *args) == 1, i
        args[i] = None
        assert _forward(d, *args) == (3 if i == 4 else 1), i                  # pre may be missing
    for i in range(8):
        args = [OK] * 8
        args[i] = None
        assert _grad(d, *args) == 1, i
    assert _forward(_desc(T=0), None, None, None, None, None) == 0            # nothing to do
    assert _grad(_desc(T=0), None, None, None, None, None, None, None, OK) == 1   # the weights' gradients are zeros there
    assert _bytes(d, 2) == 0 and mhcl.lib().mhcl_ffn_workspace_bytes(None, 0) == 0


def test_the_workspace_holds_the_hidden_numbers():
    d = _desc(C=1024, H=4096, T=8192)
    assert 8192 * 4096 * 2 <= _bytes(d, mhcl.OP_FFN) < 2 * 8192 * 4096 * 2
    assert 3 * 8192 * 4096 * 2 <= _bytes(d, mhcl.OP_FFN_GRAD)


def test_tensors_that_do_not_fit_are_refused():
    x, up, down = torch.ones(3, 64), torch.ones(48, 64), torch.ones(64, 24)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        mhcl.gated_ffn(x, up, down)                                           # on the CPU
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        mhcl.gated_ffn_grad(x, up, down, torch.ones(3, 48), x)
    for kw in (dict(io=torch.float16), dict(io=torch.float64)):
        with pytest.raises(ValueError):
            mhcl.FfnDesc(64, 64, 1, **kw)
    with pytest.raises(ValueError):
        mhcl.FfnDesc(2 ** 40, 64, 1)


def _grad_of(d, *args, ws=None, bytes_=0):
    return mhcl.lib().mhcl_ffn_grad_of(ctypes.byref(d), *(args or (OK,) * 8), ws, bytes_, None)


def test_gradients_that_are_not_asked_for_may_be_missing():
    d = _desc()
    for i in range(8):
        args = [OK] * 8
        args[i] = None
        assert _grad_of(d, *args) == (1 if i < 5 else 3), i
        args[i] = OK + 8
        assert _grad_of(d, *args) == 1, i
    assert _grad_of(d, OK, OK, OK, OK, OK, None, None, OK) == 3
    assert _grad_of(d, OK, OK, OK, OK, OK, None, None, None) == 1
    assert _grad_of(d, ws=OK, bytes_=_bytes(d, mhcl.OP_FFN_GRAD) - 1) == 3
    assert _grad_of(_desc(C=12)) == 1 and _grad_of(_desc(T=2 ** 30 + 1)) == 2
    assert _grad_of(_desc(T=0), *(None,) * 8) == 0                            # nothing to do
    assert mhcl.lib().mhcl_ffn_grad_of(None, *(OK,) * 8, None, 0, None) == 1


@pytest.mark.parametrize("wanted", list(itertools.product((False, True), repeat=3)))
def test_autograd_forms_what_is_asked_for(monkeypatch, wanted):
    asked = []

    def forward(x, W_up, W_down, keep=False):
        pre = x @ W_up.t()
        a, b = pre.chunk(2, dim=-1)
        y = (torch.nn.functional.silu(a) * b) @ W_down.t()
        return (y, pre) if keep else y

    def backward(x, W_up, W_down, kept, g_y, wanted=(True, True, True)):
        asked.append(tuple(wanted))
        with torch.enable_grad():
            leaves = [t.detach().requires_grad_() for t in (x, W_up, W_down)]
            grads = torch.autograd.grad(forward(*leaves), leaves, g_y.detach())
        return tuple(g if w else None for g, w in zip(grads, wanted))

    monkeypatch.setattr(ffn, "gated_ffn", forward)
    monkeypatch.setattr(ffn, "gated_ffn_grad", backward)
    leaves = [torch.randn(s, requires_grad=w) for s, w in zip(((3, 8), (32, 8), (8, 16)), wanted)]
    y = ffn.apply_gated_ffn(*leaves)
    if not any(wanted):
        assert not y.requires_grad
        return
    y.sum().backward()
    assert asked == [wanted] and [t.grad is not None for t in leaves] == list(wanted)


def test_which_gradients_are_wanted_is_checked():
    x, up, down = torch.ones(3, 64), torch.ones(48, 64), torch.ones(64, 24)
    for wanted in ((False, False, False), (True, True), (True,) * 4):
        with pytest.raises(ValueError, match="wanted"):
            mhcl.gated_ffn_grad(x, up, down, torch.ones(3, 48), x, wanted)
