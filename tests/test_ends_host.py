"""Host side of the two ends of a language model (no GPU needed): descriptors, workspaces and refusals of the C ABI, and which
calls the extension in C++ leaves to Python."""
import ctypes

import pytest
import torch

import paper_2601_05732_amd as mhcl
from paper_2601_05732_amd import autograd, binding, ends

OK = 4096      # an aligned, never dereferenced address: validation fails first


def _desc(**kw):
    base = dict(n=4, C=64, T=16, V=100, io_dtype=mhcl.BF16, w_dtype=mhcl.BF16, id_dtype=mhcl.I64, scale=1.0, eps=1e-6)
    base.update(kw)
    return binding._CEndsDesc(*[base[k] for k, _ in binding._CEndsDesc._fields_])


def _bytes(d, op):
    return mhcl.lib().mhcl_ends_workspace_bytes(ctypes.byref(d), op)


def _calls(d):
    """Every entry point with the descriptor and plausible arguments, but no workspace."""
    L, r = mhcl.lib(), ctypes.byref(d)
    return dict(
        embed=lambda: L.mhcl_embed(r, None, None, None, None),
        embed_bwd=lambda: L.mhcl_embed_bwd(r, OK, OK, OK, 0, None, 0, None),
        norm=lambda: L.mhcl_streams_norm(r, None, None, None, None),
        norm_bwd=lambda: L.mhcl_streams_norm_bwd(r, OK, OK, OK, OK, OK, None, 0, None),
        head=lambda: L.mhcl_head_loss(r, OK, OK, OK, OK, OK, None, 0, None),
        head_grad=lambda: L.mhcl_head_loss_grad(r, OK, OK, OK, None, OK, OK, OK, OK, None, 0, None),
        total=lambda: L.mhcl_head_total(r, None, None, None, None, None))


@pytest.mark.parametrize("kw,refused", [
    (dict(C=0), "embed embed_bwd norm norm_bwd head head_grad total"), (dict(C=12), "embed embed_bwd norm norm_bwd head head_grad total"),
    (dict(T=-1), "embed embed_bwd norm norm_bwd head head_grad total"), (dict(io_dtype=5), "embed embed_bwd norm norm_bwd head head_grad total"),
    (dict(n=0), "embed embed_bwd norm norm_bwd"), (dict(n=9), "embed embed_bwd norm norm_bwd"),
    (dict(V=0), "embed embed_bwd head head_grad total"), (dict(w_dtype=2), "embed embed_bwd head head_grad total"),
    (dict(id_dtype=7), "embed embed_bwd head head_grad total"),
    (dict(scale=float("inf")), "embed embed_bwd"), (dict(scale=float("nan")), "embed embed_bwd"),
    (dict(eps=-1.0), "norm norm_bwd"), (dict(eps=float("nan")), "norm norm_bwd"),
])
def test_invalid_descriptors(kw, refused):
    d = _desc(**kw)
    for name in refused.split():
        assert _calls(d)[name]() == 1, name
    ops = dict(embed_bwd=mhcl.OP_EMBED_BWD, norm_bwd=mhcl.OP_STREAMS_NORM_BWD, head=mhcl.OP_HEAD_LOSS, head_grad=mhcl.OP_HEAD_LOSS_GRAD)
    for name, op in ops.items():
        assert (_bytes(d, op) == 0) == (name in refused.split()), name


@pytest.mark.parametrize("kw,refused", [
    (dict(C=32776), ("embed_bwd", "norm_bwd", "head", "head_grad")), (dict(T=2 ** 30 + 1), ("embed_bwd", "norm_bwd", "head", "head_grad")),
    (dict(V=2 ** 30 + 1), ("embed_bwd", "head", "head_grad")), (dict(w_dtype=mhcl.F32), ("head", "head_grad")),
])
def test_unsupported_descriptors(kw, refused):
    d = _desc(**kw)
    for name in refused:
        assert _calls(d)[name]() == 2, name


def test_pointers_and_workspaces():
    d = _desc()
    calls = _calls(d)
    assert calls["embed"]() == 1 and calls["norm"]() == 1 and calls["total"]() == 1      # null tensors
    for name in ("embed_bwd", "norm_bwd", "head", "head_grad"):
        assert calls[name]() == 3                                                        # no workspace
    L, r = mhcl.lib(), ctypes.byref(d)
    assert L.mhcl_head_loss(r, OK, OK, OK, OK, OK, OK, _bytes(d, mhcl.OP_HEAD_LOSS) - 1, None) == 3
    assert L.mhcl_head_loss(r, OK + 4, OK, OK, OK, OK, None, 0, None) == 1               # h at 16 bytes
    assert L.mhcl_head_loss(r, OK, OK, OK + 8, OK + 4, OK + 4, None, 0, None) == 3       # targets at 8, losses at 4
    assert L.mhcl_head_loss(r, OK, OK, OK + 4, OK, OK, None, 0, None) == 1
    i32 = _desc(id_dtype=mhcl.I32)
    assert L.mhcl_head_loss(ctypes.byref(i32), OK, OK, OK + 4, OK, OK, None, 0, None) == 3
    assert L.mhcl_embed_bwd(r, OK, OK, OK + 8, 0, None, 0, None) == 1
    assert L.mhcl_scale(OK, 9, 8, OK, None) == 1 and L.mhcl_scale(OK, mhcl.F32, -1, OK, None) == 1
    assert L.mhcl_scale(OK + 4, mhcl.F32, 8, OK, None) == 1 and L.mhcl_scale(None, mhcl.F32, 0, OK, None) == 0
    for name in ("embed", "norm", "head"):                                               # no tokens: nothing to do
        assert _calls(_desc(T=0))[name]() == 0
    assert mhcl.lib().mhcl_ends_workspace_bytes(r, 4) == 0 and mhcl.lib().mhcl_ends_workspace_bytes(None, 0) == 0


def test_the_head_s_workspace_stays_bounded():
    small = _bytes(_desc(T=16384, C=1024, V=50257), mhcl.OP_HEAD_LOSS_GRAD)
    large = _bytes(_desc(T=2 ** 20, C=1024, V=50257), mhcl.OP_HEAD_LOSS_GRAD)
    assert 16384 * 50257 * 2 < small < large < 6 * 2 ** 30
    assert _bytes(_desc(T=2 ** 20, C=1024, V=50257), mhcl.OP_HEAD_LOSS) < 4 * 2 ** 30


def test_types_that_have_no_number():
    for kw in (dict(io=torch.float16), dict(w=torch.float64), dict(ids=torch.int16), dict(V=2 ** 40)):
        with pytest.raises(ValueError):
            mhcl.EndsDesc(64, 1, **kw)


def test_tensors_of_the_cpu_are_left_to_python_and_refused():
    native = autograd._native()
    table, ids = torch.ones(10, 64), torch.zeros(3, dtype=torch.int64)
    x, gain, h = torch.ones(3, 2, 64), torch.ones(64), torch.ones(3, 64)
    if torch.cuda.is_available():
        assert native.norm(x, gain, 1e-6) is None
    for call in (lambda: ends.embed_tokens(table, ids, 2), lambda: ends.embed_tokens_grad(ids, x, 10),
                 lambda: ends.streams_norm(x, gain), lambda: ends.streams_norm_grad(x, gain, h),
                 lambda: ends.head_loss(h, table, ids), lambda: ends.head_loss_grad(h, table, ids)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            call()


def test_a_shared_table_has_to_fit():
    with pytest.raises(ValueError, match="table must be"):
        ends.Head(10, 64, dtype=torch.bfloat16, device="cpu", table=torch.nn.Parameter(torch.ones(10, 64)))


@pytest.mark.parametrize("io", ["BF16", "F32"])
def test_the_head_s_vocabulary_is_bounded_where_its_offsets_are(io):
    kw = dict(io_dtype=getattr(mhcl, io), w_dtype=getattr(mhcl, io))
    most = 2 ** 22 - 256       # 256 rows of as many numerators of two bytes, or 128 of four, are just under 2^31 bytes
    for op in (mhcl.OP_HEAD_LOSS, mhcl.OP_HEAD_LOSS_GRAD):
        assert _bytes(_desc(V=most, **kw), op) > 0
        assert _bytes(_desc(V=most + 1, **kw), op) == 0
    d = _desc(V=most + 1, **kw)
    for name in ("head", "head_grad"):
        assert _calls(d)[name]() == 2, name
    assert _bytes(_desc(V=most + 1, **kw), mhcl.OP_EMBED_BWD) > 0      # a table may have more
