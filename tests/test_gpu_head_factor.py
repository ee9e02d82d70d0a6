"""A factor on the head's loss: bf16 gradients are rounded once, with the factor in them.

Bounds, fixed before the first run: where every sum is one of a few bf16 numbers, a gradient is off by one rounding to bf16, 2^-8 of
itself, and by fp32 roundings, 2^-22 of the sum of its terms' sizes.  Elsewhere the fp32 gradients, rounded, are the bf16 ones' bits.
"""
import pytest
import torch

import paper_2601_05732_amd as mhcl

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("factor", [1 / 3, 1 / 6, 0.7, 1.0, 2.0])
def test_bf16_gradients_are_rounded_once(factor, weighted):
    # softmaxes that are 1 for a row which is not the target's: g is 1 there and -1 at the target, nothing else is rounded
    T, V, C = 64, 40, 64
    head = mhcl.Head(V, C, dtype=BF, std=1.0)
    W = head.W.detach()
    wrong = torch.arange(T, device="cuda") % 20
    targets = 20 + torch.randint(0, 20, (T,), device="cuda", generator=_gen(1))
    h = (4 * W[wrong]).clone().requires_grad_()
    assert torch.equal(torch.softmax(h.double() @ W.double().t(), dim=1).argmax(dim=1), wrong)
    weight = torch.full((T,), 0.3, device="cuda") if weighted else None
    (head(h, targets, weight) * factor).backward()
    one = (float(weight[0]) if weighted else 1 / T) * float(torch.tensor(factor))
    ref_h = one * (W[wrong].double() - W[targets].double())
    size_h = one * (W[wrong].double().abs() + W[targets].double().abs())
    ref_W, size_W = (torch.zeros(V, C, device="cuda", dtype=torch.float64) for _ in range(2))
    for rows, sign in ((wrong, 1.0), (targets, -1.0)):
        ref_W.index_add_(0, rows, sign * one * h.detach().double())
        size_W.index_add_(0, rows, one * h.detach().double().abs())
    for name, got, ref, size in (("g_h", h.grad, ref_h, size_h), ("g_W", head.W.grad, ref_W, size_W)):
        over = (got.double() - ref).abs() / (2 ** -8 * ref.abs() + 2 ** -22 * size)
        assert float(over.max()) <= 1, f"{name}: {float(over.max()):.3f} of the bound"


@pytest.mark.parametrize("T,C,V", [(1, 8, 1), (333, 520, 1003), (1030, 136, 90), (2049, 72, 8200), (40, 128, 30011), (1300, 16, 2 ** 20),
                                   (4200, 4104, 1100)])
@pytest.mark.parametrize("weighted", [False, True])
def test_unrounded_gradients_round_to_the_bf16_ones(T, C, V, weighted):
    g = _gen(T + V)
    h = torch.empty(T, C, device="cuda").normal_(generator=g).to(BF)
    W = torch.empty(V, C, device="cuda").normal_(0.0, 1.5 / C ** 0.5, generator=g).to(BF)
    targets = torch.randint(-V // 8, V, (T,), device="cuda", generator=g)
    weight = torch.rand(T, device="cuda", generator=g) if weighted else None
    rounded = mhcl.head_loss_grad(h, W, targets, weight)
    full = mhcl.head_loss_grad(h, W, targets, weight, dtype=F)
    assert full[2].dtype is F and full[3].dtype is F
    for a, b in zip(rounded, full):
        assert torch.equal(a, b.to(a.dtype))


def test_python_and_native_calls_agree_on_unrounded_gradients(monkeypatch):
    from paper_2601_05732_amd import ends
    g = _gen(5)
    h, W = (torch.empty(n, 64, device="cuda").normal_(generator=g).to(BF) for n in (40, 90))
    targets = torch.randint(0, 90, (40,), device="cuda", generator=g)
    quick = mhcl.head_loss_grad(h, W, targets, dtype=F)
    monkeypatch.setattr(ends, "_native", lambda: None)
    for a, b in zip(quick, mhcl.head_loss_grad(h, W, targets, dtype=F)):
        assert a.dtype is b.dtype and torch.equal(a, b)


def test_no_tokens_unrounded():
    W = torch.ones(30, 64, device="cuda", dtype=BF)
    out = mhcl.head_loss_grad(torch.empty(0, 64, device="cuda", dtype=BF), W, torch.empty(0, device="cuda", dtype=torch.int64), dtype=F)
    assert out[2].shape == (0, 64) and out[3].dtype is F and not out[3].any()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("count", [1, 7, 8, 1003, 4096 * 2048 + 5])
def test_scale_to(dtype, count):
    x = torch.empty(count, device="cuda").normal_(generator=_gen(4))
    for value in (1.0, 1 / 3, float("nan")):
        out = torch.empty(count, device="cuda", dtype=dtype)
        mhcl.mhcl_scale_to(x, torch.tensor(value, device="cuda"), out)
        assert torch.equal(out.nan_to_num(7.0), (x * value).to(dtype).nan_to_num(7.0))


def test_refusals():
    h, W = torch.ones(5, 64, device="cuda", dtype=BF), torch.ones(9, 64, device="cuda", dtype=BF)
    targets, one = torch.zeros(5, device="cuda", dtype=torch.int64), torch.ones(1, device="cuda")
    for call in (lambda: mhcl.head_loss_grad(h, W, targets, dtype=torch.float16), lambda: mhcl.head_loss_grad(h.float(), W.float(), targets, dtype=BF),
                 lambda: mhcl.mhcl_scale_to(h, one, torch.empty_like(h)), lambda: mhcl.mhcl_scale_to(h.float(), one, h[:3]),
                 lambda: mhcl.mhcl_scale_to(h.float(), one, h.half())):
        with pytest.raises(ValueError):
            call()
