"""The head under torch.autograd on the GPU: the gradient on the tokens' weights."""
import pytest
import torch

import paper_2601_05732_amd as mhcl

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _case(io, T=70, V=130, C=64):
    g = torch.Generator(device="cuda").manual_seed(3)
    head = mhcl.Head(V, C, dtype=io, std=0.2)
    h = torch.empty(T, C, device="cuda").normal_(generator=g).to(io)
    return head, h, torch.randint(-30, V, (T,), device="cuda", generator=g), torch.rand(T, device="cuda", generator=g)


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("others", [False, True])
def test_the_gradient_on_a_weight_is_the_loss(io, others):
    head, h, targets, weight = _case(io)
    h.requires_grad_(others)
    head.W.requires_grad_(others)
    weight[7] = 0.0
    weight.requires_grad_()
    (0.375 * head(h, targets, weight)).backward()
    with torch.no_grad():
        loss = (mhcl.head_loss_grad(h, head.W, targets, weight) if others else mhcl.head_loss(h, head.W, targets))[0]
    assert torch.equal(weight.grad, loss * 0.375) and not weight.grad[targets < 0].any()
    if others:
        grads = mhcl.head_loss_grad(h.detach(), head.W.detach(), targets, weight.detach(), dtype=F)[2:]
        assert all(torch.equal(got, (g * 0.375).to(io)) for got, g in zip((h.grad, head.W.grad), grads))
    else:
        assert h.grad is None and head.W.grad is None


def test_a_strided_weight_and_one_of_another_type():
    head, h, targets, weight = _case(F)
    wide = torch.stack([weight, weight], dim=1).requires_grad_()
    head(h, targets, wide[:, 1]).backward()
    assert not wide.grad[:, 0].any() and torch.equal(wide.grad[:, 1], mhcl.head_loss_grad(h, head.W.detach(), targets, weight)[0])
    for bad in (weight.double(), weight[:-1]):
        for grad in (False, True):
            head.W.requires_grad_(grad)
            with pytest.raises(ValueError):
                head(h, targets, bad.detach().requires_grad_())
