"""The head's exponentials where nothing else hides their error: a few logits that bf16 operands give exactly.

The bounds, fixed before the first run, by units of 2^-24 (an fp32 rounding to nearest):
  * an exponential of x = z - max z <= 0: 2 |x| for the rounded product with log2(e) and that constant, 2 for the instruction;
  * the sum of V of them, the largest 1: their errors, weighted by what they are, and V roundings of the sum;
  * the logarithm of a sum s: the sum's error over s, 2 |log s| for the logarithm, and a rounding where the maximum is added.
"""
import pytest
import torch

import paper_2601_05732_amd as mhcl

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
UNIT = 2.0 ** -24


@pytest.mark.parametrize("T", [1, 40, 2000])          # tiles of one token, of few, of many
@pytest.mark.parametrize("V,spread", [(2, 1.0), (2, 12.0), (3, 0.25), (8, 1.0), (8, 30.0)])
@pytest.mark.parametrize("grad", [False, True])
def test_loss_and_lse_of_exact_logits(grad, V, spread, T):
    g = torch.Generator(device="cuda").manual_seed(V * T)
    C = 8
    # one product of bf16 numbers each: 16 bits, exact in fp32
    h = torch.zeros(T, C, device="cuda", dtype=BF)
    h[:, 0] = (torch.rand(T, device="cuda", generator=g) * spread).to(BF)
    W = torch.zeros(V, C, device="cuda", dtype=BF)
    W[:, 0] = -torch.arange(V, device="cuda").to(BF) / V
    targets = torch.randint(0, V, (T,), device="cuda", generator=g)
    z = h[:, :1].double() @ W[:, :1].double().t()
    assert torch.equal(z, z.float().double())
    e = z.exp()                                        # the largest logit is 0
    s = e.sum(dim=1)
    lse = s.log()
    z_y = z.gather(1, targets.unsqueeze(1)).squeeze(1)
    of_sum = (e * (2 * z.abs() + 2)).sum(dim=1) + V * s
    e_lse = UNIT * (of_sum / s + 3 * lse.abs())
    e_loss = e_lse + UNIT * (z_y.abs() + (lse - z_y).abs())
    got = mhcl.head_loss_grad(h, W, targets) if grad else mhcl.head_loss(h, W, targets)
    for name, a, ref, bound in (("loss", got[0], lse - z_y, e_loss), ("lse", got[1], lse, e_lse)):
        over = (a.double() - ref).abs() / bound
        assert float(over.max()) <= 1, f"{name}: {float(over.max()):.2f} of the bound"
