"""A second derivative through the layers: refused by the nodes in C++ and by those in Python; a recorded backward that nobody
differentiates gives the plain one's bits."""
import gc

import pytest
import torch

from paper_2601_05732_amd import autograd
from paper_2601_05732_amd.autograd import HyperConnection, HyperConnectionStack

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["C++", "Python"], autouse=True)
def nodes(request, monkeypatch):
    if request.param == "Python":
        monkeypatch.setattr(autograd, "_plain", lambda *t: False)
    return request.param


def _layer(L=1):
    g = torch.Generator(device="cuda").manual_seed(L)
    f = torch.nn.Linear(64, 64, device="cuda")
    net = HyperConnection(3, 64, "sk") if L == 1 else HyperConnectionStack(3, 64, [f] * L, "sk")
    with torch.no_grad():
        for p in [*net.parameters(), *f.parameters()]:
            p.add_(torch.randn(p.shape, device="cuda", generator=g) * 0.1)
    x = torch.randn(*((9, 3, 64) if L == 1 else (9, 64)), device="cuda", generator=g, requires_grad=True)
    return (net, f, x, net(x, f)) if L == 1 else (net, f, x, net(x))


@pytest.mark.parametrize("L", [1, 3])
@pytest.mark.parametrize("linear", [False, True])      # a loss whose gradient on the output is a constant
@pytest.mark.parametrize("wrt", ["x", "parameters", "bias", "all"])
def test_refused(L, linear, wrt):
    net, f, x, out = _layer(L)
    value = out.sum() if linear else out.square().sum()
    grads = torch.autograd.grad(value, [x, *net.parameters(), *f.parameters()], create_graph=True, allow_unused=True)
    penalty = sum(g.square().sum() for g in grads if g is not None)
    ones = [f.bias] if wrt == "bias" else [x] if wrt == "x" else list(net.parameters())[:1]
    with pytest.raises(RuntimeError, match="no second derivative"):
        penalty.backward() if wrt == "all" else torch.autograd.grad(penalty, ones, allow_unused=True)


def test_an_end_of_a_stack_without_layers_between():
    stack = HyperConnectionStack(3, 64, [lambda h: h])
    x = torch.randn(9, 64, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(stack(x).square().sum(), [x], create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        torch.autograd.grad(g.sum(), [x])


@pytest.mark.parametrize("L", [1, 3])
def test_a_recorded_backward_gives_the_same_bits_and_lets_go(L):
    def run(create):
        net, f, x, out = _layer(L)
        return [t.detach() for t in torch.autograd.grad(out.square().sum(), [x, *net.parameters(), f.bias], create_graph=create)]
    torch.manual_seed(0)
    plain = run(False)
    for _ in range(2):
        torch.manual_seed(0)
        for a, b in zip(plain, run(True)):
            assert torch.equal(a, b) and a.shape == b.shape
    gc.collect()
    before = torch.cuda.memory_allocated()
    run(True)
    gc.collect()
    assert torch.cuda.memory_allocated() == before
