"""The ends' autograd nodes on the CPU, with torch's formulas in place of the library's calls: which gradient goes where, and what is refused."""
import pytest
import torch

from paper_2601_05732_amd import binding, ends


def _losses(h, W, targets):
    z = h @ W.t()
    lse = torch.logsumexp(z, dim=1)
    loss = lse - z.gather(1, targets.clamp(min=0).unsqueeze(1)).squeeze(1)
    return torch.where(targets >= 0, loss, 0.0), lse


def _sum(targets, loss, weight):
    if weight is None:
        return loss.sum() / max(1, int((targets >= 0).sum()))
    w = torch.where(targets >= 0, weight, 0.0)
    return torch.where(w != 0, w * loss, 0.0).sum()


def _loss_grad(h, W, targets, weight=None, dtype=None):
    with torch.enable_grad():
        h, W = h.detach().requires_grad_(), W.detach().requires_grad_()
        loss, lse = _losses(h, W, targets)
        g_h, g_W = torch.autograd.grad(_sum(targets, loss, None if weight is None else weight.detach()), [h, W])
    return loss.detach(), lse.detach(), g_h, g_W


def _norm(x, gain, eps):
    s = x.sum(dim=1)
    return gain * s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt()


def _norm_grad(x, gain, g_h, eps=1e-6):
    with torch.enable_grad():
        x, gain = x.detach().requires_grad_(), gain.detach().requires_grad_()
        return torch.autograd.grad(_norm(x, gain, eps), [x, gain], g_h.detach())


def _embed(table, ids, n, scale=1.0, dtype=None):
    return torch.where((ids >= 0).unsqueeze(1), scale * table[ids.clamp(min=0)], 0.0).unsqueeze(1).repeat(1, n, 1)


def _embed_grad(ids, g_x, V, scale=1.0, dtype=None):
    rows = torch.where((ids >= 0).unsqueeze(1), scale * g_x.detach().sum(dim=1), 0.0)
    return torch.zeros(V, g_x.shape[2]).index_add_(0, ids.clamp(min=0), rows)


@pytest.fixture(autouse=True)
def _formulas(monkeypatch):
    no_grad = torch.no_grad()
    for name, f in dict(head_loss=no_grad(_losses), head_loss_grad=_loss_grad, streams_norm=no_grad(_norm), streams_norm_grad=_norm_grad,
                        embed_tokens=no_grad(_embed), embed_tokens_grad=_embed_grad).items():
        monkeypatch.setattr(ends, name, f)
    monkeypatch.setattr(ends, "_total", no_grad(lambda h, W, targets, loss, weight: _sum(targets, loss, weight)))
    monkeypatch.setattr(binding, "mhcl_scale", no_grad(lambda t, f: t.mul_(f)))


def _case(seed=0, T=12, V=9, C=8):
    g = torch.Generator().manual_seed(seed)
    head = ends.Head(V, C, dtype=torch.float32, std=0.5, device="cpu")
    with torch.no_grad():
        head.W.copy_(torch.randn(V, C, generator=g) / 2)
    targets = torch.randint(0, V, (T,), generator=g)
    targets[::5] = -1
    return head, torch.randn(T, C, generator=g), targets, torch.rand(T, generator=g)


@pytest.mark.parametrize("others", [True, False])
def test_a_weight_that_needs_a_gradient_gets_the_losses(others):
    head, h, targets, weight = _case()
    h.requires_grad_(others)
    head.W.requires_grad_(others)
    logits = weight.clone().requires_grad_()
    total = head(h, targets, torch.sigmoid(logits))
    (1.5 * total).backward()
    got = logits.grad.clone()
    grads = [h.grad, head.W.grad]
    logits.grad = h.grad = head.W.grad = None
    (1.5 * _sum(targets, _losses(h, head.W, targets)[0], torch.sigmoid(logits))).backward()
    assert torch.allclose(got, logits.grad, rtol=1e-5, atol=1e-7) and not got[targets < 0].any()
    for a, b in zip(grads, [h.grad, head.W.grad]):
        assert a is b is None or torch.allclose(a, b, rtol=1e-5, atol=1e-6)


def test_a_weight_of_zero_keeps_what_a_place_holds_out_of_its_gradient():
    head, h, targets, weight = _case()
    at = int((targets >= 0).nonzero()[0])
    weight[at] = 0.0
    weight.requires_grad_()
    head(h, targets, weight).backward()
    assert torch.allclose(weight.grad, _losses(h, head.W, targets)[0])            # a place of weight 0 has its loss as gradient ...
    h[at] = float("nan")
    weight.grad = None
    head(h, targets, weight).backward()
    assert torch.isfinite(weight.grad).all() and float(weight.grad[at]) == 0.0    # ... unless that is no number


@pytest.mark.parametrize("which", ["h", "W", "weight"])
@pytest.mark.parametrize("grad", [False, True])
def test_a_forward_mode_tangent_is_refused(which, grad):
    head, h, targets, weight = _case()
    head.W.requires_grad_(False)
    with torch.autograd.forward_ad.dual_level(), torch.set_grad_enabled(grad):
        dual = dict(h=h, W=head.W.detach(), weight=weight)
        dual[which] = torch.autograd.forward_ad.make_dual(dual[which], torch.ones_like(dual[which]))
        if which == "W":
            del head.W
            head.W = dual["W"]
        with pytest.raises(NotImplementedError, match="jvp"):
            head(dual["h"], targets, dual["weight"])


def test_without_gradients_none_are_taken(monkeypatch):
    head, h, targets, weight = _case()
    h.requires_grad_()
    monkeypatch.setattr(ends, "head_loss_grad", lambda *a: pytest.fail("gradients were taken"))
    with torch.no_grad():
        assert torch.allclose(head(h, targets, weight), _sum(targets, _losses(h, head.W, targets)[0], weight))
    head.W.requires_grad_(False)
    assert not head(h.detach(), targets).requires_grad


def _through_head(a):
    head, h, targets, weight = _case()
    return head(h @ a, targets, weight), [a, head.W]


def _through_head_alone(a):            # nothing before it: the gradient that arrives is a constant
    head, h, targets, weight = _case()
    head.W.requires_grad_(False)
    return head(a, targets[:8]), [a]


def _through_norm(a):
    norm = ends.StreamsNorm(8, device="cpu")
    return (norm(a.unsqueeze(1)) * torch.arange(8.0)).sum(), [a, norm.gain]


def _through_norm_s_gradient(a):       # linear in the gain, whose gradient depends on a
    norm = ends.StreamsNorm(8, device="cpu")
    return (norm(a.detach().unsqueeze(1)) * a).sum(), [norm.gain]


def _through_embedding(a):
    emb = ends.TokenEmbedding(9, 8, 2, dtype=torch.float32, device="cpu")
    return (emb(torch.tensor([1, 3, -1, 3])) * a[:4].unsqueeze(1)).sum(), [emb.table]


_PATHS = [_through_head, _through_head_alone, _through_norm, _through_norm_s_gradient, _through_embedding]


@pytest.mark.parametrize("path", _PATHS)
@pytest.mark.parametrize("only", [False, True])
def test_a_second_derivative_is_refused(path, only):
    a = torch.randn(8, 8, generator=torch.Generator().manual_seed(1)).requires_grad_()
    value, wrt = path(a)
    grads = torch.autograd.grad(value, wrt, create_graph=True)
    penalty = sum(g.square().sum() for g in grads) + a.square().sum()
    with pytest.raises(RuntimeError, match="no second derivative"):
        torch.autograd.grad(penalty, [a]) if only else penalty.backward()


@pytest.mark.parametrize("path", _PATHS)
def test_a_recorded_backward_returns_the_same_gradients(path):
    a = torch.randn(8, 8, generator=torch.Generator().manual_seed(1)).requires_grad_()
    torch.manual_seed(2)
    value, wrt = path(a)
    recorded = torch.autograd.grad(value, wrt, create_graph=True)
    torch.manual_seed(2)
    value, wrt = path(a)
    for x, y in zip(recorded, torch.autograd.grad(value, wrt)):
        assert torch.equal(x, y) and x.shape == y.shape
        (x.detach() + a.sum()).sum().backward()


def test_a_place_without_gradients_in_a_recorded_backward():
    head, h, targets, _ = _case()
    head.W.requires_grad_(False)
    h.requires_grad_()
    head(h, targets).backward(create_graph=True)
    assert h.grad is not None and head.W.grad is None
