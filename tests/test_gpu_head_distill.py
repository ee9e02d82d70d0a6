"""The head against a teacher's top logits: against its definition in 64 bits element by element, at the sizes, slots and masks where it
can go wrong; its gradients against differences; under torch.autograd, captured.  Bounds: head_reference.py."""
import math

import pytest
import torch

import head_reference as ref
import paper_2601_05732_amd as mhcl
from paper_2601_05732_amd import ends

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=F):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _inputs(seed, T, C, V, K, io, short=0.3, holes=0.2, ids_dtype=torch.int64, spread=2.0):
    """Slots in no order, ids that repeat where K is not far below V, lists that end early, tokens without any."""
    g = _gen(seed)
    h, W = _normal(g, T, C, dtype=io), _normal(g, V, C, std=1.5 / math.sqrt(C), dtype=io)
    ids = torch.randint(0, V, (T, K), device="cuda", generator=g)
    logits = _normal(g, T, K, std=spread)
    u = torch.rand(T, 2, device="cuda", generator=g)
    count = torch.where(u[:, 0] < short, (u[:, 1] * K).long() + 1, K)
    count = torch.where(torch.rand(T, device="cuda", generator=g) < holes, 0, count)
    order = torch.rand(T, K, device="cuda", generator=g).argsort(dim=1)       # empty slots anywhere
    ids = torch.where(order < count.unsqueeze(1), ids, -1 - ids)
    return h, W, ids.to(ids_dtype), logits


def _check(h, W, ids, logits, weight=None, tau=1.0, rows=1024):
    refs = ref.distill(h, W, ids, logits, weight, tau, rows)
    got = dict(zip(("loss", "lse", "g_h", "g_W"), mhcl.head_distill_grad(h, W, ids, logits, weight=weight, temperature=tau)))
    for name, (value, bound) in refs.items():
        ref.within(got[name], value, bound, name)
    alone = mhcl.head_distill(h, W, ids, logits, temperature=tau)
    ref.within(alone[0], *refs["loss"], "loss alone")
    ref.within(alone[1], *refs["lse"], "lse alone")
    again = mhcl.head_distill_grad(h, W, ids, logits, weight=weight, temperature=tau)
    assert all(torch.equal(a, b) for a, b in zip(got.values(), again))
    return got


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,C,V,K", [
    (1, 8, 1, 1), (1, 4096, 1000, 64), (2, 64, 2, 3), (16, 264, 127, 256), (33, 72, 1001, 65), (64, 512, 257, 7), (65, 136, 300, 129),
    (130, 1024, 999, 20), (333, 520, 1003, 8), (1000, 64, 40, 100), (40, 128, 30011, 200), (500, 256, 4099, 1), (2049, 72, 8200, 33),
])
def test_distill(io, T, C, V, K):
    _check(*_inputs(T + V, T, C, V, K, io), tau=(1.0, 2.0, 0.5)[(T + K) % 3])


def test_distill_in_the_largest_tiles():
    _check(*_inputs(1, 4100, 72, 4200, 48, BF), tau=2.0)


@pytest.mark.parametrize("io,T,C,V,holes", [(BF, 4200, 2048, 16400, 0.4), (F, 4200, 2048, 16400, 0.0), (BF, 500, 4096, 70000, 0.2), (F, 2049, 4096, 16500, 0.7),
                                            (BF, 2049, 4096, 16500, 1.1)])
def test_products_that_are_large_enough_leave_tokens_out(io, T, C, V, holes):
    h, W, ids, logits = _inputs(T, T, C, V, 17, io, holes=holes)
    weight = torch.rand(T, device="cuda", generator=_gen(4))
    weight[::5] = 0.0
    none = ~(ids >= 0).any(dim=1)
    _check(h, W, ids, logits, None, 2.0)
    got = _check(h, W, ids, logits, weight, 2.0)
    assert not got["g_h"][none].any() and not got["loss"][none].any()
    h[none] = math.nan
    again = mhcl.head_distill_grad(h, W, ids.to(torch.int32), logits, weight, 2.0)
    for name, b in zip(got, again):
        if name == "lse":
            assert torch.equal(got[name][~none], b[~none])
        else:
            assert torch.equal(got[name], b)


@pytest.mark.parametrize("io", [BF, F])
def test_weights_and_types_of_ids_and_logits(io):
    h, W, ids, logits = _inputs(2, 200, 96, 500, 12, io, ids_dtype=torch.int32)
    weight = torch.rand(200, device="cuda", generator=_gen(3)) - 0.3
    weight[::3] = 0.0
    _check(h, W, ids, logits, weight, 3.0)
    half = logits.to(BF)
    _check(h, W, ids, half.float(), weight)
    assert all(torch.equal(a, b) for a, b in zip(mhcl.head_distill_grad(h, W, ids, half, weight), mhcl.head_distill_grad(h, W, ids, half.float(), weight)))


@pytest.mark.parametrize("io", [BF, F])
def test_one_slot_is_the_cross_entropy(io):
    h, W, ids, logits = _inputs(4, 150, 64, 333, 1, io)
    loss, lse = mhcl.head_distill(h, W, ids, logits)
    want, want_lse = mhcl.head_loss(h, W, ids[:, 0].contiguous())
    assert torch.equal(lse, want_lse)
    assert float((loss - want).abs().max()) <= 2.0 ** -21 * float(want.abs().max() + want_lse.abs().max())


@pytest.mark.parametrize("io", [BF, F])
def test_a_student_that_is_its_teacher_has_no_loss(io):
    g = _gen(5)
    h, W = _normal(g, 60, 64, dtype=io), _normal(g, 50, 64, std=0.2, dtype=io)
    z = h.double() @ W.double().t()
    order = torch.rand(60, 50, device="cuda", generator=g).argsort(dim=1)
    loss, _, g_h, g_W = mhcl.head_distill_grad(h, W, order, z.gather(1, order).float())
    scale = mhcl.head_distill_grad(h, W, order, z.flip(1).gather(1, order).float())
    assert float(loss.abs().max()) <= 1e-5
    for got, other in ((g_h, scale[2]), (g_W, scale[3])):
        assert float(got.double().norm()) <= 1e-3 * float(other.double().norm())


@pytest.mark.parametrize("io", [BF, F])
def test_slots_without_a_number(io):
    h, W, ids, logits = _inputs(6, 90, 64, 200, 10, io, short=0.0, holes=0.0)
    logits[3, 4] = -math.inf                   # empty
    logits[4] = -math.inf                      # a token that does not count
    ids[5] = -1
    logits[5] = math.nan                       # (nobody reads it)
    logits[6, 1] = torch.finfo(F).min          # a slot that vanishes
    got = _check(h, W, ids, logits.nan_to_num(0.0, neginf=-math.inf))
    clean = mhcl.head_distill_grad(h, W, ids, logits)
    assert all(torch.equal(a, b) for a, b in zip(got.values(), clean))
    assert not got["loss"][4:6].any() and not got["g_h"][4:6].any()
    # the lowest numbers as a mask: of some slots, and of all, which are then alike, at any temperature
    low = logits.clone()
    low[7, 2:], low[8] = torch.finfo(F).min, torch.finfo(F).min
    for tau in (1.0, 0.5):
        loss, _, g_h, _ = mhcl.head_distill_grad(h, W, ids, low, temperature=tau)
        few, even = low.clone(), low.clone()
        few[7, 2:], even[8] = -math.inf, 0.0
        want = mhcl.head_distill_grad(h, W, ids, few, temperature=tau)
        assert abs(float(loss[7] - want[0][7])) <= 1e-6 * float(loss[7])
        assert float((g_h[7] - want[2][7]).double().norm()) <= 0.01 * float(want[2][7].double().norm())
        want = mhcl.head_distill_grad(h, W, ids, even, temperature=tau)
        assert torch.equal(loss[8], want[0][8]) and torch.equal(g_h[8], want[2][8]) and torch.isfinite(loss[8])
    # mistakes: NaN, infinity, a row past the vocabulary
    logits[10, 2], logits[11, 0], ids[12, 9], ids[13, 9] = math.nan, math.inf, 200, 2 ** 40
    weight = torch.ones(90, device="cuda")
    loss, lse, g_h, g_W = mhcl.head_distill_grad(h, W, ids, logits, weight)
    rest = [t for t in range(90) if t not in (10, 11, 12, 13)]
    assert torch.isnan(loss[10:14]).all() and torch.isnan(g_h[10:14]).all() and torch.isnan(g_W).all()
    assert torch.isfinite(loss[rest]).all() and torch.isfinite(g_h[rest]).all() and torch.isfinite(lse).all()
    weight[10:14] = 0
    loss, _, g_h, g_W = mhcl.head_distill_grad(h, W, ids, logits, weight)
    assert torch.isnan(loss[10:14]).all() and torch.isfinite(g_h).all() and torch.isfinite(g_W).all()


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,C,V", [(90, 64, 200), (1500, 64, 200), (2100, 1024, 65000)])
@pytest.mark.parametrize("mistake", ["nan", "inf", "row"])
def test_each_mistake_alone_is_in_all_of_the_gradient(io, T, C, V, mistake):
    # (the last size takes the tokens in an order of their own)
    h, W, ids, logits = _inputs(12, T, C, V, 10, io, short=0.0)
    at = int((ids >= 0).all(dim=1).nonzero()[3])
    if mistake == "row":
        ids[at, 2] = V
    else:
        logits[at, 2] = math.nan if mistake == "nan" else math.inf
    for weight in (None, torch.ones(T, device="cuda")):
        loss, _, g_h, g_W = mhcl.head_distill_grad(h, W, ids, logits, weight)
        assert torch.isnan(loss[at]) and torch.isnan(g_h[at]).all() and torch.isnan(g_W).all()
        rest = torch.arange(T, device="cuda") != at
        assert torch.isfinite(loss[rest]).all() and torch.isfinite(g_h[rest]).all()
    weight[at] = 0.0
    _, _, g_h, g_W = mhcl.head_distill_grad(h, W, ids, logits, weight)
    assert torch.isfinite(g_h).all() and torch.isfinite(g_W).all()


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T", [50, 1500])
def test_places_that_do_not_count_may_hold_anything(io, T):
    h, W, ids, logits = _inputs(7, T, 128, 300, 6, io)
    weight = torch.ones(T, device="cuda")
    weight[4] = 0.0
    bad = ~(ids >= 0).any(dim=1) | (weight == 0)
    clean = h.clone()
    clean[bad] = 0
    h[bad] = math.nan
    h[int(bad.nonzero()[0])] = math.inf
    _, _, g_h, g_W = mhcl.head_distill_grad(h, W, ids, logits, weight)
    want = mhcl.head_distill_grad(clean, W, ids, logits, weight)
    assert torch.equal(g_h, want[2]) and torch.equal(g_W, want[3])


@pytest.mark.parametrize("io", [BF, F])
def test_without_tokens_and_without_a_teacher(io):
    h, W, ids, logits = _inputs(8, 70, 64, 200, 5, io, holes=1.1)
    got = _check(h, W, ids, logits)
    assert not got["loss"].any() and not got["g_h"].any() and not got["g_W"].any() and torch.isfinite(got["lse"]).all()
    loss, lse, g_h, g_W = mhcl.head_distill_grad(h[:0], W, ids[:0], logits[:0])
    assert loss.shape == lse.shape == (0,) and g_h.shape == (0, 64) and not g_W.any()
    head = mhcl.Head(200, 64, dtype=io)
    total = head.distill(h.requires_grad_(), ids, logits)
    total.backward()
    assert float(total) == 0.0 and not head.W.grad.any() and not h.grad.any()
    assert float(head.distill(h[:0], ids[:0], logits[:0])) == 0.0


def test_large_logits_and_temperatures():
    h, W, ids, logits = _inputs(9, 90, 64, 700, 16, F)
    W = 4 * W
    h[3] *= 20
    h[4] = 0
    for tau in (0.05, 1.0, 50.0):
        _check(h, W, ids, 20 * logits, tau=tau)


@pytest.mark.parametrize("io,C", [(BF, 8), (F, 8), (BF, 128)])
def test_blocks_of_tokens(io, C):
    # a vocabulary so long that a block is of 256 tokens: marks of all of them, lists of a block's; C = 128: in an order of their own
    V = 2 ** 22 - 256
    h, W, ids, logits = _inputs(10, 300, C, V, 4, io)
    ids[:, 0] = torch.where(ids[:, 0] >= 0, V - 1, -1)
    got = dict(zip(("loss", "lse", "g_h", "g_W"), mhcl.head_distill_grad(h, W, ids, logits)))
    W64 = W.double()
    held = ids >= 0
    counted = int(held.any(dim=1).sum())
    g_W = torch.zeros_like(W64)
    for t0 in range(0, 300, 50):
        b = slice(t0, t0 + 50)
        logq = torch.log_softmax(h[b].double() @ W64.t(), dim=1)
        p = torch.softmax(logits[b].double().masked_fill(~held[b], -1e300), dim=1).masked_fill(~held[b], 0.0)
        at = ids[b].clamp(min=0)
        loss = torch.special.xlogy(p, p).sum(dim=1) - (p * logq.gather(1, at)).sum(dim=1)
        assert float((got["loss"][b] - loss).abs().max()) <= 1e-4
        g = logq.exp_().scatter_add_(1, at, -p) * (held[b].any(dim=1).double() / counted).unsqueeze(1)
        want = g @ W64
        assert float((got["g_h"][b].double() - want).norm()) <= (0.01 if io is BF else 1e-4) * float(want.norm())
        g_W += g.t() @ h[b].double()
    assert float((got["g_W"].double() - g_W).norm()) <= (0.01 if io is BF else 1e-4) * float(g_W.norm())


def test_gradients_against_differences():
    h, W, ids, logits = _inputs(11, 5, 16, 30, 4, F, holes=0.0)
    weight = torch.rand(5, device="cuda", generator=_gen(12))
    tau = 1.5

    def value(h, W):
        logq = torch.log_softmax(h @ W.t() / tau, dim=1)
        held = ids >= 0
        p = torch.softmax((logits.double() / tau).masked_fill(~held, -1e300), dim=1).masked_fill(~held, 0.0)
        return float(((torch.special.xlogy(p, p) - p * logq.gather(1, ids.clamp(min=0))).sum(dim=1) * weight.double()).sum())

    _, _, g_h, g_W = mhcl.head_distill_grad(h, W, ids, logits, weight, tau)
    at = [h.double(), W.double()]
    for k, grad in enumerate((g_h, g_W)):
        for i in (0, grad.numel() // 3, grad.numel() - 1):
            step = torch.zeros_like(at[k])
            step.view(-1)[i] = 1e-5
            up, down = (value(*(t + sign * step if j == k else t for j, t in enumerate(at))) for sign in (1, -1))
            slope = (up - down) / 2e-5
            assert abs(float(grad.reshape(-1)[i]) - slope) <= 1e-4 * max(1.0, abs(slope))


def test_operands_that_do_not_fit_are_refused():
    h, W, ids, logits = _inputs(13, 9, 64, 40, 3, BF)
    weight = torch.ones(9, device="cuda")
    for args in ((h, W, ids[:-1], logits), (h, W, ids, logits[:, :-1]), (h, W, ids[:, 0], logits[:, 0]), (h, W, ids.float(), logits),
                 (h, W, ids, logits.double()), (h.float()[:, :-8], W, ids, logits), (h, W, ids, logits.cpu()), (h, W, ids, logits, weight[:-1]),
                 (h, W, ids, logits, weight.double())):
        with pytest.raises(ValueError):
            mhcl.head_distill_grad(*args)
    for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf)):
        with pytest.raises(mhcl.MhclError):
            mhcl.head_distill(h, W, ids, logits, **kw)
    with pytest.raises(mhcl.MhclError):
        mhcl.head_distill(h, W.float(), ids, logits)
    with pytest.raises(mhcl.MhclError):
        mhcl.head_distill(h, W, ids[:, :0], logits[:, :0])
    with pytest.raises(mhcl.MhclError):
        mhcl.head_distill(h, W, ids.repeat(1, 100), logits.repeat(1, 100))
    with pytest.raises(ValueError):
        mhcl.head_distill_grad(h, W, ids, logits, dtype=torch.float16)


def test_strided_operands():
    h, W, ids, logits = _inputs(14, 37, 72, 90, 5, BF)
    weight = torch.rand(37, device="cuda", generator=_gen(1))
    want = mhcl.head_distill_grad(h, W, ids, logits, weight)

    def strided(t):
        return torch.empty(*t.shape[:-1], 2 * t.shape[-1], device="cuda", dtype=t.dtype)[..., ::2].copy_(t)

    got = mhcl.head_distill_grad(*(strided(t) for t in (h, W, ids, logits, weight)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("io", [BF, F])
def test_python_and_native_calls_agree(monkeypatch, io):
    h, W, ids, logits = _inputs(15, 45, 64, 136, 7, io)
    weight = torch.rand(45, device="cuda", generator=_gen(1))

    def calls():
        return [*mhcl.head_distill(h, W, ids, logits, 2.0), *mhcl.head_distill_grad(h, W, ids, logits, weight, 2.0),
                *mhcl.head_distill_grad(h, W, ids, logits, dtype=F)]

    quick = calls()
    monkeypatch.setattr(ends, "_native", lambda: None)
    for a, b in zip(quick, calls()):
        assert a.dtype is b.dtype and a.shape == b.shape and torch.equal(a, b)


@pytest.mark.parametrize("io", [BF, F])
def test_under_autograd(io):
    h, W, ids, logits = _inputs(16, 70, 64, 100, 9, io)
    head = mhcl.Head(100, 64, dtype=io)
    with torch.no_grad():
        head.W.copy_(W)
    h.requires_grad_()
    weight = torch.rand(70, device="cuda", generator=_gen(2)).requires_grad_()
    loss, _, g_h, g_W = mhcl.head_distill_grad(h.detach(), W, ids, logits, weight.detach(), 2.0)
    total = head.distill(h, ids, logits, weight, temperature=2.0)
    assert abs(float(total.detach()) - float((loss.double() * weight.detach().double()).sum())) <= 1e-6 * float(loss.abs().sum())
    total.backward()
    assert torch.equal(h.grad, g_h) and torch.equal(head.W.grad, g_W) and torch.equal(weight.grad, loss)
    h.grad = head.W.grad = None
    (0.25 * head.distill(h, ids, logits, weight, temperature=2.0)).backward()
    assert torch.equal(h.grad, g_h * 0.25) and torch.equal(head.W.grad, g_W * 0.25)
    # the mean over the tokens that count
    counted = (ids >= 0).any(dim=1)
    with torch.no_grad():
        mean = head.distill(h, ids, logits)
    plain = mhcl.head_distill(h.detach(), W, ids, logits)[0].double()[counted].mean()
    assert abs(float(mean) - float(plain)) <= 1e-6 * abs(float(plain))
    total = head.distill(h, ids, logits)
    total.backward(retain_graph=True)
    with pytest.raises(RuntimeError):
        total.backward()
    g, = torch.autograd.grad(head.distill(h, ids, logits), h, create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().square().sum().backward()
    with pytest.raises(ValueError):
        head.distill(h, ids, logits.requires_grad_())
    import torch.autograd.forward_ad as fwd
    with fwd.dual_level(), pytest.raises((RuntimeError, NotImplementedError)):
        head.distill(fwd.make_dual(h.detach(), torch.ones_like(h)), ids, logits.detach())


@pytest.mark.parametrize("T,C,V", [(40, 64, 700), (1300, 64, 700), (2100, 2048, 33000)])
def test_captured_and_replayed(T, C, V):
    h, W, ids, logits = _inputs(17, T, C, V, 9, BF)
    h2, _, ids2, logits2 = _inputs(18, T, C, V, 9, BF, holes=0.5)

    def step():
        return mhcl.head_distill_grad(h, W, ids, logits)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        for a, b in ((h, h2), (ids, ids2), (logits, logits2)):
            a.copy_(b if i % 2 else b.flip(0))
        if i == 3:
            ids[T // 4:] = -1          # far fewer tokens than when it was captured
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
