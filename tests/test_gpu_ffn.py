"""The gated feed-forward block against its definition in 64 bits, element by element, at the sizes, types and layouts where it can
go wrong; its gradients against differences; under torch.autograd, captured, on another stream.

The bounds (_bounds) are carried through the formulas from the roundings and were fixed before the first run.
"""
import itertools
import math

import pytest
import torch

import paper_2601_05732_amd as mhcl
from paper_2601_05732_amd import ffn, lm

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=F):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _inputs(seed, T, C, H, io):
    g = _gen(seed)
    return (_normal(g, T, C, dtype=io), _normal(g, 2 * H, C, std=1.5 / math.sqrt(C), dtype=io), _normal(g, C, H, std=1 / math.sqrt(H), dtype=io),
            _normal(g, T, C, dtype=io))


def _bounds(x, W_up, W_down, g_y):
    """{name: (result, largest error)} of y, kept, g_x, g_W_up, g_W_down.
      * a sum of products over K: 2^-24 of the sum of their sizes for each of the ceil(K / 32) additions to the fp32 accumulator, six times
        as many for fp32 operands, and 2^-23 for the products of their parts that are left out; or, of few rows, for each of the up to
        eight additions to a lane's sum for every 512 of K (fp32: four for 256) and the six that join the lanes';
      * the sigmoid by the instructions: 2^-23 |G| for the exponent's rounding, an ulp each for exp2 and 1 / v, half a one for the sum, and a
        half for each product after it: 2^-21 + 2^-23 |G| of the result;
      * silu and its derivative have slopes of at most 1.1 and 0.5;
      * a rounding to the type: finfo.eps / 2 of the value;
      * 2 % for products of two errors."""
    bf = x.dtype is BF
    last = torch.finfo(x.dtype).eps / 2

    def summed(K):
        by_tiles, by_lanes = (-(-K // 32) + 1 if bf else 6 * -(-K // 32) + 3), 8 * -(-K // 512) + 6
        return max(by_tiles, by_lanes if len(x) <= 2 else 0) * 2.0 ** -24

    X, Up, Dn, gy = (t.double() for t in (x, W_up, W_down, g_y))
    T, (C, H) = len(X), Dn.shape
    pre = X @ Up.t()
    e_pre = summed(C) * (X.abs() @ Up.abs().t())
    G, U = pre.chunk(2, dim=1)
    e_G, e_U = e_pre.chunk(2, dim=1)
    s = torch.sigmoid(G)
    silu, slope = G * s, s * (1 + G * (1 - s))
    a = silu * U
    rel = 2.0 ** -21 + 2.0 ** -23 * G.abs()

    def e_a(e_G, e_U):
        return 1.1 * e_G * U.abs() + silu.abs() * e_U + (rel + last) * a.abs()

    out = dict(kept=(pre, e_pre))
    y = a @ Dn.t()
    out["y"] = (y, e_a(e_G, e_U) @ Dn.abs().t() + summed(H) * (a.abs() @ Dn.abs().t()) + last * y.abs())
    ga = gy @ Dn
    e_ga = summed(C) * (gy.abs() @ Dn.abs())
    gU, gG = ga * silu, ga * U * slope
    e_gU = e_ga * silu.abs() + 1.1 * ga.abs() * e_G + (rel + last) * gU.abs()
    e_gG = (e_ga * (U * slope).abs() + ga.abs() * e_U * slope.abs() + 0.5 * (ga * U).abs() * e_G
            + (ga * U).abs() * s * (1 + G.abs()) * (2 * rel) + (rel + last) * gG.abs())
    gp, e_gp = torch.cat([gG, gU], dim=1), torch.cat([e_gG, e_gU], dim=1)
    g_x = gp @ Up
    out["g_x"] = (g_x, e_gp @ Up.abs() + summed(2 * H) * (gp.abs() @ Up.abs()) + last * g_x.abs())
    g_up = gp.t() @ X
    out["g_W_up"] = (g_up, e_gp.t() @ X.abs() + summed(T) * (gp.abs().t() @ X.abs()) + last * g_up.abs())
    g_dn = gy.t() @ a
    out["g_W_down"] = (g_dn, gy.abs().t() @ (e_a(e_G, e_U) + summed(T) * a.abs()) + last * g_dn.abs())
    return {k: (v, 1.02 * e) for k, (v, e) in out.items()}


def _within(got, ref, bound, what):
    assert got.shape == ref.shape
    over = (got.double() - ref).abs() / bound.clamp(min=1e-37)
    assert bool((over <= 1).all()), f"{what}: {float(over.max()):.3f} of the bound"


def _check(x, W_up, W_down, g_y):
    y, kept = mhcl.gated_ffn(x, W_up, W_down, keep=True)
    got = dict(zip(("y", "kept", "g_x", "g_W_up", "g_W_down"), (y, kept, *mhcl.gated_ffn_grad(x, W_up, W_down, kept, g_y))))
    for name, (ref, bound) in _bounds(x, W_up, W_down, g_y).items():
        assert got[name].dtype is (F if name == "kept" else x.dtype)
        _within(got[name], ref, bound, name)
    assert torch.equal(y, mhcl.gated_ffn(x, W_up, W_down))
    assert all(torch.equal(a, b) for a, b in zip((got["g_x"], got["g_W_up"], got["g_W_down"]), mhcl.gated_ffn_grad(x, W_up, W_down, kept, g_y)))
    return got


SIZES = [(1, 8, 8), (2, 520, 2056), (2, 8200, 40), (2, 16392, 24), (4, 1032, 1000), (5, 136, 264), (16, 2056, 4104), (64, 520, 1000), (17, 2056, 24), (48, 1000, 520), (1, 4096, 1000), (2, 64, 24), (16, 264, 136), (31, 4096, 8), (33, 72, 1000), (64, 8, 2056), (65, 136, 520), (130, 1024, 264),
         (333, 520, 1000), (1000, 64, 40), (40, 128, 8200), (2049, 72, 264), (777, 2056, 16)]


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,C,H", SIZES)
def test_ffn(io, T, C, H):
    _check(*_inputs(T + C, T, C, H, io))


@pytest.mark.parametrize("T,C,H", [(4104, 72, 4104), (300, 4104, 4104), (4104, 4104, 72)])
def test_ffn_in_the_largest_tiles(T, C, H):
    _check(*_inputs(T, T, C, H, BF))


@pytest.mark.parametrize("io", [BF, F])
def test_ffn_without_rows(io):
    x, up, down, g_y = _inputs(1, 0, 64, 40, io)
    y, kept = mhcl.gated_ffn(x, up, down, keep=True)
    assert y.shape == (0, 64) and kept.shape == (0, 80)
    g_x, g_up, g_down = mhcl.gated_ffn_grad(x, up, down, kept, g_y)
    assert g_x.shape == (0, 64) and not g_up.any() and not g_down.any()


@pytest.mark.parametrize("io", [BF, F])
def test_ffn_of_large_and_vanishing_gates(io):
    x, up, down, g_y = _inputs(2, 70, 64, 40, io)
    x[3] *= 40
    x[4] = 0
    up[:40] *= 4             # gates from about -200 to 200
    _check(x, up, down, g_y)


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T", [40, 700])
def test_a_row_that_is_not_finite_stays_alone(io, T):
    x, up, down, g_y = _inputs(3, T, 128, 72, io)
    clean = mhcl.gated_ffn(x, up, down)
    bad = [0, 17, T - 1]
    x[bad] = torch.tensor([math.nan, math.inf, -math.inf], device="cuda", dtype=io).unsqueeze(1)
    y, kept = mhcl.gated_ffn(x, up, down, keep=True)
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[bad] = False
    assert torch.equal(y[rest], clean[rest]) and not torch.isfinite(y[bad]).any()
    g_x, g_up, g_down = mhcl.gated_ffn_grad(x, up, down, kept, g_y)
    assert torch.isfinite(g_x[rest]).all() and torch.isnan(g_up).all() and torch.isnan(g_down).all()


@pytest.mark.parametrize("io", [BF, F])
def test_strided_and_unaligned_operands(io):
    x, up, down, g_y = _inputs(4, 37, 72, 48, io)

    def odd(t):          # dense, but one number past a 16-byte boundary
        return torch.empty(t.numel() + 1, device="cuda", dtype=t.dtype)[1:].view(t.shape).copy_(t)

    def strided(t):      # every other column
        return torch.empty(t.shape[0], 2 * t.shape[1], device="cuda", dtype=t.dtype)[:, ::2].copy_(t)

    def turned(t):
        return t.t().contiguous().t()

    y, kept = mhcl.gated_ffn(x, up, down, keep=True)
    grads = mhcl.gated_ffn_grad(x, up, down, kept, g_y)
    for f in (odd, strided, turned):
        args = [f(t) for t in (x, up, down)]
        assert torch.equal(mhcl.gated_ffn(*args), y)
        again = mhcl.gated_ffn_grad(*args, f(kept), f(g_y))
        assert all(torch.equal(a, b) for a, b in zip(grads, again))


def test_operands_that_do_not_fit_are_refused():
    x, up, down, g_y = _inputs(5, 9, 64, 40, BF)
    _, kept = mhcl.gated_ffn(x, up, down, keep=True)
    for args in ((x, up[:-2], down), (x, up, down[:, :-8]), (x[:, :-8], up, down), (x.float(), up, down), (x, up.float(), down), (x[0], up, down)):
        with pytest.raises(ValueError):
            mhcl.gated_ffn(*args)
    for args in ((kept[:-1], g_y), (kept[:, :-8], g_y), (kept.to(BF), g_y), (kept, g_y[:-1]), (kept, g_y.float()), (kept, g_y.cpu())):
        with pytest.raises(ValueError):
            mhcl.gated_ffn_grad(x, up, down, *args)
    with pytest.raises(mhcl.MhclError):          # widths that are no multiple of 8
        mhcl.gated_ffn(x[:, :60].contiguous(), up[:, :60].contiguous(), down[:60].contiguous())


@pytest.mark.parametrize("io", [BF, F])
def test_python_and_native_calls_agree(monkeypatch, io):
    x, up, down, g_y = _inputs(6, 45, 64, 136, io)

    def calls():
        y, kept = mhcl.gated_ffn(x, up, down, keep=True)
        return [mhcl.gated_ffn(x, up, down), y, kept, *mhcl.gated_ffn_grad(x, up, down, kept, g_y)]

    quick = calls()
    monkeypatch.setattr(ffn, "_native", lambda: None)
    for a, b in zip(quick, calls()):
        assert a.dtype is b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_gradients_against_differences():
    x, up, down, g_y = _inputs(7, 3, 16, 8, F)

    def value(x, up, down):
        G, U = (x @ up.t()).chunk(2, dim=1)
        return float((g_y.double() * ((G * torch.sigmoid(G) * U) @ down.t())).sum())

    _, kept = mhcl.gated_ffn(x, up, down, keep=True)
    grads = mhcl.gated_ffn_grad(x, up, down, kept, g_y)
    at = [x.double(), up.double(), down.double()]
    for k, grad in enumerate(grads):
        for i in (0, grad.numel() // 3, grad.numel() - 1):
            step = torch.zeros_like(at[k])
            step.view(-1)[i] = 1e-5
            up_, dn_ = (value(*(t + sign * step if j == k else t for j, t in enumerate(at))) for sign in (1, -1))
            slope = (up_ - dn_) / 2e-5
            assert abs(float(grad.reshape(-1)[i]) - slope) <= 1e-4 * max(1.0, abs(slope))


def test_under_autograd():
    g = _gen(8)
    net = mhcl.GatedFeedForward(64, 40)
    x = _normal(g, 3, 11, 64, dtype=BF).requires_grad_()
    G = _normal(g, 3, 11, 64, dtype=BF)
    y = net(x)
    y.backward(G)
    flat = x.detach().view(33, 64)
    ref, kept = mhcl.gated_ffn(flat, net.W_up.detach(), net.W_down.detach(), keep=True)
    grads = mhcl.gated_ffn_grad(flat, net.W_up.detach(), net.W_down.detach(), kept, G.view(33, 64))
    assert torch.equal(y.detach(), ref.view(3, 11, 64))
    assert torch.equal(x.grad, grads[0].view(3, 11, 64)) and torch.equal(net.W_up.grad, grads[1]) and torch.equal(net.W_down.grad, grads[2])
    with torch.no_grad():
        assert torch.equal(net(x), ref.view(3, 11, 64))
    # the gradient of an expanded result
    net(x).sum().backward()
    # a second derivative is refused, and a forward-mode tangent
    g_x, = torch.autograd.grad(net(x).float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g_x.float().sum().backward()
    import torch.autograd.forward_ad as fwd
    with fwd.dual_level(), pytest.raises((RuntimeError, NotImplementedError)):
        net(fwd.make_dual(x.detach(), torch.ones_like(x)))


@pytest.mark.parametrize("T", [5, 600])
def test_captured_and_replayed(T):
    x, up, down, g_y = _inputs(9, T, 136, 264, BF)
    x2, _, _, g2 = _inputs(10, T, 136, 264, BF)

    def step():
        y, kept = mhcl.gated_ffn(x, up, down, keep=True)
        return [y, *mhcl.gated_ffn_grad(x, up, down, kept, g_y)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.copy_(x2 if i % 2 else x2.flip(0))
        g_y.copy_(g2 if i % 2 else g2.flip(0))
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


def test_on_another_stream():
    x, up, down, g_y = _inputs(11, 200, 264, 136, BF)
    ref, kept_ref = mhcl.gated_ffn(x, up, down, keep=True)
    refs = mhcl.gated_ffn_grad(x, up, down, kept_ref, g_y)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    out = []
    for side in sides * 3:       # two at once
        with torch.cuda.stream(side):
            y, kept = mhcl.gated_ffn(x, up, down, keep=True)
            out.append([y, *mhcl.gated_ffn_grad(x, up, down, kept, g_y)])
    torch.cuda.synchronize()
    for got in out:
        assert all(torch.equal(a, b) for a, b in zip(got, [ref, *refs]))


@pytest.mark.parametrize("io", [BF, F])
def test_the_model_s_block_is_the_feed_forward_block(io):
    block = lm.Block(64, 40, io, "cuda")
    h = _normal(_gen(12), 50, 64, dtype=io).requires_grad_()
    y = block(h)
    y.backward(torch.ones_like(y))
    norm = block.norm(h.detach()).detach()
    ref, kept = mhcl.gated_ffn(norm, block.up.weight.detach(), block.down.weight.detach(), keep=True)
    grads = mhcl.gated_ffn_grad(norm, block.up.weight.detach(), block.down.weight.detach(), kept, torch.ones_like(ref))
    assert torch.equal(y.detach(), ref) and torch.equal(block.up.weight.grad, grads[1]) and torch.equal(block.down.weight.grad, grads[2])
    assert sorted(block.state_dict()) == ["down.weight", "norm.gain", "up.weight"]


def test_blocks_that_the_kernels_do_not_take_run_as_they_are():
    h = _normal(_gen(13), 50, 64, dtype=BF)
    for hidden in (40, 20):                      # 20: no multiple of 8
        block = lm.Block(64, hidden, BF, "cuda")
        norm = block.norm(h)
        a, b = block.up(norm).chunk(2, dim=-1)
        ref = block.down(torch.nn.functional.silu(a) * b).double()
        assert float((block(h).double() - ref).norm()) <= 0.02 * float(ref.norm())
    # maps in place of the block's own, and maps that something looks at
    block.up = torch.nn.Linear(64, 80, device="cuda", dtype=BF)
    block.down = torch.nn.Linear(40, 64, bias=False, device="cuda", dtype=BF)
    with torch.no_grad():
        block.up.bias.fill_(3.0)
    a, b = block.up(norm).chunk(2, dim=-1)
    assert torch.equal(block(h), block.down(torch.nn.functional.silu(a) * b))
    block, seen = lm.Block(64, 40, BF, "cuda"), []
    block.down.register_forward_hook(lambda *args: seen.append(1))
    block(h)
    assert seen == [1]


def test_a_map_s_own_forward_is_called():
    h = _normal(_gen(14), 50, 64, dtype=BF)
    block = lm.Block(64, 40, BF, "cuda")
    before, ours = block(h), block.down.forward
    block.down.forward = lambda x: ours(x) + 1.0
    a, b = block.up(block.norm(h)).chunk(2, dim=-1)
    assert torch.equal(block(h), block.down(torch.nn.functional.silu(a) * b)) and float((block(h) - before).float().mean()) > 0.9


ASKED = [w for w in itertools.product((False, True), repeat=3) if any(w)]


@pytest.mark.parametrize("io,T,C,H", [(io, *s) for io in (BF, F) for s in [(1, 64, 24), (5, 136, 264), (65, 136, 520), (333, 520, 1000), (2049, 72, 264), (40, 128, 8200)]]
                         + [(BF, 4104, 72, 4104), (BF, 300, 4104, 4104), (BF, 4104, 4104, 72)])
def test_gradients_that_are_asked_for(monkeypatch, io, T, C, H):
    x, up, down, g_y = _inputs(T + H, T, C, H, io)
    _, kept = mhcl.gated_ffn(x, up, down, keep=True)
    every = mhcl.gated_ffn_grad(x, up, down, kept, g_y)
    again = mhcl.gated_ffn_grad(x, up, down, kept, g_y, (True, True, True))
    assert all(torch.equal(a, b) for a, b in zip(every, again))
    for native in (True, False):
        if not native:
            monkeypatch.setattr(ffn, "_native", lambda: None)
        for wanted in ASKED:
            some = mhcl.gated_ffn_grad(x, up, down, kept, g_y, wanted)
            assert all(torch.equal(a, b) if w else b is None for a, b, w in zip(every, some, wanted)), wanted


@pytest.mark.parametrize("io", [BF, F])
def test_gradients_of_frozen_weights(io):
    T, C, H = 70, 64, 40
    x, up, down, g_y = _inputs(15, T, C, H, io)
    _, kept = mhcl.gated_ffn(x, up, down, keep=True)
    every = mhcl.gated_ffn_grad(x, up, down, kept, g_y)
    for wanted in ASKED:
        net = mhcl.GatedFeedForward(C, H, dtype=io)
        with torch.no_grad():
            net.W_up.copy_(up)
            net.W_down.copy_(down)
        net.W_up.requires_grad_(wanted[1])
        net.W_down.requires_grad_(wanted[2])
        own = x.clone().requires_grad_(wanted[0])
        net(own).backward(g_y)
        for got, want, w in zip((own.grad, net.W_up.grad, net.W_down.grad), every, wanted):
            assert torch.equal(got, want) if w else got is None, wanted
    none = x[:0]
    for wanted in ASKED:
        g = mhcl.gated_ffn_grad(none, up, down, kept[:0], none, wanted)
        assert all((t is None) if not w else not t.any() for t, w in zip(g, wanted))


# few rows against more outputs than a unit has blocks of sixteen for: of the second product (C > 4096), and in fp32 of the first one (H > 4096)
@pytest.mark.parametrize("io,T,C,H", [(io, *s) for io in (BF, F) for s in [(31, 4104, 136), (64, 4104, 1000), (33, 8200, 264), (3, 4104, 72), (17, 32768, 8)]]
                         + [(F, 20, 4096, 4104), (F, 64, 4096, 4104), (F, 64, 4104, 4104), (F, 16, 520, 4112)])
def test_few_rows_and_many_outputs(io, T, C, H):
    _check(*_inputs(T + C, T, C, H, io))


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T", [0, 40, 700])
def test_the_call_that_forms_every_gradient(io, T):
    x, up, down, g_y = _inputs(16, T, 72, 136, io)
    _, kept = mhcl.gated_ffn(x, up, down, keep=True)
    d = mhcl.FfnDesc(72, 136, T, io)
    got = [torch.full_like(t, math.nan) for t in (x, up, down)]
    ws = torch.empty(mhcl.ffn_workspace_bytes(d, mhcl.OP_FFN_GRAD), dtype=torch.uint8, device="cuda")
    mhcl.mhcl_ffn_grad(d, x, up, down, kept, g_y, *got, ws)
    assert all(torch.equal(a, b) for a, b in zip(got, mhcl.gated_ffn_grad(x, up, down, kept, g_y)))
    if T:
        with pytest.raises(mhcl.MhclError):
            mhcl.mhcl_ffn_grad(d, x, up, down, kept, g_y, None, *got[1:], ws)
