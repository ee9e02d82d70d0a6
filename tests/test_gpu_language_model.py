"""The ends under torch.autograd and the language model that joins them to the layers.

The modules' gradients are the functions' (test_gpu_ends.py holds those to 64 bits); here the wiring is checked: which
gradient goes where, factors, shared tables, what is refused, and that a model learns.
"""
import pytest
import torch

import paper_2601_05732_amd as mhcl
from paper_2601_05732_amd import ends, lm

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=F):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g).to(dtype)


@pytest.mark.parametrize("io,table_dtype", [(BF, F), (F, F), (BF, BF)])
def test_embedding_module(io, table_dtype):
    g = _gen(1)
    emb = mhcl.TokenEmbedding(50, 64, 3, scale=2.0, dtype=io, table_dtype=table_dtype)
    ids = torch.randint(-2, 50, (33,), device="cuda", generator=g)
    x = emb(ids)
    G = _normal(g, *x.shape, dtype=io)
    x.backward(G)
    assert torch.equal(x, mhcl.embed_tokens(emb.table.detach(), ids, 3, 2.0, io))
    assert torch.equal(emb.table.grad, mhcl.embed_tokens_grad(ids, G, 50, 2.0, table_dtype))


def test_norm_module_on_streams_and_on_one_row():
    g = _gen(2)
    norm = mhcl.StreamsNorm(64, eps=1e-5)
    with torch.no_grad():
        norm.gain.copy_(1 + _normal(g, 64, std=0.2))
    for shape in ((21, 3, 64), (21, 64)):
        norm.zero_grad()
        x = _normal(g, *shape, dtype=BF).requires_grad_()
        G = _normal(g, 21, 64, dtype=BF)
        h = norm(x)
        h.backward(G)
        x3 = x.detach().reshape(21, -1, 64)
        assert torch.equal(h, mhcl.streams_norm(x3, norm.gain.detach(), 1e-5))
        g_x, g_gain = mhcl.streams_norm_grad(x3, norm.gain.detach(), G, 1e-5)
        assert torch.equal(x.grad, g_x.reshape(shape)) and torch.equal(norm.gain.grad, g_gain)


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("weighted", [False, True])
def test_head_module(io, weighted):
    g = _gen(3)
    T, V, C = 70, 130, 64
    head = mhcl.Head(V, C, dtype=io, std=0.2)
    h = _normal(g, T, C, dtype=io).requires_grad_()
    targets = torch.randint(-30, V, (T,), device="cuda", generator=g)
    weight = torch.rand(T, device="cuda", generator=g) if weighted else None
    if weighted:
        weight[targets < 0] = float("nan")                  # (not read there)
    loss, _, g_h, g_W = mhcl.head_loss_grad(h.detach(), head.W.detach(), targets, weight)
    total = head(h, targets, weight)
    there = targets >= 0
    want = (loss[there].double() * (weight[there].double() if weighted else 1 / int(there.sum()))).sum()
    assert total.shape == () and abs(float(total) - float(want)) <= 1e-6 * abs(float(want))
    total.backward(retain_graph=True)
    assert torch.equal(h.grad, g_h) and torch.equal(head.W.grad, g_W)
    with pytest.raises(RuntimeError, match="run the head again"):
        total.backward()
    # a factor on the loss, here a power of two: the same gradients times it
    h.grad = head.W.grad = None
    (0.25 * head(h, targets, weight)).backward()
    assert torch.equal(h.grad, g_h * 0.25) and torch.equal(head.W.grad, g_W * 0.25)
    # one that does not need a gradient gets none
    h.grad = head.W.grad = None
    head(h.detach(), targets, weight).backward()
    assert h.grad is None and torch.equal(head.W.grad, g_W)
    # no gradient at all
    with torch.no_grad():
        assert torch.equal(head(h, targets, weight), head(h.detach(), targets, weight))
        assert abs(float(head(h, targets, weight)) - float(want)) <= 1e-5 * abs(float(want))
    assert torch.equal(head.score(h, targets)[0][~there], torch.zeros(int((~there).sum()), device="cuda"))


def test_head_total_without_targets_is_zero():
    head = mhcl.Head(20, 64)
    total = head(torch.ones(5, 64, device="cuda", dtype=BF, requires_grad=True), torch.full((5,), -1, device="cuda"))
    total.backward()
    assert float(total) == 0.0 and not head.W.grad.any()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("count", [1, 7, 8, 1003, 4096 * 2048 + 5])
def test_scale(dtype, count):
    t = _normal(_gen(4), count, dtype=dtype)
    for value in (1.0, 0.375, float("nan")):
        factor = torch.tensor(value, device="cuda")
        got = t.clone()
        mhcl.mhcl_scale(got, factor)
        assert torch.equal(got.nan_to_num(7.0), (t.float() * factor).to(dtype).nan_to_num(7.0))


@pytest.mark.parametrize("case", ["embed", "embed_grad", "into", "norm", "norm_grad", "head", "head_grad"])
def test_python_and_native_calls_agree(monkeypatch, case):
    g = _gen(5)
    T, n, C, V = 40, 2, 64, 90
    table, ids = _normal(g, V, C, dtype=BF), torch.randint(0, V, (T,), device="cuda", generator=g)
    x, h, gain = _normal(g, T, n, C, dtype=BF), _normal(g, T, C, dtype=BF), 1 + _normal(g, C, std=0.1)
    held = _normal(g, V, C)
    call = dict(
        embed=lambda: [mhcl.embed_tokens(table, ids, n, 1.5, F)], embed_grad=lambda: [mhcl.embed_tokens_grad(ids, x, V, 1.5, F)],
        into=lambda: [mhcl.embed_tokens_grad(ids, x, V, into=held.clone())], norm=lambda: [mhcl.streams_norm(x, gain)],
        norm_grad=lambda: mhcl.streams_norm_grad(x, gain, h), head=lambda: mhcl.head_loss(h, table, ids),
        head_grad=lambda: mhcl.head_loss_grad(h, table, ids))[case]
    quick = call()
    monkeypatch.setattr(ends, "_native", lambda: None)
    for a, b in zip(quick, call()):
        assert a.dtype is b.dtype and a.shape == b.shape and torch.equal(a, b)


@pytest.mark.parametrize("tied", [False, True])
def test_gradients_reach_every_parameter(tied):
    net = lm.LanguageModel(60, 64, n=3, layers=2, dtype=F, tied=tied)
    tokens = lm.synthetic_tokens(60, 41)
    loss = net(tokens[:-1], tokens[1:])
    loss.backward()
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in net.parameters())
    assert (net.head.W is net.embedding.table) == tied
    if tied:       # the sum of both uses: against a model whose ends are apart and equal
        apart = lm.LanguageModel(60, 64, n=3, layers=2, dtype=F)
        own = dict(net.named_parameters())
        with torch.no_grad():
            for name, p in apart.named_parameters():
                p.copy_(own["embedding.table" if name == "head.W" else name])
        apart(tokens[:-1], tokens[1:]).backward()
        both = apart.embedding.table.grad + apart.head.W.grad
        assert float((net.head.W.grad - both).abs().max()) <= 1e-6 * float(both.abs().max())


@pytest.mark.parametrize("dtype,tied", [(BF, False), (BF, True), (F, False)])
def test_a_model_learns(dtype, tied):
    torch.manual_seed(0)
    V = 100
    net = lm.LanguageModel(V, 64, n=4, layers=2, dtype=dtype, tied=tied)
    tokens = lm.synthetic_tokens(V, 4 * 512 + 1)
    losses = lm.train(net, tokens, steps=60, batch=512)
    assert torch.isfinite(losses).all()
    assert float(losses[-1]) < 0.5 * float(losses[0])
    scores = net.score(tokens[:512], tokens[1:513])
    assert scores.shape == (512,) and float(scores.mean()) < float(losses[0])
    # one token at a time gives what the batch gives, to the rounding of the batch's and the single token's kernels
    alone = torch.cat([net.score(tokens[t:t + 1], tokens[t + 1:t + 2]) for t in range(5)])
    assert float((alone - scores[:5]).abs().max()) <= (0.25 if dtype is BF else 1e-3)
