"""The ends' kernels that only large calls reach: the sort by digits and the longer chunks of the embedding's gradient, reads past the
caches, blocks that take several tokens or several whole tiles, products in many parts, several blocks of tokens.

The embedding's sums are of small whole numbers here, exact in fp32, so that every result is known to the bit.  The norm and the head have
the bounds of test_gpu_ends.py, which hold for any size.
"""
import math

import pytest
import torch

import paper_2601_05732_amd as mhcl
import test_gpu_ends as base

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
I64, I32 = torch.int64, torch.int32


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- embedding


def _ids(g, T, V, kind, dtype):
    if kind == "same":
        ids = torch.full((T,), V - 1, device="cuda")
    elif kind == "none":
        ids = torch.full((T,), -1, device="cuda")
    elif kind == "spread":
        ids = torch.randint(0, V, (T,), device="cuda", generator=g)
    elif kind == "falling":
        ids = torch.arange(T - 1, -1, -1, device="cuda") % V
    else:                                               # a few tokens make up much of it
        ids = ((torch.rand(T, device="cuda", generator=g).double() * math.log(V + 1)).exp().long().clamp(1, V) - 1)
    if kind in ("holes", "past"):
        ids = torch.where(torch.rand(T, device="cuda", generator=g) < 0.3, -1 - ids, ids)
    if kind == "past":
        ids = torch.where(torch.rand(T, device="cuda", generator=g) < 0.3, V + ids // 2, ids)
    return ids.to(dtype)


@pytest.mark.parametrize("T,n,C,V,kind,ids_of,io,w", [
    # at most 8192 tokens are ranked; more are sorted by digits: one pass of nine bits up to V = 511 ...
    (8192, 2, 16, 300, "some", I64, BF, BF), (8193, 2, 16, 300, "past", I32, F, F), (8193, 1, 8, 511, "spread", I64, BF, F),
    (8193, 3, 8, 512, "holes", I64, BF, F),
    # ... two, three and four passes; chunks of 16 tokens from 16384 on, of 32 from 32768 on
    (16385, 3, 24, 5000, "holes", I64, BF, BF), (16384, 1, 8, 2 ** 18 - 1, "falling", I64, F, F), (32769, 4, 8, 2 ** 18 + 3, "some", I32, BF, F),
    (32768, 1, 72, 40, "spread", I64, F, BF), (70001, 2, 8, 2 ** 27, "spread", I64, BF, BF),
    # several tiles of 2048 tokens for each of the 64 sorting blocks; a row in thousands of chunks
    (131072, 1, 8, 70000, "some", I64, BF, F), (135170, 1, 8, 70000, "past", I64, BF, F), (200001, 1, 8, 2 ** 18 + 3, "same", I64, BF, F),
    (140000, 2, 8, 600, "none", I32, BF, F), (150001, 1, 8, 9, "falling", I32, F, F),
    # gradients past the size of the caches, read once
    (16385, 4, 264, 1000, "holes", I64, BF, F), (9001, 8, 128, 1000, "some", I64, F, BF), (33001, 2, 264, 5000, "some", I32, BF, BF),
])
def test_embedding_of_many_tokens_to_the_bit(T, n, C, V, kind, ids_of, io, w):
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = _ids(g, T, V, kind, ids_of)
    g_x = torch.randint(-8, 9, (T, n, C), device="cuda", generator=g).to(io)
    held_there = (ids >= 0) & (ids < V)
    rows, at = ids[held_there].long().unique(return_inverse=True)
    sums = torch.zeros(len(rows), C, dtype=torch.float64, device="cuda").index_add_(0, at, 0.5 * g_x[held_there].double().sum(dim=1))
    assert sums.numel() == 0 or float(sums.abs().max()) < 2 ** 23
    got = mhcl.embed_tokens_grad(ids, g_x, V, scale=0.5, dtype=w)
    assert torch.equal(got[rows], sums.to(w))
    into = torch.randint(-8, 9, (V, C), device="cuda", generator=g, dtype=torch.int8).to(w)
    want = (into[rows].double() + sums).to(w)
    untouched = into.clone()
    mhcl.embed_tokens_grad(ids, g_x, V, scale=0.5, into=into)
    assert torch.equal(into[rows], want)
    got[rows] = 0
    into[rows] = untouched[rows] = 0
    assert not got.any() and torch.equal(into, untouched)


@pytest.mark.parametrize("T,V", [(20001, 70), (20001, 300000), (140001, 5000)])
def test_embedding_gradient_adds_in_the_tokens_order(T, V):
    # the same bits from call to call, and those of the tokens of one id alone in the same chunks' order
    g = torch.Generator(device="cuda").manual_seed(V)
    ids, g_x = torch.randint(0, V, (T,), device="cuda", generator=g), torch.randn(T, 2, 16, device="cuda", generator=g)
    first = mhcl.embed_tokens_grad(ids, g_x, V)
    assert all(torch.equal(first, mhcl.embed_tokens_grad(ids, g_x, V)) for _ in range(3))
    ref = torch.zeros(V, 16, dtype=torch.float64, device="cuda").index_add_(0, ids, g_x.double().sum(dim=1))
    size = torch.zeros(V, 16, dtype=torch.float64, device="cuda").index_add_(0, ids, g_x.double().abs().sum(dim=1))
    adds = 1 + 32 + T / V / 16 + 64                     # of a row: its streams, a chunk's tokens, its chunks by four threads
    assert bool(((first.double() - ref).abs() <= adds * 2.0 ** -24 * size + 1e-30).all())


# ---------------------------------------------------------------- norm


@pytest.mark.parametrize("io,T,n,C", [
    # past the size of the last cache: read once
    (BF, 8193, 4, 4104), (F, 8193, 4, 2056), (BF, 1048577, 2, 64), (BF, 2051, 8, 8200), (F, 40001, 3, 600),
    # several tokens a block and a second turn of the backward's 512 blocks; one token a block and more than one turn
    (BF, 4999, 3, 512), (F, 2100, 1, 256), (F, 5000, 5, 24), (BF, 1025, 4, 4096), (BF, 600, 2, 8200), (F, 700, 1, 8200), (F, 1537, 1, 16392),
])
def test_norm(io, T, n, C):
    base.test_norm(io, T, n, C)


# ---------------------------------------------------------------- head


def _workspace(T, C, V, io, tokens, rows, parts_h, parts_w):
    """The workspace of a plan: a block's tokens, the first product's rows of V (tiles of 256 or 128, a partial sum for half a tile), and the parts
    of the products for g_h and g_W."""
    es = 2 if io is BF else 4
    ld = -(-V // rows) * rows
    sizes = [tokens * C * es, tokens * ld * es, tokens * (ld // (rows // 2)) * 8, tokens * 4, 4]
    sizes += [parts * k * C * 4 for parts, k in ((parts_h, tokens), (parts_w, V)) if parts > 1]
    sizes += [V * C * 4] if io is BF and tokens < T else []
    return (sum(-(-s // 256) * 256 for s in sizes) + 1 + 255) // 256 * 256


@pytest.mark.parametrize("io,T,C,V,tokens,rows,parts_h,parts_w", [
    # the largest tile in all products, both gradients in parts, edges in every direction
    (BF, 4097, 4104, 4100, 4097, 256, 3, 3),
    # the same, g_h whole: blocks that stay take several whole tiles
    (BF, 8192, 4096, 4352, 8192, 256, 1, 4),
    # g_h by middle tiles in parts, g_W by large ones
    (BF, 8192, 768, 50257, 8192, 256, 4, 3),
    # neither in parts: 1008 and 4096 tiles, the last of a column with one row of tokens past a whole tile
    (BF, 15873, 4096, 65536, 15873, 256, 1, 1),
    # blocks of tokens, the last one short, whole tiles of g_W that add up
    (BF, 1300, 256, 2 ** 20, 1024, 256, 32, 1),
    # fp32: more than 512 middle tiles of g_W, two of them in C
    (F, 600, 256, 40000, 600, 128, 25, 1), (F, 2048, 768, 50257, 2048, 128, 8, 1),
    # fp32 blocks of tokens
    (F, 1100, 136, 2 ** 19, 1024, 128, 32, 1),
])
def test_head(io, T, C, V, tokens, rows, parts_h, parts_w):
    d = mhcl.EndsDesc(C, T, 1, V, io, io)
    assert mhcl.ends_workspace_bytes(d, mhcl.OP_HEAD_LOSS_GRAD) == _workspace(T, C, V, io, tokens, rows, parts_h, parts_w)
    base._check_head(*base._head_inputs(19, T, C, V, io), rows=128 if V > 2 ** 18 else 1024)


@pytest.mark.parametrize("io,T,C,V", [(BF, 1025, 64, 300), (F, 1025, 64, 300), (BF, 5001, 264, 90), (F, 3001, 72, 1100)])
def test_head_weights_of_more_than_1024_tokens(io, T, C, V):
    # the weights' common factor by a kernel of its own, several turns of its loop and of the total's
    h, W, targets = base._head_inputs(23, T, C, V, io)
    weight = torch.rand(T, device="cuda", generator=base._gen(6))
    weight[::3] = 0.0
    weight[T - 1] = 3.0                                  # the largest, of a late turn
    targets[T - 1] = 1
    loss = base._check_head(h, W, targets, weight)[0]
    head = mhcl.Head(V, C, dtype=io, table=torch.nn.Parameter(W))
    for w in (weight, None):
        there = targets >= 0
        want = float((loss.double() * weight.double())[there].sum() if w is not None else loss.double()[there].mean())
        with torch.enable_grad():
            total = head(h, targets, w)
        assert abs(float(total.detach()) - want) <= 2 ** -23 * abs(want)
