"""The two ends of a language model (embedding, norm of the streams' sum, head with cross entropy) against their
definitions in 64 bits, at the sizes, types, masks and layouts where they can go wrong.

Tolerances, fixed before the first run:
  * embedding and norm, of max |got - ref| / max(|ref|, rms(ref)): fp32 results 1e-5, the repository's bound for fp32 paths; bf16
    results, fp32 values rounded once, 2^-8, twice a rounding to nearest.
  * head: a bound for every element, carried through the formulas from the roundings (_head64 below).
"""
import math

import pytest
import torch

import paper_2601_05732_amd as mhcl

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
ONCE = 2.0 ** -8


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0, dtype=F):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _err(got, ref):
    assert got.shape == ref.shape
    if ref.numel() == 0:
        return 0.0
    got = got.double()
    rms = ref.square().mean().sqrt().clamp(min=1e-300)
    return float(((got - ref).abs() / torch.maximum(ref.abs(), rms)).max())


def _check(got, ref, tol, what=""):
    e = _err(got, ref)
    assert e <= tol, f"{what}: {e:.3e} > {tol:.1e}"


# ---------------------------------------------------------------- embedding


def _embed64(table, ids, n, scale):
    V = table.shape[0]
    ok = (ids >= 0) & (ids < V)
    rows = torch.zeros(len(ids), table.shape[1], dtype=torch.float64, device="cuda")
    rows[ok] = table.double()[ids[ok].long()] * scale
    rows[ids >= V] = math.nan
    return rows.unsqueeze(1).repeat(1, n, 1)


def _embed_grad64(ids, g_x, V, scale):
    ok = (ids >= 0) & (ids < V)
    out = torch.zeros(V, g_x.shape[2], dtype=torch.float64, device="cuda")
    out.index_put_((ids[ok].long(),), g_x.double().sum(dim=1)[ok] * scale, accumulate=True)
    return out


def _ids(g, T, V, kind, dtype):
    if kind == "same":
        return torch.full((T,), V - 1, device="cuda", dtype=dtype)
    if kind == "none":
        return torch.full((T,), -1, device="cuda", dtype=dtype)
    u = torch.rand(T, device="cuda", generator=g)
    ids = ((u.double() * math.log(V + 1)).exp().long().clamp(1, V) - 1).to(dtype)     # a few tokens make up much of it
    if kind == "holes":
        ids = torch.where(torch.rand(T, device="cuda", generator=g) < 0.3, -1 - ids, ids)
    return ids


@pytest.mark.parametrize("io,w", [(BF, BF), (BF, F), (F, F), (F, BF)])
@pytest.mark.parametrize("T,n,C,V,kind", [
    (1, 1, 8, 1, "same"), (1, 4, 4096, 5000, "some"), (15, 4, 64, 7, "some"), (16, 3, 72, 40, "holes"),
    (17, 2, 136, 1000, "same"), (300, 8, 24, 257, "holes"), (1000, 4, 512, 333, "same"), (999, 1, 2056, 50, "some"),
    (4097, 5, 40, 65536, "holes"), (70, 4, 256, 90, "none"),
])
def test_embedding(io, w, T, n, C, V, kind):
    g = _gen(T + C)
    scale = 1.75
    table, ids = _normal(g, V, C, dtype=w), _ids(g, T, V, kind, torch.int64 if T % 2 else torch.int32)
    g_x = _normal(g, T, n, C, dtype=io)
    x = mhcl.embed_tokens(table, ids, n, scale=scale, dtype=io)
    assert x.dtype is io
    _check(x, _embed64(table, ids, n, scale), ONCE if io is BF else 1e-6, "x")
    ref = _embed_grad64(ids, g_x, V, scale)
    got = mhcl.embed_tokens_grad(ids, g_x, V, scale=scale, dtype=w)
    assert got.dtype is w
    _check(got, ref, ONCE if w is BF else 1e-5, "g_table")
    assert torch.equal(got, mhcl.embed_tokens_grad(ids, g_x, V, scale=scale, dtype=w))
    # added to what is there
    held = _normal(g, V, C, dtype=w)
    into = held.clone()
    assert mhcl.embed_tokens_grad(ids, g_x, V, scale=scale, into=into) is into
    _check(into, held.double() + ref, ONCE if w is BF else 1e-5, "accumulated")
    absent = torch.ones(V, dtype=torch.bool, device="cuda")
    absent[ids[(ids >= 0)].long()] = False
    assert torch.equal(into[absent], held[absent])
    assert not got[absent].any()


def test_embedding_tokens_out_of_the_vocabulary():
    g = _gen(3)
    V, C, T, n = 50, 64, 100, 2
    table, g_x = _normal(g, V, C, dtype=BF), _normal(g, T, n, C, dtype=BF)
    ids = torch.arange(T, device="cuda") % 47
    ids[5], ids[77], ids[3], ids[99] = V, 2 ** 40, -1, -(2 ** 40)
    x = mhcl.embed_tokens(table, ids, n)
    ref = _embed64(table, ids, n, 1.0)
    assert torch.isnan(x[[5, 77]]).all() and not x[[3, 99]].any()
    assert torch.equal(x.double()[~torch.isnan(ref)], ref[~torch.isnan(ref)])
    _check(mhcl.embed_tokens_grad(ids, g_x, V, dtype=F), _embed_grad64(ids, g_x, V, 1.0), 1e-5)


def test_embedding_gradient_does_not_read_what_holds_no_token():
    g = _gen(4)
    ids = torch.tensor([3, -1, 2, 9, 3], device="cuda")
    g_x = _normal(g, 5, 2, 16)
    g_x[1] = math.nan
    g_x[3] = math.inf
    got = mhcl.embed_tokens_grad(ids, g_x, 9)          # 9 is out of the vocabulary
    _check(got, _embed_grad64(ids, g_x, 9, 1.0), 1e-5)


# ---------------------------------------------------------------- norm


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,n,C", [
    (1, 4, 4096), (1, 1, 8), (7, 3, 64), (5, 2, 264), (130, 4, 512), (33, 5, 776), (600, 1, 1024), (9, 8, 2048), (3, 4, 2056),
    (1030, 2, 256), (4, 4, 8200), (2, 1, 16392), (3, 2, 32768),
])
def test_norm(io, T, n, C):
    g = _gen(T * C)
    eps = 1e-5
    x, g_h, gain = _normal(g, T, n, C, dtype=io), _normal(g, T, C, dtype=io), 1 + _normal(g, C, std=0.2)
    x64, gain64 = x.double().requires_grad_(), gain.double().requires_grad_()
    s = x64.sum(dim=1)
    h = gain64 * s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt()
    ref_x, ref_gain = torch.autograd.grad(h, [x64, gain64], g_h.double())
    tol = ONCE if io is BF else 1e-5
    _check(mhcl.streams_norm(x, gain, eps=eps), h.detach(), tol, "h")
    g_x, g_gain = mhcl.streams_norm_grad(x, gain, g_h, eps=eps)
    _check(g_x, ref_x, tol, "g_x")
    _check(g_gain, ref_gain, 1e-5, "g_gain")


def test_norm_gradient_against_differences():
    g = _gen(9)
    T, n, C, eps = 3, 2, 16, 1e-3
    x, g_h, gain = _normal(g, T, n, C), _normal(g, T, C), 1 + _normal(g, C, std=0.2)
    g_x, g_gain = mhcl.streams_norm_grad(x, gain, g_h, eps=eps)

    def value(x64, gain64):
        s = x64.sum(dim=1)
        return (g_h.double() * gain64 * s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt()).sum()

    step = 1e-5
    for t, i, c in [(0, 0, 0), (1, 1, 7), (2, 0, 15)]:
        d = torch.zeros_like(x, dtype=torch.float64)
        d[t, i, c] = step
        slope = (value(x.double() + d, gain.double()) - value(x.double() - d, gain.double())) / (2 * step)
        assert abs(float(g_x[t, i, c]) - float(slope)) <= 1e-4 * max(1.0, abs(float(slope)))
    d = torch.zeros_like(gain, dtype=torch.float64)
    d[5] = step
    slope = (value(x.double(), gain.double() + d) - value(x.double(), gain.double() - d)) / (2 * step)
    assert abs(float(g_gain[5]) - float(slope)) <= 1e-4 * max(1.0, abs(float(slope)))


def test_norm_of_zeros_is_zero():
    x, gain = torch.zeros(3, 2, 64, device="cuda", dtype=BF), torch.ones(64, device="cuda")
    assert not mhcl.streams_norm(x, gain).any()
    g_x, g_gain = mhcl.streams_norm_grad(x, gain, torch.ones(3, 64, device="cuda", dtype=BF))
    assert torch.isfinite(g_x).all() and not g_gain.any()


# ---------------------------------------------------------------- head


def _head64(h, W, targets, weight, rows=1024):
    """loss, lse, g_h, g_W and for each the largest error that its roundings allow:
      * a sum of products over K: 2^-24 of the sum of their sizes for each of the ceil(K / 32) additions to the fp32 accumulator, six times
        as many for fp32 operands, and 2^-23 for the products of their parts that are left out; for a logit at most e_z in a row;
      * lse: e_z and 2^-22 of itself, loss with the target's logit besides;
      * a probability, relative: 2 e_z, and 2^-21 for each unit of |z - lse| and |lse| that goes through an exponential in fp32;
      * g: the probability's error, for bf16 also 2^-11 of it (numerators of 10 bits; none below 2^-63) and 2^-8 of g, its rounding;
      * g_h, g_W: those errors times |W|, |h|, that of the sum of |g| |W|, |g| |h|, and the rounding of the result."""
    bf = h.dtype is BF

    def summed(K):
        return (-(-K // 32) + 1) * 2.0 ** -24 if bf else (6 * -(-K // 32) + 3) * 2.0 ** -24

    V = W.shape[0]
    W64 = W.double()
    out = {k: [] for k in ("loss", "lse", "g_h", "e_loss", "e_lse", "e_h")}
    g_W, e_W = torch.zeros_like(W64), torch.zeros_like(W64)
    last = 2.0 ** -8 if bf else 2.0 ** -23
    for t0 in range(0, len(h), rows):
        x, y, w = h[t0:t0 + rows].double(), targets[t0:t0 + rows].long(), weight[t0:t0 + rows].double()
        z = x @ W64.t()
        e_z = summed(h.shape[1]) * (x.abs() @ W64.abs().t()).amax(dim=1)
        lse = torch.logsumexp(z, dim=1)
        counts = y >= 0
        hit = torch.nn.functional.one_hot(y.clamp(min=0), V).double() * counts.unsqueeze(1)
        z_y = z.gather(1, y.clamp(min=0).unsqueeze(1)).squeeze(1)
        out["lse"].append(lse)
        out["loss"].append(torch.where(counts, lse - z_y, 0.0))
        out["e_lse"].append(e_z + 2.0 ** -22 * (1 + lse.abs()))
        out["e_loss"].append(2 * e_z + 2.0 ** -22 * (1 + lse.abs() + z_y.abs()))
        w = torch.where(counts, w, 0.0).unsqueeze(1)
        away = z - lse.unsqueeze(1)
        p = torch.exp(away)
        g = (p - hit) * w
        rel = 2 * e_z.unsqueeze(1) + 2.0 ** -21 * (1 + away.abs() + lse.abs().unsqueeze(1)) + (2.0 ** -11 if bf else 0.0)
        e_g = w.abs() * (p * rel + 2.0 ** -63) + last * g.abs()
        on = (w != 0).squeeze(1)
        gone = ~on.unsqueeze(1)
        g, e_g, x = g.masked_fill(gone, 0.0), e_g.masked_fill(gone, 0.0), x.masked_fill(gone, 0.0)
        out["g_h"].append(g @ W64)
        out["e_h"].append((e_g + summed(V) * g.abs()) @ W64.abs())
        g_W += g.t().contiguous() @ x
        e_W += (e_g + summed(len(h)) * g.abs()).t().contiguous() @ x.abs()
    out = {k: torch.cat(v) for k, v in out.items()}
    out["e_h"] += last * out["g_h"].abs()
    return (out["loss"], out["lse"], out["g_h"], g_W), (out["e_loss"], out["e_lse"], out["e_h"], e_W + last * g_W.abs())


def _head_inputs(seed, T, C, V, io, holes=0.2, std=None):
    g = _gen(seed)
    h, W = _normal(g, T, C, dtype=io), _normal(g, V, C, std=std or 1.5 / math.sqrt(C), dtype=io)
    targets = torch.randint(0, V, (T,), device="cuda", generator=g)
    return h, W, torch.where(torch.rand(T, device="cuda", generator=g) < holes, -100, targets)


def _within(got, ref, bound, what):
    assert got.shape == ref.shape
    over = (got.double() - ref).abs() / bound.clamp(min=1e-45)
    assert bool((over <= 1).all()), f"{what}: {float(over.max()):.3f} of the bound"


def _check_head(h, W, targets, weight=None, rows=1024):
    mean = 1.0 / max(1, int((targets >= 0).sum()))
    w = torch.full((len(h),), mean, device="cuda", dtype=torch.float64) if weight is None else weight
    refs, bounds = _head64(h, W, targets, w, rows)
    got = mhcl.head_loss_grad(h, W, targets, weight)
    for name, a, b, e in zip(("loss", "lse", "g_h", "g_W"), got, refs, bounds):
        _within(a, b, e, name)
    alone = mhcl.head_loss(h, W, targets)
    _within(alone[0], refs[0], bounds[0], "loss alone")
    _within(alone[1], refs[1], bounds[1], "lse alone")
    again = mhcl.head_loss_grad(h, W, targets, weight)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    return got


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,C,V", [
    (1, 8, 1), (1, 4096, 1000), (2, 64, 2), (16, 264, 127), (33, 72, 1001), (64, 512, 257), (65, 136, 300), (130, 1024, 999),
    (333, 520, 1003), (1000, 64, 40), (40, 128, 30011), (500, 256, 4099), (2049, 72, 8200),
])
def test_head(io, T, C, V):
    _check_head(*_head_inputs(T + V, T, C, V, io))


@pytest.mark.parametrize("io", [BF, F])
def test_head_weights_and_token_types(io):
    h, W, targets = _head_inputs(5, 200, 96, 500, io)
    weight = torch.rand(200, device="cuda", generator=_gen(6))
    weight[::3] = 0.0
    _check_head(h, W, targets.to(torch.int32), weight)


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T", [50, 700])
def test_head_places_that_do_not_count_may_hold_anything(io, T):
    h, W, targets = _head_inputs(7, T, 128, 300, io)
    weight = torch.ones(T, device="cuda")
    weight[4] = 0.0
    bad = (targets < 0) | (weight == 0)
    h[bad] = math.nan
    h[int(bad.nonzero()[0])] = math.inf
    clean = h.clone()
    clean[bad] = 0
    _, _, g_h, g_W = mhcl.head_loss_grad(h, W, targets, weight)
    ref = mhcl.head_loss_grad(clean, W, targets, weight)
    assert torch.equal(g_h, ref[2]) and torch.equal(g_W, ref[3])


@pytest.mark.parametrize("io", [BF, F])
def test_head_without_any_target(io):
    h, W, targets = _head_inputs(8, 70, 64, 200, io, holes=1.1)
    loss, lse, g_h, g_W = _check_head(h, W, targets)
    assert not loss.any() and not g_h.any() and not g_W.any() and torch.isfinite(lse).all()


@pytest.mark.parametrize("io", [BF, F])
def test_head_target_out_of_the_vocabulary(io):
    h, W, targets = _head_inputs(9, 70, 64, 200, io)
    targets[11], targets[12] = 200, 2 ** 40
    weight = torch.ones(70, device="cuda")
    loss, lse, g_h, g_W = mhcl.head_loss_grad(h, W, targets, weight)
    assert torch.isnan(loss[[11, 12]]).all() and torch.isnan(g_h[[11, 12]]).all() and torch.isnan(g_W).all()
    rest = [t for t in range(70) if t not in (11, 12)]
    assert torch.isfinite(loss[rest]).all() and torch.isfinite(g_h[rest]).all() and torch.isfinite(lse).all()
    weight[[11, 12]] = 0
    loss, _, g_h, g_W = mhcl.head_loss_grad(h, W, targets, weight)
    assert torch.isnan(loss[[11, 12]]).all() and torch.isfinite(g_h).all() and torch.isfinite(g_W).all()


def test_head_large_and_lowest_logits():
    # logits of some hundreds, one token's all far below the others', numerators that vanish
    h, W, targets = _head_inputs(10, 90, 64, 700, F, std=4.0)
    h[3] *= 20
    h[4] = 0
    _check_head(h, W, targets)
    low = torch.zeros(40, 8, device="cuda")
    low[:, 0] = torch.finfo(F).min / 4                       # every logit at about the lowest value
    loss, lse, g_h, g_W = mhcl.head_loss_grad(low, torch.ones(100, 8, device="cuda"), torch.arange(40, device="cuda"))
    assert torch.isfinite(lse).all() and torch.isfinite(g_W).all()
    assert float((g_h.abs()).max()) <= 1e-6                  # the softmax is even: its mean row is the target's


def test_head_small_probabilities_keep_their_gradient():
    # a row of W whose probability is exp(-30): its gradient is as exact as the others'
    h = torch.ones(64, 16, device="cuda", dtype=BF)
    W = torch.zeros(50, 16, device="cuda", dtype=BF)
    W[7] = -30.0 / 16
    targets = torch.arange(64, device="cuda") % 7
    weight = torch.full((64,), 1 / 64, device="cuda")
    g_W = mhcl.head_loss_grad(h, W, targets, weight)[3]
    ref = _head64(h, W, targets, weight)[0][3]
    assert float(ref[7].abs().max()) < 1e-13
    assert float(((g_W[7].double() - ref[7]) / ref[7]).abs().max()) <= 2 ** -7


def test_head_gradient_against_differences():
    h, W, targets = _head_inputs(12, 9, 16, 33, F)
    weight = torch.rand(9, device="cuda", generator=_gen(1)).double()
    _, _, g_h, g_W = mhcl.head_loss_grad(h, W, targets, weight.float())

    def value(h64, W64):
        z = h64 @ W64.t()
        y = targets.clamp(min=0).unsqueeze(1)
        loss = torch.logsumexp(z, dim=1) - z.gather(1, y).squeeze(1)
        return (torch.where(targets >= 0, loss, 0.0) * weight.float().double()).sum()

    step = 1e-5
    for (a, b), which in [((2, 3), 0), ((8, 15), 0), ((0, 0), 1), ((32, 7), 1)]:
        d = [torch.zeros_like(h, dtype=torch.float64), torch.zeros_like(W, dtype=torch.float64)]
        d[which][a, b] = step
        slope = float(value(h.double() + d[0], W.double() + d[1]) - value(h.double() - d[0], W.double() - d[1])) / (2 * step)
        got = float((g_h, g_W)[which][a, b])
        assert abs(got - slope) <= 1e-4 * max(1.0, abs(slope))


@pytest.mark.parametrize("io,T,V", [(BF, 1300, 2 ** 20), (F, 1100, 2 ** 18 + 5)])
def test_head_blocks_of_tokens(io, T, V):
    # more tokens than a block of the workspace holds: g_W adds up over the blocks
    h, W, targets = _head_inputs(13, T, 16, V, io)
    d = mhcl.EndsDesc(16, T, 1, V, io, io)
    assert mhcl.ends_workspace_bytes(d, mhcl.OP_HEAD_LOSS_GRAD) < 3 * 2 ** 30
    _check_head(h, W, targets, rows=128)


def test_head_blocks_of_tokens_in_fp32():
    h, W, targets = _head_inputs(16, 1100, 16, 2 ** 19 + 5, F)
    d = mhcl.EndsDesc(16, 1100, 1, 2 ** 19 + 5, F, F)
    assert mhcl.ends_workspace_bytes(d, mhcl.OP_HEAD_LOSS_GRAD) < 3 * 2 ** 30
    _check_head(h, W, targets, rows=64)


@pytest.mark.parametrize("io,T,C,V", [(BF, 7001, 64, 130), (BF, 1030, 136, 90), (F, 3003, 264, 190), (F, 2000, 1000, 700), (F, 33, 64, 9001)])
def test_head_few_rows_of_the_vocabulary_or_few_tokens(io, T, C, V):
    # products of few tiles and a long depth, which is split
    _check_head(*_head_inputs(17, T, C, V, io))


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("C", [8, 32, 40, 64, 96, 104, 128, 136, 192, 200, 256, 264, 328])
def test_head_every_remainder_of_the_depth(io, C):
    _check_head(*_head_inputs(C, 37, C, 270, io))


# ---------------------------------------------------------------- how they are called


def test_strided_and_misaligned_tensors():
    g = _gen(20)
    T, n, C, V = 60, 2, 64, 100
    tokens = torch.randint(0, V, (T + 1,), device="cuda", generator=g)
    table = _normal(g, V, 2 * C, dtype=BF)[:, :C]
    x = mhcl.embed_tokens(table, tokens[1:], n)
    assert torch.equal(x, mhcl.embed_tokens(table.contiguous(), tokens[1:].clone(), n))
    wide = _normal(g, T, n, C + 8, dtype=BF)[:, :, 8:]
    g_h, gain = _normal(g, C, T, dtype=BF).t(), 1 + _normal(g, C + 1, std=0.1)[1:]
    assert torch.equal(mhcl.streams_norm(wide, gain), mhcl.streams_norm(wide.contiguous(), gain.clone()))
    for a, b in zip(mhcl.streams_norm_grad(wide, gain, g_h), mhcl.streams_norm_grad(wide.contiguous(), gain.clone(), g_h.contiguous())):
        assert torch.equal(a, b)
    flat = _normal(g, T * C + 1, dtype=BF)
    h = flat[1:].view(T, C)                                   # 2 bytes past an aligned address
    every = torch.stack([tokens, tokens], dim=1)[:, 0]        # every second token in memory
    for a, b in zip(mhcl.head_loss_grad(h, table, every[1:]), mhcl.head_loss_grad(h.clone(), table.contiguous(), tokens[1:].clone())):
        assert torch.equal(a, b)


def test_no_tokens():
    V, C, n = 30, 64, 3
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    table, gain = torch.ones(V, C, device="cuda", dtype=BF), torch.ones(C, device="cuda")
    x = mhcl.embed_tokens(table, ids, n)
    assert x.shape == (0, n, C)
    assert not mhcl.embed_tokens_grad(ids, x, V, dtype=F).any()
    held = torch.ones(V, C, device="cuda")
    assert torch.equal(mhcl.embed_tokens_grad(ids, x, V, into=held.clone()), held)
    h = mhcl.streams_norm(x, gain)
    assert h.shape == (0, C) and not mhcl.streams_norm_grad(x, gain, h)[1].any()
    loss, lse, g_h, g_W = mhcl.head_loss_grad(h, table, ids)
    assert loss.shape == lse.shape == (0,) and g_h.shape == (0, C) and not g_W.any()
    assert mhcl.head_loss(h, table, ids)[0].shape == (0,)


def test_on_another_stream_and_in_a_graph():
    g = _gen(21)
    T, n, C, V = 150, 4, 128, 700
    table, gain = _normal(g, V, C, std=0.1, dtype=BF), 1 + _normal(g, C, std=0.1)
    ids, targets = (torch.randint(0, V, (T,), device="cuda", generator=g) for _ in range(2))

    def step():
        x = mhcl.embed_tokens(table, ids, n)
        h = mhcl.streams_norm(x, gain)
        loss, lse, g_h, g_W = mhcl.head_loss_grad(h, table, targets)
        g_x, g_gain = mhcl.streams_norm_grad(x, gain, g_h)
        return [loss, lse, g_gain, mhcl.embed_tokens_grad(ids, g_x, V, into=g_W)]

    ref = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        ids.copy_(torch.randint(0, V, (T,), device="cuda", generator=g))
        targets.copy_(torch.randint(0, V, (T,), device="cuda", generator=g))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_refusals():
    V, C, T, n = 20, 64, 5, 2
    table, ids = torch.ones(V, C, device="cuda", dtype=BF), torch.zeros(T, dtype=torch.int64, device="cuda")
    x, gain = torch.ones(T, n, C, device="cuda", dtype=BF), torch.ones(C, device="cuda")
    h = torch.ones(T, C, device="cuda", dtype=BF)
    for call in (
        lambda: mhcl.embed_tokens(table.cpu(), ids, n),
        lambda: mhcl.embed_tokens(table, ids.cpu(), n),
        lambda: mhcl.embed_tokens(table.half(), ids, n),
        lambda: mhcl.embed_tokens(table, ids.short(), n),
        lambda: mhcl.embed_tokens(table, ids.view(1, T), n),
        lambda: mhcl.embed_tokens_grad(ids, x[:3], V),
        lambda: mhcl.embed_tokens_grad(ids, x, V, into=torch.ones(V, C + 8, device="cuda")),
        lambda: mhcl.embed_tokens_grad(ids, x, V, into=torch.ones(C, V, device="cuda").t()),
        lambda: mhcl.streams_norm(x, gain[:-1]),
        lambda: mhcl.streams_norm(x, gain.to(BF)),
        lambda: mhcl.streams_norm_grad(x, gain, h.float()),
        lambda: mhcl.head_loss(h, table[:, :-8], ids),
        lambda: mhcl.head_loss(h, table, ids[1:]),
        lambda: mhcl.head_loss_grad(h, table, ids, torch.ones(T, device="cuda", dtype=BF)),
    ):
        with pytest.raises(ValueError):
            call()
    for call in (
        lambda: mhcl.embed_tokens(table, ids, 9),
        lambda: mhcl.embed_tokens(table[:, :12], ids, n),
        lambda: mhcl.embed_tokens(table, ids, n, scale=math.inf),
        lambda: mhcl.streams_norm(x, gain, eps=-1.0),
        lambda: mhcl.head_loss(h, table.float(), ids),                          # types have to agree
        lambda: mhcl.streams_norm(torch.ones(1, 1, 32776, device="cuda", dtype=BF), torch.ones(32776, device="cuda")),
    ):
        with pytest.raises(mhcl.MhclError):
            call()
