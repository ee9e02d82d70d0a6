"""The head's loss of pairs of sequences: against its definition in 64 bits element by element, at the lengths, masks and offsets where it can
go wrong; its gradients against differences; under torch.autograd, captured.  Bounds: head_reference.py."""
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


def _inputs(seed, T, C, V, pairs, io, lead=0, tail=0, holes=0.3, dtype=torch.int64):
    """Ragged sequences, some empty, from `lead` to T - tail; a reference near the sequences' log probabilities."""
    g = _gen(seed)
    h, W = _normal(g, T, C, dtype=io), _normal(g, V, C, std=1.5 / math.sqrt(C), dtype=io)
    targets = torch.randint(0, V, (T,), device="cuda", generator=g)
    targets = torch.where(torch.rand(T, device="cuda", generator=g) < holes, -100, targets)
    cuts = torch.sort(torch.randint(lead, T - tail + 1, (2 * pairs - 1,), device="cuda", generator=g))[0] if pairs else torch.empty(0, device="cuda").long()
    offsets = torch.cat([torch.tensor([lead], device="cuda"), cuts] + ([torch.tensor([T - tail], device="cuda")] if pairs else []))
    logp = torch.zeros(2 * pairs, device="cuda", dtype=torch.float64)
    ce = torch.log_softmax(h.double() @ W.double().t(), dim=1).gather(1, targets.clamp(min=0).unsqueeze(1)).squeeze(1).masked_fill(targets < 0, 0.0)
    for i in range(2 * pairs):
        logp[i] = ce[int(offsets[i]):int(offsets[i + 1])].sum()
    reference = (logp + 10 * _normal(g, 2 * pairs, dtype=torch.float64)).float()
    return h, W, targets, offsets.to(dtype), reference


def _check(h, W, targets, offsets, reference, weight=None, beta=0.1, smoothing=0.0, rows=1024):
    refs = ref.preference(h, W, targets, offsets, reference, weight, beta, smoothing, rows)
    got = dict(zip(("loss", "logp", "g_h", "g_W"), mhcl.head_preference_grad(h, W, targets, offsets, reference, weight, beta, smoothing)))
    for name, (value, bound) in refs.items():
        ref.within(got[name], value, bound, name)
    alone = mhcl.head_preference(h, W, targets, offsets, reference, beta, smoothing)
    ref.within(alone[0], *refs["loss"], "loss alone")
    ref.within(alone[1], *refs["logp"], "logp alone")
    again = mhcl.head_preference_grad(h, W, targets, offsets, reference, weight, beta, smoothing)
    assert all(torch.equal(a, b) for a, b in zip(got.values(), again))
    return got


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,C,V,pairs", [
    (1, 8, 1, 1), (2, 64, 2, 1), (2, 4096, 1000, 1), (16, 264, 127, 9), (33, 72, 1001, 3), (64, 512, 257, 2), (65, 136, 300, 40),
    (130, 1024, 999, 1), (333, 520, 1003, 7), (1025, 64, 40, 2), (40, 128, 30011, 3), (500, 256, 4099, 5), (2049, 72, 8200, 300),
])
def test_preference(io, T, C, V, pairs):
    _check(*_inputs(T + V, T, C, V, pairs, io, lead=T // 7, tail=T // 9), smoothing=0.1 if T % 2 else 0.0)


def test_preference_in_the_largest_tiles():
    _check(*_inputs(1, 4100, 72, 4200, 8, BF, tail=100))


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,C,V,pairs,holes", [(2100, 1024, 8200, 5, 0.3), (5000, 264, 13100, 40, 0.7), (300, 4096, 16000, 2, 0.0), (9000, 72, 27000, 3, 0.3),
                                               (2049, 1032, 8200, 3, 1.1)])
def test_products_that_are_large_enough_leave_tokens_out(io, T, C, V, pairs, holes):
    h, W, targets, offsets, reference = _inputs(T, T, C, V, pairs, io, lead=T // 7, tail=T // 9, holes=holes)
    weight = torch.rand(pairs, device="cuda", generator=_gen(4))
    weight[0] = 0.0
    bad = targets < 0
    bad[:T // 7] = bad[T - T // 9:] = True
    got = _check(h, W, targets, offsets, reference, weight, smoothing=0.1)
    assert not got["g_h"][bad].any()
    h[bad] = math.nan
    again = mhcl.head_preference_grad(h, W, targets.to(torch.int32), offsets.to(torch.int32), reference, weight, 0.1, 0.1)
    assert all(torch.equal(a, b) for a, b in zip(got.values(), again))
    h[bad] = math.inf
    assert torch.equal(mhcl.head_preference(h, W, targets, offsets, reference, smoothing=0.1)[1], mhcl.head_preference_grad(h, W, targets, offsets)[1])


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("dtype", [torch.int64, torch.int32])
def test_weights_types_and_no_reference(io, dtype):
    h, W, targets, offsets, reference = _inputs(2, 700, 96, 500, 6, io, dtype=dtype)
    weight = torch.rand(6, device="cuda", generator=_gen(3)) - 0.3
    weight[2] = 0.0
    _check(h, W, targets.to(torch.int32), offsets, reference, weight, 0.3, 0.25)
    _check(h, W, targets, offsets.to(torch.int32 if dtype is torch.int64 else torch.int64), None, weight, 0.01)
    _check(h, W, targets, offsets, reference, beta=0.0)
    _check(h, W, targets, offsets, reference, beta=-0.2, smoothing=1.0)


@pytest.mark.parametrize("io", [BF, F])
def test_empty_sequences_and_pairs(io):
    h, W, targets, offsets, reference = _inputs(4, 90, 64, 200, 3, io)
    offsets = torch.tensor([10, 10, 40, 40, 40, 70, 70], device="cuda")
    got = _check(h, W, targets, offsets, reference)
    assert not got["logp"][[0, 2, 3, 5]].any()
    outside = torch.ones(90, dtype=torch.bool, device="cuda")
    outside[10:70] = False
    assert not got["g_h"][outside].any()
    # no pair at all, no token at all, no target at all
    loss, logp, g_h, g_W = mhcl.head_preference_grad(h, W, targets, offsets[:1])
    assert loss.shape == (0,) and logp.shape == (0,) and not g_h.any() and not g_W.any()
    loss, logp, g_h, g_W = mhcl.head_preference_grad(h[:0], W, targets[:0], torch.zeros(5, device="cuda", dtype=torch.int64), reference[:4])
    m = 0.1 * (reference[1:4:2] - reference[0:4:2]).double()
    assert float((loss.double() - torch.nn.functional.softplus(-m)).abs().max()) <= 1e-5
    assert not logp.any() and g_h.shape == (0, 64) and not g_W.any()
    got = _check(h, W, torch.full_like(targets, -1), offsets, reference)
    assert not got["g_h"].any() and not got["g_W"].any() and not got["logp"].any()


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T", [80, 1400])
def test_places_that_do_not_count_may_hold_anything(io, T):
    h, W, targets, offsets, reference = _inputs(5, T, 128, 300, 3, io, lead=5, tail=9)
    weight = torch.tensor([1.0, 0.0, 0.5], device="cuda")
    at = torch.arange(T, device="cuda")
    bad = (targets < 0) | (at < offsets[0]) | (at >= offsets[-1]) | ((at >= offsets[2]) & (at < offsets[4]))
    clean = h.clone()
    clean[bad] = 0
    h[bad] = math.nan
    loss, logp, g_h, g_W = mhcl.head_preference_grad(h, W, targets, offsets, reference, weight)
    want = mhcl.head_preference_grad(clean, W, targets, offsets, reference, weight)
    assert torch.equal(g_h, want[2]) and torch.equal(g_W, want[3])
    assert torch.equal(loss[[0, 2]], want[0][[0, 2]]) and torch.equal(logp[[0, 1, 4, 5]], want[1][[0, 1, 4, 5]])


@pytest.mark.parametrize("io", [BF, F])
def test_mistakes_are_loud_and_stay_in_their_pair(io):
    h, W, targets, offsets, reference = _inputs(6, 120, 64, 200, 4, io, holes=0.0)
    offsets = torch.tensor([0, 20, 40, 50, 60, 80, 90, 100, 120], device="cuda")
    good = mhcl.head_preference(h, W, targets, offsets, reference)
    weight = torch.ones(4, device="cuda")
    for change in ("target", "past", "descends", "negative"):
        y, o = targets.clone(), offsets.clone()
        if change == "target":
            y[45] = 200
        elif change == "past":
            o[-1] = 2 ** 40
        elif change == "descends":
            o[-1] = 95
        else:
            o[0] = -3
        pair = dict(target=1, past=3, descends=3, negative=0)[change]
        others = [p for p in range(4) if p != pair]
        loss, logp, g_h, g_W = mhcl.head_preference_grad(h, W, y, o, reference, weight)
        assert torch.isnan(loss[pair]) and torch.equal(loss[others], good[0][others]), change
        assert torch.isnan(g_W).all(), change
        weight[pair] = 0
        _, _, g_h, g_W = mhcl.head_preference_grad(h, W, y, o, reference, weight)
        assert torch.isfinite(g_h).all() and torch.isfinite(g_W).all(), change
        weight[pair] = 1


# offsets [9] of 4 pairs of 120 tokens, and which pairs are mistakes
OUT_OF_ORDER = [
    ([0, 50, 30, 40, 60, 80, 90, 100, 120], [0]),           # pair 1 begins before the middle of pair 0
    ([70, 10, 20, 30, 40, 80, 90, 100, 120], [0]),          # the first one lies inside a later pair
    ([0, 20, 40, 50, 60, 80, 90, 100, 30], [3]),            # the last one before earlier pairs' ends
    ([0, 20, 40, 50, 60, 80, 90, 100, 0], [3]),
    ([5, 20, 40, 50, 60, 80, 90, 100, -5], [3]),
    ([0, 20, 40, 35, 30, 50, 80, 100, 120], [1, 2]),        # pair 2 begins before the end of pair 0
    ([0, 20, 40, 35, 30, 30, 30, 100, 120], [1, 3]),        # pair 2 is empty, and pair 3 begins there
    ([10, 20, 40, 200, 50, 70, 60, 100, 115], [1, 2]),
    ([-9, 20, 2 ** 33, 50, 60, 80, -2 ** 40, 7, 2 ** 62], [0, 1, 2, 3]),
]


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("offsets,bad", OUT_OF_ORDER)
def test_offsets_out_of_order_leave_the_other_pairs_alone(io, offsets, bad):
    _out_of_order(*_inputs(15, 120, 64, 200, 4, io, holes=0.2), offsets, bad)


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("offsets,bad", OUT_OF_ORDER)
def test_offsets_out_of_order_where_products_leave_tokens_out(io, offsets, bad):
    # (how many tokens are left decides into how many parts the sums of g_h are split: not the same bits)
    _out_of_order(*_inputs(17, 4200, 1024, 8200, 4, io, holes=0.4), [35 * o if abs(o) <= 200 else o for o in offsets], bad, same_bits=False)


def _out_of_order(h, W, targets, _, reference, offsets, bad, same_bits=True):
    good = [p for p in range(4) if p not in bad]
    # the same pairs by themselves, where there is a gap before them one of weight 0
    held, clean, at = [], [0], 0
    for p in good:
        empty = offsets[2 * p] == offsets[2 * p + 2]       # (wherever it lies)
        if offsets[2 * p] != at and not empty:
            clean += [at, offsets[2 * p]]
            held.append(None)
        held.append(p)
        clean += [at, at] if empty else offsets[2 * p + 1:2 * p + 3]
        at = clean[-1]
    where = [held.index(p) for p in good]
    rows = torch.zeros(len(h), dtype=torch.bool, device="cuda")
    for p in good:
        rows[offsets[2 * p]:offsets[2 * p + 2]] = True

    def of(values, empty):
        return torch.tensor([empty if p is None else values[p] for p in held], device="cuda", dtype=F)

    halves = reference.view(4, 2)
    weight = [0.3 + p for p in range(4)]
    own = [torch.stack([of(halves[:, i].tolist(), 0.0) for i in range(2)], dim=1).view(-1), of(weight, 0.0)]
    want = mhcl.head_preference_grad(h, W, targets, torch.tensor(clean, device="cuda"), *own, smoothing=0.1)
    refs = ref.preference(h, W, targets, torch.tensor(clean, device="cuda"), *own, 0.1, 0.1)
    for name, value in zip(("loss", "logp", "g_h", "g_W"), want):
        ref.within(value, *refs[name], name)
    o = torch.tensor(offsets, device="cuda")
    for on in (0.0, 1.0):
        w = torch.tensor([on if p in bad else weight[p] for p in range(4)], device="cuda")
        loss, logp, g_h, g_W = got = mhcl.head_preference_grad(h, W, targets, o, reference, w, smoothing=0.1)
        assert torch.isnan(loss[bad]).all() and torch.isnan(logp.view(4, 2)[bad]).all()
        assert torch.equal(loss[good], want[0][where]) and torch.equal(logp.view(4, 2)[good], want[1].view(-1, 2)[where])
        there = rows if on else slice(None)
        ref.within(g_h[there], *(t[there] for t in refs["g_h"]), "g_h")
        assert not same_bits or torch.equal(g_h[there], want[2][there])
        assert on == 0 or torch.isnan(g_W).all()
        if on == 0:
            ref.within(g_W, *refs["g_W"], "g_W")
            assert not same_bits or torch.equal(g_W, want[3])
        alone = mhcl.head_preference(h, W, targets, o, reference, smoothing=0.1)
        for a, b in zip((*got, *alone), (*mhcl.head_preference_grad(h, W, targets, o, reference, w, smoothing=0.1), loss, logp)):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) and torch.equal(a.isnan(), b.isnan())


@pytest.mark.parametrize("io", [BF, F])
@pytest.mark.parametrize("T,C,V", [(120, 64, 200), (1500, 64, 200), (4200, 1024, 8200)])
@pytest.mark.parametrize("offsets,others", [([5, 3, 2], []), ([40, 40, 20], []), ([9, 5, -1, 0, 0], [0.0]), ([20, 10, 0, 0, 60], [1.0])])
def test_a_mistake_without_tokens_is_in_the_gradient(io, T, C, V, offsets, others):
    pairs = len(offsets) // 2
    h, W, targets, _, reference = _inputs(18, T, C, V, pairs, io)
    o = torch.tensor(offsets, device="cuda", dtype=torch.int32)
    for weight in (None, torch.tensor([0.5, 0.0][:pairs], device="cuda")):
        loss, _, g_h, g_W = mhcl.head_preference_grad(h, W, targets, o, reference, weight)
        assert torch.isnan(loss[0]) and torch.isnan(g_W).all()
    loss, _, g_h, g_W = mhcl.head_preference_grad(h, W, targets, o, reference, torch.tensor([0.0] + others, device="cuda"))
    assert torch.isnan(loss[0]) and torch.isfinite(g_h).all() and torch.isfinite(g_W).all()


def test_many_pairs_with_one_out_of_order():
    # more pairs than a block has threads, and than a thread has of them
    for pairs in (513, 1500):
        h, W, targets, offsets, reference = _inputs(16, 2000, 72, 90, pairs, F, lead=3, tail=5)
        weight = torch.rand(pairs, device="cuda", generator=_gen(5))
        weight[pairs // 2] = 0.0
        want = _check(h, W, targets, offsets, reference, weight)
        broken = offsets.clone()
        broken[2 * (pairs // 2) + 1] = 1999        # its middle behind its end
        loss, logp, g_h, g_W = mhcl.head_preference_grad(h, W, targets, broken, reference, weight)
        assert torch.isnan(loss[pairs // 2]) and torch.equal(g_h, want["g_h"]) and torch.equal(g_W, want["g_W"])
        rest = torch.arange(pairs, device="cuda") != pairs // 2
        assert torch.equal(loss[rest], want["loss"][rest]) and torch.equal(logp.view(-1, 2)[rest], want["logp"].view(-1, 2)[rest])


@pytest.mark.parametrize("pairs,near", [(6, 9), (60, 0), (400, 5), (512, 40), (700, 5), (5000, 9), (5000, 300)])
def test_offsets_in_any_order(pairs, near):
    # mostly ascending by little, with some that lie anywhere: which pairs are mistakes, and one writer for every weight
    T = 500
    h, W, targets, _, reference = _inputs(19, T, 64, 90, pairs, F)
    g = torch.Generator().manual_seed(pairs + near)
    offsets = torch.sort(torch.randint(0, T + 1, (2 * pairs + 1,), generator=g))[0]
    away = torch.rand(2 * pairs + 1, generator=g) < near / (2 * pairs + 1)
    offsets = torch.where(away, torch.randint(-5, T + 6, (2 * pairs + 1,), generator=g), offsets)
    o, end, bad, owner = offsets.tolist(), 0, [], torch.full((T,), -1)
    for p in range(pairs):
        a, b, c = o[2 * p:2 * p + 3]
        ascends = 0 <= a <= b <= c <= T
        if not ascends or (a < end and a < c):
            bad.append(p)
        elif a < c:
            owner[a:c] = p
        end = max(end, c) if ascends else end
    weight = torch.rand(pairs, generator=g) + 0.1
    weight[bad] = 0.0
    args = (h, W, targets, offsets.cuda(), reference, weight.cuda())
    loss, _, g_h, g_W = got = mhcl.head_preference_grad(*args)
    isnan = torch.zeros(pairs, dtype=torch.bool)
    isnan[bad] = True
    assert torch.equal(loss.isnan().cpu(), isnan) and torch.isfinite(g_h).all() and torch.isfinite(g_W).all()
    nobody = (owner < 0).cuda() | (targets < 0)
    assert not g_h[nobody].any()
    # the weight of each token is that of the pair that holds it: its cross entropy's factor
    w = torch.zeros(T, dtype=torch.float64)
    m = 0.1 * (got[1].view(-1, 2)[:, 0] - got[1].view(-1, 2)[:, 1] - reference[0::2] + reference[1::2]).double().cpu()
    for t in range(T):
        p = int(owner[t])
        if p >= 0:
            w[t] = (0.1 if t < o[2 * p + 1] else -0.1) * torch.sigmoid(-m[p]) * weight[p]
    want = mhcl.head_loss_grad(h, W, targets, w.float().cuda())
    # (m here is of fp32 numbers of up to some hundreds, 2^-24 of them each: 1e-5 of a weight)
    for a, b in zip((g_h, g_W), want[2:]):
        assert float((a.double() - b.double()).norm()) <= 1e-4 * float(b.double().norm())
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(got, mhcl.head_preference_grad(*args)))
    again = mhcl.head_preference_grad(*args[:5], torch.ones(pairs, device="cuda"))
    assert bool(torch.isnan(again[3]).all()) == bool(bad) and torch.equal(again[0].isnan().cpu(), isnan)


def test_large_margins():
    h, W, targets, offsets, reference = _inputs(7, 400, 64, 300, 4, F)
    reference += torch.tensor([1e4, 0, 0, 1e4, -3e4, 0, 0, -3e4], device="cuda")
    got = _check(h, W, targets, offsets, reference, beta=0.5)
    assert torch.isfinite(got["loss"]).all() and torch.isfinite(got["g_h"]).all()


@pytest.mark.parametrize("C,holes", [(8, 0.0), (16, 0.0), (16, 0.1), (16, 0.5)])
def test_blocks_of_tokens(C, holes):
    # a vocabulary so long that a block is of 256 tokens, and pairs that lie in two of them, or (tokens left out) all in one
    V = 2 ** 22 - 256
    g = _gen(8)
    h, W = _normal(g, 300, C, dtype=BF), _normal(g, V, C, std=0.5, dtype=BF)
    targets = torch.randint(0, V, (300,), device="cuda", generator=g)
    targets = torch.where(torch.rand(300, device="cuda", generator=g) < holes, -1, targets)
    offsets = torch.tensor([3, 150, 290], device="cuda")
    ce = mhcl.head_loss(h, W, targets)[0].double()
    L = -torch.stack([ce[3:150].sum(), ce[150:290].sum()])
    reference = (L + torch.tensor([20.0, -10.0], device="cuda")).float()
    loss, logp, g_h, g_W = mhcl.head_preference_grad(h, W, targets, offsets, reference, beta=0.05)
    m = 0.05 * ((L[0] - reference[0].double()) - (L[1] - reference[1].double()))
    assert float((logp.double() - L).abs().max()) <= 1e-3 and abs(float(loss) - float(torch.nn.functional.softplus(-m))) <= 1e-4
    w = torch.zeros(300, device="cuda")
    w[3:150], w[150:290] = 0.05 * torch.sigmoid(-m).float(), -0.05 * torch.sigmoid(-m).float()
    want = mhcl.head_loss_grad(h, W, targets, w)
    for a, b in ((g_h, want[2]), (g_W, want[3])):
        assert float((a.double() - b.double()).norm()) <= 1e-3 * float(b.double().norm())


def test_gradients_against_differences():
    h, W, targets, offsets, reference = _inputs(9, 12, 16, 30, 2, F, holes=0.1)
    offsets = torch.tensor([0, 3, 5, 9, 12], device="cuda")
    weight = torch.tensor([0.7, -0.4], device="cuda")

    def value(h, W):
        logp = torch.log_softmax(h @ W.t(), dim=1).gather(1, targets.clamp(min=0).unsqueeze(1)).squeeze(1).masked_fill(targets < 0, 0.0)
        ratio = torch.stack([logp[a:b].sum() for a, b in ((0, 3), (3, 5), (5, 9), (9, 12))]) - reference.double()
        m = 0.3 * (ratio[0::2] - ratio[1::2])
        soft = torch.nn.functional.softplus
        return float(((0.9 * soft(-m) + 0.1 * soft(m)) * weight.double()).sum())

    _, _, g_h, g_W = mhcl.head_preference_grad(h, W, targets, offsets, reference, weight, 0.3, 0.1)
    at = [h.double(), W.double()]
    for k, grad in enumerate((g_h, g_W)):
        for i in (0, grad.numel() // 3, grad.numel() - 1):
            step = torch.zeros_like(at[k])
            step.view(-1)[i] = 1e-5
            up, down = (value(*(t + sign * step if j == k else t for j, t in enumerate(at))) for sign in (1, -1))
            slope = (up - down) / 2e-5
            assert abs(float(grad.reshape(-1)[i]) - slope) <= 1e-4 * max(1.0, abs(slope))


def test_operands_that_do_not_fit_are_refused():
    h, W, targets, offsets, reference = _inputs(10, 9, 64, 40, 2, BF)
    weight = torch.ones(2, device="cuda")
    for args in ((h, W, targets[:-1], offsets), (h, W, targets, offsets[:-1]), (h, W, targets, offsets.float()), (h, W, targets, offsets, reference[:-1]),
                 (h, W, targets, offsets, reference.double()), (h, W, targets, offsets, reference, weight[:-1]), (h, W, targets, offsets.cpu()),
                 (h[:, :-8], W, targets, offsets), (h, W, targets, offsets.view(1, -1))):
        with pytest.raises(ValueError):
            mhcl.head_preference_grad(*args)
    for kw in (dict(beta=math.nan), dict(beta=math.inf), dict(smoothing=-0.1), dict(smoothing=1.1), dict(smoothing=math.nan)):
        with pytest.raises(mhcl.MhclError):
            mhcl.head_preference(h, W, targets, offsets, reference, **kw)
    with pytest.raises(mhcl.MhclError):
        mhcl.head_preference(h, W.float(), targets, offsets)


@pytest.mark.parametrize("io", [BF, F])
def test_python_and_native_calls_agree(monkeypatch, io):
    h, W, targets, offsets, reference = _inputs(11, 45, 64, 136, 3, io)
    weight = torch.rand(3, device="cuda", generator=_gen(1))

    def calls():
        return [*mhcl.head_preference(h, W, targets, offsets, reference, 0.2), *mhcl.head_preference_grad(h, W, targets, offsets, reference, weight),
                *mhcl.head_preference_grad(h, W, targets, offsets, dtype=F)]

    quick = calls()
    monkeypatch.setattr(ends, "_native", lambda: None)
    for a, b in zip(quick, calls()):
        assert a.dtype is b.dtype and a.shape == b.shape and torch.equal(a, b)


@pytest.mark.parametrize("io", [BF, F])
def test_under_autograd(io):
    h, W, targets, offsets, reference = _inputs(12, 70, 64, 100, 3, io)
    head = mhcl.Head(100, 64, dtype=io)
    with torch.no_grad():
        head.W.copy_(W)
    h.requires_grad_()
    weight = torch.rand(3, device="cuda", generator=_gen(2)).requires_grad_()
    loss, logp, g_h, g_W = mhcl.head_preference_grad(h.detach(), W, targets, offsets, reference, weight.detach(), 0.2, 0.1)
    total, held = head.prefer(h, targets, offsets, reference, weight, beta=0.2, smoothing=0.1)
    assert torch.equal(held, logp) and not held.requires_grad
    assert abs(float(total.detach()) - float((loss.double() * weight.detach().double()).sum())) <= 1e-6 * float(loss.abs().sum())
    total.backward()
    assert torch.equal(h.grad, g_h) and torch.equal(head.W.grad, g_W) and torch.equal(weight.grad, loss)
    h.grad = head.W.grad = None
    (0.25 * head.prefer(h, targets, offsets, reference, weight, beta=0.2, smoothing=0.1)[0]).backward()
    assert torch.equal(h.grad, g_h * 0.25) and torch.equal(head.W.grad, g_W * 0.25)
    with torch.no_grad():
        mean, _ = head.prefer(h, targets, offsets, reference)
    plain = mhcl.head_preference(h.detach(), W, targets, offsets, reference)[0].double().mean()
    assert abs(float(mean) - float(plain)) <= 1e-6 * float(plain)
    total, _ = head.prefer(h, targets, offsets, reference)
    total.backward(retain_graph=True)
    with pytest.raises(RuntimeError):
        total.backward()
    g, = torch.autograd.grad(head.prefer(h, targets, offsets, reference)[0], h, create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().square().sum().backward()
    with pytest.raises(ValueError):
        head.prefer(h, targets, offsets, reference.requires_grad_())


@pytest.mark.parametrize("T,C,V", [(40, 64, 700), (1300, 64, 700), (2100, 520, 33000)])
def test_captured_and_replayed(T, C, V):
    h, W, targets, offsets, reference = _inputs(13, T, C, V, 3, BF)
    h2, _, targets2, offsets2, reference2 = _inputs(14, T, C, V, 3, BF)

    def step():
        return mhcl.head_preference_grad(h, W, targets, offsets, reference)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        for a, b in ((h, h2), (targets, targets2)):
            a.copy_(b if i % 2 else b.flip(0))
        if i == 2:
            offsets.copy_(offsets2)
            reference.copy_(reference2)
        if i == 3:
            targets[T // 4:] = -1          # far fewer tokens than when it was captured
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


@pytest.mark.parametrize("io", [BF, F])
def test_many_tokens_in_an_order_of_their_own(io):
    # more tokens than a block of threads places and than one launch counts, in few distinct rows: sums that are known
    T, C, V = 70001, 8, 64000
    g = _gen(20)
    W = _normal(g, V, C, std=0.3, dtype=io)
    h = _normal(g, 7, C, dtype=io).repeat(T // 7 + 1, 1)[:T].contiguous()
    targets = torch.randint(0, V, (T,), device="cuda", generator=g)
    targets = torch.where(torch.rand(T, device="cuda", generator=g) < 0.4, -1, targets)
    offsets = torch.tensor([100, 30000, 33333, 33333, 69000], device="cuda", dtype=torch.int32)
    loss, logp, g_h, g_W = mhcl.head_preference_grad(h, W, targets, offsets)
    ce = mhcl.head_loss(h, W, targets)[0].double()
    want = -torch.stack([ce[a:b].sum() for a, b in ((100, 30000), (30000, 33333), (33333, 33333), (33333, 69000))])
    assert float((logp.double() - want).abs().max()) <= 1e-5 * float(want.abs().max())
    m = 0.1 * (want[0::2] - want[1::2])
    w = torch.zeros(T, device="cuda", dtype=torch.float64)
    for i, (a, b) in enumerate(((100, 30000), (30000, 33333), (33333, 33333), (33333, 69000))):
        w[a:b] = (0.1 if i % 2 == 0 else -0.1) * torch.sigmoid(-m[i // 2]) / 2
    ref_h, ref_W = mhcl.head_loss_grad(h, W, targets, w.float())[2:]
    out = (targets < 0) | (w == 0)
    assert not g_h[out].any()
    for a, b in ((g_h, ref_h), (g_W, ref_W)):
        assert float((a.double() - b.double()).norm()) <= (0.006 if io is BF else 1e-4) * float(b.double().norm())
