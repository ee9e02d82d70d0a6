"""A fine-tuning step of the language model as it is used: the feed-forward blocks with the head's losses against a teacher and of pairs, together;
alone, captured, and beside each other."""
import subprocess
import sys

import pytest
import torch

import paper_2601_05732_amd as mhcl
from paper_2601_05732_amd import lm

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _model(dtype, seed, **kw):
    torch.manual_seed(seed)
    return lm.LanguageModel(90, 64, n=3, layers=2, dtype=dtype, **kw)


@pytest.mark.parametrize("dtype,tied", [(BF, False), (BF, True), (F, False)])
def test_gradients_reach_every_parameter(dtype, tied):
    net, teacher = _model(dtype, 0, tied=tied), _model(dtype, 1)
    tokens = lm.synthetic_tokens(90, 61)
    best, logits = teacher.likeliest(tokens[:-1], 7, rows=16)
    assert best.shape == logits.shape == (60, 7)
    net.distill(tokens[:-1], best, logits, temperature=2.0).backward()
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in net.parameters())
    for p in net.parameters():
        p.grad = None
    offsets = torch.tensor([0, 20, 35, 35, 60], device="cuda")
    with torch.no_grad():
        _, reference = teacher.prefer(tokens[:-1], tokens[1:], offsets)
    loss, logp = net.prefer(tokens[:-1], tokens[1:], offsets, reference)
    loss.backward()
    assert logp.shape == (4,) and float(logp[2]) == 0.0
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in net.parameters())
    # a sequence's log probability is the sum of its tokens' scores
    scores = net.score(tokens[:-1], tokens[1:]).double()
    want = -torch.stack([scores[0:20].sum(), scores[20:35].sum(), scores[:0].sum(), scores[35:60].sum()])
    assert float((logp.double() - want).abs().max()) <= 1e-4 * float(want.abs().max())


def test_the_gradient_of_the_whole_step_against_differences():
    net, teacher = _model(F, 2), _model(F, 3)
    tokens = lm.synthetic_tokens(90, 41)
    best, logits = teacher.likeliest(tokens[:-1], 5)
    offsets = torch.tensor([0, 11, 20, 28, 40], device="cuda")

    def value():
        return net.distill(tokens[:-1], best, logits) + net.prefer(tokens[:-1], tokens[1:], offsets)[0]

    value().backward()
    for p in (net.blocks[0].up.weight, net.blocks[1].down.weight, net.head.W):
        direction = p.grad / p.grad.norm()
        with torch.no_grad():
            values = []
            for sign in (1, -1):
                p += sign * 0.02 * direction
                values.append(float(value().double()))
                p -= sign * 0.02 * direction
        slope = (values[0] - values[1]) / 0.04
        assert abs(slope - float(p.grad.norm())) <= 0.02 * float(p.grad.norm())     # (third derivatives at this step, and fp32 values)


def test_training_runs():
    net, student = _model(BF, 4), _model(BF, 5)
    text = lm.synthetic_tokens(90, 2049)
    assert torch.isfinite(lm.train(net, text, 6, 256)).all()
    assert torch.isfinite(lm.train(student, text, 6, 256, teacher=net, k=4, temperature=2.0)).all()
    assert torch.isfinite(lm.train_on_pairs(net, text, 4, 8, 16)).all()


def test_two_losses_of_one_pass_and_a_captured_step():
    net = _model(BF, 6)
    tokens = lm.synthetic_tokens(90, 301)
    ids, targets = tokens[:-1].clone(), tokens[1:].clone()
    best, logits = _model(BF, 7).likeliest(ids, 6)
    offsets = torch.tensor([0, 70, 150, 220, 290], device="cuda")

    def step():
        for p in net.parameters():
            p.grad = None
        h = net.features(ids)
        total = net.head.distill(h, best, logits) + 0.5 * net.head.prefer(h, targets, offsets)[0] + net.head(h, targets)
        return torch.autograd.grad(total, list(net.parameters()))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        ids.copy_(ids.roll(7))
        targets.copy_(targets.roll(7))
        graph.replay()
        torch.cuda.synchronize()
        got = [g.clone() for g in held]
        eager = step()
        assert all(torch.equal(a, b) for a, b in zip(got, eager))


def test_the_command():
    r = subprocess.run([sys.executable, "-m", "paper_2601_05732_amd.lm", "--V", "50", "--C", "64", "--layers", "1", "--batch", "128", "--steps", "3",
                        "--teach", "4", "--pairs", "2"], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr
    assert "the student's" in r.stdout and "loss of pairs" in r.stdout
