"""A small language model of hyper-connection layers from token ids to the loss: the embedding writes the streams, layers of
:class:`HyperConnection` mix them around ordinary blocks, and the norm of their sum goes into the head.

    x    = embedding(ids)                         [T, n, C]
    x    = H_res x + H_post^T f(H_pre x)          for each block f
    h    = norm(sum of the streams)               [T, C]
    loss = mean cross entropy of h W^T with the next tokens

The blocks here are norm and a gated feed-forward block (what a user replaces by attention and the like); the paper does not say how
streams begin and end, so the ends are this package's choice.

Besides the next tokens the head learns from a teacher's likeliest ones and from pairs of sequences (:meth:`LanguageModel.distill`,
:meth:`LanguageModel.prefer`).

``python -m paper_2601_05732_amd.lm`` trains one on a synthetic language, a fixed random successor for each token with some noise (``--teach K``
and ``--pairs P``: and then in those ways).
"""
from __future__ import annotations

import argparse

import torch
from torch.nn.modules.module import _has_any_global_hook

from .autograd import HyperConnection
from .ends import Head, StreamsNorm, TokenEmbedding
from .ffn import apply_gated_ffn, takes


class Block(torch.nn.Module):
    """h [T, C] -> [T, C]: RMS norm, a gated pair of linear maps."""

    def __init__(self, C: int, hidden: int, dtype, device):
        super().__init__()
        self.norm = StreamsNorm(C, device=device)
        self.up = torch.nn.Linear(C, 2 * hidden, bias=False, device=device, dtype=dtype)
        self.down = torch.nn.Linear(hidden, C, bias=False, device=device, dtype=dtype)

    def forward(self, h):
        h = self.norm(h)
        if _plain_linear(self.up, h) and _plain_linear(self.down, h):
            W_up, W_down = self.up.weight, self.down.weight
            C, H = W_down.shape
            if W_up.shape == (2 * H, C) and takes(C, H, h.dtype):
                return apply_gated_ffn(h, W_up, W_down)
        a, b = self.up(h).chunk(2, dim=-1)      # widths that the kernels do not take, or maps that a user put in place of these
        return self.down(torch.nn.functional.silu(a) * b)


_LINEAR = torch.nn.Linear.forward


def _plain_linear(m, h) -> bool:
    """Whether `m` is a linear map as Block makes it, and nothing takes the place of its call or looks at it: a `forward` of its own (offloading,
    adapters), a weight of a tensor subclass, hooks of it or of all modules, a compiled call."""
    return (type(m) is torch.nn.Linear and "forward" not in vars(m) and torch.nn.Linear.forward is _LINEAR and m._compiled_call_impl is None
            and not (m._forward_hooks or m._forward_pre_hooks or m._backward_hooks or m._backward_pre_hooks or _has_any_global_hook())
            and m.bias is None and type(m.weight) in (torch.nn.Parameter, torch.Tensor) and m.weight.dtype is h.dtype
            and not torch.is_autocast_enabled("cuda"))


class LanguageModel(torch.nn.Module):
    def __init__(self, V: int, C: int, n: int = 4, layers: int = 2, hidden=None, res_mode: str = "lite", dtype=torch.bfloat16,
                 tied: bool = False, device="cuda"):
        """tied: the head's weights are the embedding's table (which is then of `dtype`); else the table is fp32."""
        super().__init__()
        self.embedding = TokenEmbedding(V, C, n, scale=C ** 0.5, dtype=dtype, table_dtype=dtype if tied else torch.float32,
                                        device=device)
        self.blocks = torch.nn.ModuleList([Block(C, hidden or 2 * C, dtype, device) for _ in range(layers)])
        self.layers = torch.nn.ModuleList([HyperConnection(n, C, res_mode, one_index=l % n, device=device, layer_index=l)
                                           for l in range(layers)])
        self.norm = StreamsNorm(C, device=device)
        self.head = Head(V, C, dtype=dtype, device=device, table=self.embedding.table if tied else None)

    def features(self, ids):
        """h [T, C] of token ids [T], what the head reads."""
        x = self.embedding(ids)
        for layer, block in zip(self.layers, self.blocks):
            x = layer(x, block)
        return self.norm(x)

    def forward(self, ids, targets, weight=None):
        """The loss; negative ids hold no token, negative targets do not count."""
        return self.head(self.features(ids), targets, weight)

    def distill(self, ids, teacher_ids, teacher_logits, weight=None, temperature: float = 1.0):
        """The loss against a teacher's likeliest next tokens [T, K] of each token and their logits (`likeliest` of another model)."""
        return self.head.distill(self.features(ids), teacher_ids, teacher_logits, weight, temperature)

    def prefer(self, ids, targets, offsets, reference=None, weight=None, beta: float = 0.1, smoothing: float = 0.0):
        """The loss of pairs of packed sequences, the chosen and the rejected one, and the sequences' log probabilities [2 P], which are
        the `reference` of a later model.  offsets [2 P + 1]: where sequences begin; negative targets do not count.  (These blocks see one
        token at a time: a model with attention keeps sequences apart itself.)"""
        return self.head.prefer(self.features(ids), targets, offsets, reference, weight, beta, smoothing)

    @torch.no_grad()
    def likeliest(self, ids, k: int, rows: int = 4096):
        """``ids [T, k], logits [T, k]`` of the k likeliest next tokens of each token, by torch's product and selection."""
        out = [(h @ self.head.W.t()).float().topk(k, dim=1) for h in self.features(ids).split(rows)]
        return torch.cat([o.indices for o in out]), torch.cat([o.values for o in out])

    @torch.no_grad()
    def score(self, ids, targets):
        """The negative log probability [T] of each target."""
        return self.head.score(self.features(ids), targets)[0]


def synthetic_tokens(V: int, count: int, noise: float = 0.1, seed: int = 0, device="cuda"):
    """`count` tokens, each the successor of the one before under a fixed random map, or with probability `noise` any token."""
    g = torch.Generator().manual_seed(seed)
    after = torch.randperm(V, generator=g).tolist()
    jumps = (torch.rand(count, generator=g) < noise).tolist()
    anywhere = torch.randint(0, V, (count,), generator=g).tolist()
    tokens = [0]
    for t in range(1, count):
        tokens.append(anywhere[t] if jumps[t] else after[tokens[-1]])
    return torch.tensor(tokens, device=device)


def train(model, tokens, steps: int, batch: int, lr: float = 3e-3, report=None, teacher=None, k: int = 8, temperature: float = 1.0):
    """AdamW on consecutive pieces of `batch` tokens; the losses.  teacher: a model whose k likeliest next tokens are learned instead of the
    text's."""
    opt = torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.0)
    losses = []
    for step in range(steps):
        at = step * batch % (len(tokens) - batch)
        if teacher is None:
            loss = model(tokens[at:at + batch], tokens[at + 1:at + batch + 1])
        else:
            loss = model.distill(tokens[at:at + batch], *teacher.likeliest(tokens[at:at + batch], k), temperature=temperature)
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if report and step % report == 0:
            print(f"step {step}: loss {float(losses[-1]):.3f}", flush=True)
    return torch.stack(losses)


def train_on_pairs(model, tokens, steps: int, pairs: int, length: int, lr: float = 1e-3, beta: float = 0.1, report=None):
    """AdamW on pairs of sequences of `length` tokens, the chosen ones out of the text and the rejected ones those in another order, measured against
    the model as it is at the start; the losses."""
    opt = torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.0)
    g = torch.Generator().manual_seed(0)
    span, losses = pairs * (length + 1), []
    if pairs < 1 or length < 1 or len(tokens) <= span:
        raise ValueError(f"{pairs} pairs of {length} tokens need more than {span} tokens, got {len(tokens)}")
    offsets = torch.arange(2 * pairs + 1, device=tokens.device) * length
    packed = []
    for step in range(steps):
        at = step * span % (len(tokens) - span)
        chosen = tokens[at:at + span].view(pairs, length + 1)
        both = torch.stack([chosen, chosen[:, torch.randperm(length + 1, generator=g).to(tokens.device)]], dim=1).view(2 * pairs, length + 1)
        packed.append((both[:, :-1].reshape(-1), both[:, 1:].reshape(-1)))
    with torch.no_grad():
        references = [model.prefer(ids, targets, offsets)[1] for ids, targets in packed]
    for step, ((ids, targets), reference) in enumerate(zip(packed, references)):
        loss, _ = model.prefer(ids, targets, offsets, reference, beta=beta)
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if report and step % report == 0:
            print(f"step {step}: loss of pairs {float(losses[-1]):.3f}", flush=True)
    return torch.stack(losses)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--V", type=int, default=1000)
    ap.add_argument("--C", type=int, default=256)
    ap.add_argument("--n", type=int, default=4)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--batch", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--tied", action="store_true")
    ap.add_argument("--teach", type=int, default=0, metavar="K", help="then train a second model on the first one's K likeliest next tokens")
    ap.add_argument("--pairs", type=int, default=0, metavar="P", help="then train on so many pairs of sequences a step")
    args = ap.parse_args()
    net = LanguageModel(args.V, args.C, args.n, args.layers, tied=args.tied)
    text = synthetic_tokens(args.V, 20 * args.batch + 1)
    train(net, text, args.steps, args.batch, report=10)
    held = synthetic_tokens(args.V, args.batch + 1)
    print(f"mean negative log probability: {float(net.score(held[:-1], held[1:]).mean()):.3f}")
    if args.teach:
        student = LanguageModel(args.V, args.C, args.n, args.layers, tied=args.tied)
        train(student, text, args.steps, args.batch, report=10, teacher=net, k=args.teach)
        print(f"the student's: {float(student.score(held[:-1], held[1:]).mean()):.3f}")
    if args.pairs:
        train_on_pairs(net, text, args.steps, args.pairs, 64, report=10)
