"""A small language model of hyper-connection layers from token ids to the loss: the embedding writes the streams, layers of
:class:`HyperConnection` mix them around ordinary blocks, and the norm of their sum goes into the head.

    x    = embedding(ids)                         [T, n, C]
    x    = H_res x + H_post^T f(H_pre x)          for each block f
    h    = norm(sum of the streams)               [T, C]
    loss = mean cross entropy of h W^T with the next tokens

The blocks here are norm, two linear maps and a gate (what a user replaces by attention and the like); the paper does not say how
streams begin and end, so the ends are this package's choice.

``python -m paper_2601_05732_amd.lm`` trains one on a synthetic language, a fixed random successor for each token with some noise.
"""
from __future__ import annotations

import argparse

import torch

from .autograd import HyperConnection
from .ends import Head, StreamsNorm, TokenEmbedding


class Block(torch.nn.Module):
    """h [T, C] -> [T, C]: RMS norm, a gated pair of linear maps."""

    def __init__(self, C: int, hidden: int, dtype, device):
        super().__init__()
        self.norm = StreamsNorm(C, device=device)
        self.up = torch.nn.Linear(C, 2 * hidden, bias=False, device=device, dtype=dtype)
        self.down = torch.nn.Linear(hidden, C, bias=False, device=device, dtype=dtype)

    def forward(self, h):
        a, b = self.up(self.norm(h)).chunk(2, dim=-1)
        return self.down(torch.nn.functional.silu(a) * b)


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


def train(model, tokens, steps: int, batch: int, lr: float = 3e-3, report=None):
    """AdamW on consecutive pieces of `batch` tokens; the losses."""
    opt = torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.0)
    losses = []
    for step in range(steps):
        at = step * batch % (len(tokens) - batch)
        loss = model(tokens[at:at + batch], tokens[at + 1:at + batch + 1])
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if report and step % report == 0:
            print(f"step {step}: loss {float(losses[-1]):.3f}", flush=True)
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
    args = ap.parse_args()
    net = LanguageModel(args.V, args.C, args.n, args.layers, tied=args.tied)
    text = synthetic_tokens(args.V, 20 * args.batch + 1)
    train(net, text, args.steps, args.batch, report=10)
    held = synthetic_tokens(args.V, args.batch + 1)
    print(f"mean negative log probability: {float(net.score(held[:-1], held[1:]).mean()):.3f}")
