"""The two ends of a language model around a stack of hyper-connection layers: what is measured of them.

A case is one pass through one operator:

  embed   token ids to the n residual streams: x[t, i] = scale * table[ids[t]] for every stream i, and in training the
          table's gradient, the sum over a token's occurrences and over the streams
  norm    the streams' sum s = sum_i x[t, i] and its RMS norm with a gain, out = gain * s / sqrt(mean(s^2) + eps), and in
          training the gradients on the streams and on the gain
  head    logits z = W h over a vocabulary and their softmax cross entropy with the next tokens, loss = lse(z) - z[target],
          and in training the gradients on h and W; negative targets do not count

Where `own` is false, run() is the plain form in 32 bits; where it is true, run() makes the package's calls.
"""
import math

import torch

own = False

EPS = 1e-6
W_STD = 0.02        # of the table and of the head's weights, the repository's choice for projections
LIFT = 6.0          # by how much half of the targets' logits stand out, as after some training
IO = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, T, C, V=0, n=1, io="bf16", w="bf16", grad=True, holes=0.0, weights=False):
    return dict(name=name, op=op, T=T, C=C, V=V, n=n, io=io, w=w, grad=grad, holes=holes, weights=weights)


def listed():
    return [
        # a decode step of a small batch at the widest streams
        _case("embed_serve_t16", "embed", 16, 4096, V=65536, n=4, grad=False),
        # a training micro-batch of 16 sequences of 1024 tokens, fp32 table, bf16 streams
        _case("embed_train_t16384", "embed", 16384, 1024, V=50257, n=4, w="f32"),
        # the largest micro-batch, table and streams in bf16
        _case("embed_train_t32768", "embed", 32768, 4096, V=65536, n=4),
        # fp32 training on ragged sequences, padding among the tokens
        _case("embed_train_f32", "embed", 3001, 768, V=50257, n=4, io="f32", w="f32", holes=0.1),
        # one token per call, as in decoding
        _case("norm_serve_t1", "norm", 1, 4096, n=4, grad=False),
        # the end of the benchmark's stack
        _case("norm_train_t32768", "norm", 32768, 4096, n=4),
        # fp32, three streams, an odd number of tokens
        _case("norm_train_f32", "norm", 4999, 768, n=3, io="f32"),
        # the probability of one next token
        _case("head_score_t1", "head", 1, 4096, V=50257, grad=False),
        # evaluation of a validation batch at the middle width
        _case("head_score_t8192", "head", 8192, 768, V=50257, grad=False),
        # a short fine-tuning step with a small vocabulary, prompts not counted, weights by token
        _case("head_train_t333", "head", 333, 520, V=1003, holes=0.4, weights=True),
        # fp32 training at the paper's middle width, two sequences
        _case("head_train_f32", "head", 2048, 768, V=50257, io="f32", w="f32", holes=0.05),
        # a training micro-batch at the widest streams
        _case("head_train_t16384", "head", 16384, 4096, V=65536, holes=0.05),
    ]


def _logspread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "norm", "head", "head"])
    grad = rng.random() < 0.7
    io = rng.choice(["bf16", "bf16", "f32"])
    C = max(8, _logspread(rng, 64, 4096) // 8 * 8)
    V = _logspread(rng, 500, 65536)
    holes = rng.choice([0.0, 0.05, 0.4])
    if op == "head":
        most = 2.0 ** 42 if io == "bf16" else 2.0 ** 36      # T * C * V
        T = _logspread(rng, 1, max(1, min(16384, int(most / (C * V)))))
        return dict(op=op, T=T, C=C, V=V, n=1, io=io, w=io, grad=grad, holes=holes, weights=rng.random() < 0.5)
    T = _logspread(rng, 1, 32768)
    n = rng.choice([1, 2, 3, 4, 4, 5, 8])
    T = max(1, min(T, 2 ** 29 // (n * C)))
    w = rng.choice(["bf16", "f32"]) if op == "embed" else "f32"
    return dict(op=op, T=T, C=C, V=V if op == "embed" else 0, n=n, io=io, w=w, grad=grad,
                holes=holes if op == "embed" else 0.0, weights=False)


def _scale(case):
    return math.sqrt(case["C"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    T, C, V, n = case["T"], case["C"], case["V"], case["n"]
    io, w = IO[case["io"]], IO[case["w"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=io):
        return torch.empty(shape, device="cuda").normal_(mean, std, generator=gen).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, device="cuda", generator=gen)

    def tokens():
        # frequencies that fall as one over the rank, the ranks spread over the vocabulary
        rank = (uniform(T).double() * math.log(V + 1)).exp().long().clamp(1, V) - 1
        ids = torch.randperm(V, device="cuda", generator=gen)[rank]
        return torch.where(uniform(T) < case["holes"], -1, ids)

    s = dict(case)
    if case["op"] == "embed":
        s.update(table=normal(V, C, std=W_STD, dtype=w), ids=tokens())
        if case["grad"]:
            s["g_x"] = normal(T, n, C)
    elif case["op"] == "norm":
        s.update(x=normal(T, n, C), gain=normal(C, std=0.1, mean=1.0, dtype=torch.float32))
        if case["grad"]:
            s["g_out"] = normal(T, C)
    else:
        W = normal(V, C, std=W_STD, dtype=w)
        ids = tokens()
        lift = LIFT / (C * W_STD ** 2) * (uniform(T, 1) < 0.5)
        s.update(W=W, targets=ids, x=(normal(T, C, dtype=torch.float32) + lift * W[ids.clamp(min=0)].float()).to(io))
        s["weight"] = uniform(T) / T if case["weights"] else None
    return s


def _token_weights(s):
    """d(result) / d(loss of a token): the caller's, or those of the mean over the tokens that count; 0 where none does."""
    counts = s["targets"] >= 0
    mean = 1.0 / counts.sum().clamp(min=1).float()
    return counts, torch.where(counts, mean if s["weight"] is None else s["weight"], 0.0)


def _plain_embed(s):
    io, ids = IO[s["io"]], s["ids"]
    there = (ids >= 0).unsqueeze(1)
    at = ids.clamp(min=0)
    rows = torch.where(there, s["table"][at].float() * _scale(s), 0.0).to(io)
    out = dict(x=rows.unsqueeze(1).expand(-1, s["n"], -1).contiguous())
    if s["grad"]:
        g = torch.where(there, s["g_x"].float().sum(dim=1) * _scale(s), 0.0)
        g_table = torch.zeros(s["V"], s["C"], device=g.device).index_add_(0, at, g)
        out["g_table"] = g_table.to(s["table"].dtype)
    return out


def _plain_norm(s):
    total = s["x"].float().sum(dim=1)
    r = torch.rsqrt(total.square().mean(dim=1, keepdim=True) + EPS)
    unit = total * r
    out = dict(out=(unit * s["gain"]).to(IO[s["io"]]))
    if s["grad"]:
        g_out = s["g_out"].float()
        g = g_out * s["gain"]
        g_total = r * (g - unit * (g * unit).mean(dim=1, keepdim=True))
        out["g_x"] = g_total.to(IO[s["io"]]).unsqueeze(1).expand(-1, s["n"], -1).contiguous()
        out["g_gain"] = (g_out * unit).sum(dim=0)
    return out


def _plain_head(s):
    x, W = s["x"].float(), s["W"].float()
    z = x @ W.t()
    top = z.amax(dim=1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(dim=1, keepdim=True)
    lse = (top + total.log()).squeeze(1)
    counts, weight = _token_weights(s)
    at = s["targets"].clamp(min=0).unsqueeze(1)
    out = dict(loss=torch.where(counts, lse - z.gather(1, at).squeeze(1), 0.0), lse=lse)
    if s["grad"]:
        g = e * (weight.unsqueeze(1) / total)
        g.scatter_add_(1, at, -weight.unsqueeze(1))
        out.update(g_x=(g @ W).to(s["x"].dtype), g_W=(g.t() @ x).to(s["W"].dtype))
    return out


def run(s):
    if not own:
        return {"embed": _plain_embed, "norm": _plain_norm, "head": _plain_head}[s["op"]](s)
    import paper_2601_05732_amd as mhcl
    if s["op"] == "embed":
        out = dict(x=mhcl.embed_tokens(s["table"], s["ids"], s["n"], scale=_scale(s), dtype=IO[s["io"]]))
        if s["grad"]:
            out["g_table"] = mhcl.embed_tokens_grad(s["ids"], s["g_x"], s["V"], scale=_scale(s), dtype=IO[s["w"]])
        return out
    if s["op"] == "norm":
        out = dict(out=mhcl.streams_norm(s["x"], s["gain"], eps=EPS))
        if s["grad"]:
            out["g_x"], out["g_gain"] = mhcl.streams_norm_grad(s["x"], s["gain"], s["g_out"], eps=EPS)
        return out
    if not s["grad"]:
        return dict(zip(("loss", "lse"), mhcl.head_loss(s["x"], s["W"], s["targets"])))
    return dict(zip(("loss", "lse", "g_x", "g_W"), mhcl.head_loss_grad(s["x"], s["W"], s["targets"], weight=s["weight"])))


def work(case):
    T, C, V, n = case["T"], case["C"], case["V"], case["n"]
    e, w = (2 if case[k] == "bf16" else 4 for k in ("io", "w"))
    if case["op"] == "embed":
        rows = min(T, V)                                      # of the table: no more than there are tokens
        size, flops = T * (n * C * e + 8) + rows * C * w, T * C
        if case["grad"]:
            size, flops = size + T * (n * C * e + 8) + V * C * w, flops + T * (n + 1) * C
    elif case["op"] == "norm":
        size, flops = T * (n + 1) * C * e + 4 * C, T * (n + 4) * C
        if case["grad"]:
            size, flops = size + T * (2 * n + 1) * C * e + 8 * C, flops + T * (n + 10) * C
    else:
        size, flops = T * (C * e + 16) + V * C * w, 2 * T * C * V
        if case["grad"]:
            size, flops = size + T * C * e + V * C * w + 4 * T * bool(case["weights"]), 3 * flops
    return dict(bytes=size, flops=flops)


# ---- the definitions in 64 bits -------------------------------------------------------------


def _exact_embed(s, n):
    V, C = s["table"].shape
    ids, scale = s["ids"], _scale(s)
    held = ids >= 0
    x = torch.zeros(len(ids), n, C, dtype=torch.float64, device=ids.device)
    x[held] = scale * s["table"].double()[ids[held]].unsqueeze(1)
    out = dict(x=x)
    if s["grad"]:
        g_table = torch.zeros(V, C, dtype=torch.float64, device=ids.device)
        g_table.index_put_((ids[held],), scale * s["g_x"].double()[held].sum(dim=1), accumulate=True)
        out["g_table"] = g_table
    return out


def _exact_norm(s):
    x = s["x"].double().requires_grad_(s["grad"])
    gain = s["gain"].double().requires_grad_(s["grad"])
    total = x.sum(dim=1)
    y = gain * total / (total.pow(2).mean(dim=1, keepdim=True) + EPS).sqrt()
    if not s["grad"]:
        return dict(out=y)
    g_x, g_gain = torch.autograd.grad(y, [x, gain], s["g_out"].double())
    return dict(out=y.detach(), g_x=g_x, g_gain=g_gain)


def _exact_head(s):
    W, targets = s["W"].double(), s["targets"]
    T, V = len(targets), len(W)
    counted = int((targets >= 0).sum())
    parts, g_W = dict(loss=[], lse=[], g_x=[]), torch.zeros_like(W)
    rows = max(1, 2 ** 27 // V)
    for t0 in range(0, T, rows):
        x, y = s["x"][t0:t0 + rows].double(), targets[t0:t0 + rows]
        z = x @ W.t()
        lse = torch.logsumexp(z, dim=1)
        hit = y.unsqueeze(1) == torch.arange(V, device=y.device)
        parts["lse"].append(lse)
        parts["loss"].append(((lse.unsqueeze(1) - z) * hit).sum(dim=1))
        if s["grad"]:
            w = (y >= 0).double()
            w = w / max(1, counted) if s["weight"] is None else w * s["weight"][t0:t0 + rows].double()
            g = (torch.exp(z - lse.unsqueeze(1)) - hit.double()) * w.unsqueeze(1)
            parts["g_x"].append(g @ W)
            g_W += g.t().contiguous() @ x
    out = {k: torch.cat(v) for k, v in parts.items() if v}
    if s["grad"]:
        out["g_W"] = g_W
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        return _exact_embed(s, case["n"])
    return _exact_norm(s) if case["op"] == "norm" else _exact_head(s)
