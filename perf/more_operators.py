"""A fine-tuning step around the hyper-connection layers: what is measured of the block between the layers and of the head's
losses beyond the next token.

A case is one pass through one operator:

  ffn      the gated feed-forward block y = (silu(x Wg^T) * (x Wu^T)) Wd^T, Wg and Wu being the halves of W_up [2 H, C], and in
           training the gradients on x and on both weights
  distill  the head's logits z = h W^T against a teacher's top logits: with p the softmax of a token's teacher logits / temperature over
           the slots that hold one (ids of -1 hold none) and q that of z / temperature over the vocabulary, loss = sum_k p_k
           (log p_k - log q[ids_k]), and in training the gradients on h and W
  prefer   pairs of packed sequences, the chosen one and the rejected one: L the sum of the log probabilities of a sequence's targets,
           m = beta ((L_c - R_c) - (L_r - R_r)) with R those of a reference model, loss = (1 - s) softplus(-m) + s softplus(m), and in
           training the gradients on h and W

Where `own` is false, run() is the plain form in 32 bits (log probabilities of sequences are added up in 64); where it is true, run()
makes the package's calls.
"""
import math

import torch

own = False

W_STD = 0.02        # of the weights, the repository's choice for projections
LIFT = 6.0          # by how much the logit of half of the likeliest next tokens stands out, as after some training
BETA = 0.1
IO = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ffn(name, T, C, H, io="bf16", grad=True):
    return dict(name=name, op="ffn", T=T, C=C, H=H, io=io, grad=grad)


def _distill(name, T, C, V, K, io="bf16", grad=True, temperature=1.0, holes=0.0, short=0.0, weights=False):
    return dict(name=name, op="distill", T=T, C=C, V=V, K=K, io=io, grad=grad, temperature=temperature, holes=holes, short=short,
                weights=weights)


def _prefer(name, T, C, V, pairs, io="bf16", grad=True, smoothing=0.0, weights=False):
    return dict(name=name, op="prefer", T=T, C=C, V=V, pairs=pairs, io=io, grad=grad, smoothing=smoothing, weights=weights)


def listed():
    return [
        # one token per call at the widest layers, as in decoding
        _ffn("ffn_serve_t1", 1, 4096, 8192, grad=False),
        # a decode step of a middle batch
        _ffn("ffn_serve_t48", 48, 1024, 4096, grad=False),
        # a short fine-tuning step of a small model, odd sizes
        _ffn("ffn_train_t333", 333, 520, 1000),
        # fp32 training at the paper's middle width, two sequences
        _ffn("ffn_train_f32", 2048, 768, 2048, io="f32"),
        # a training micro-batch at the widest layers
        _ffn("ffn_train_t16384", 16384, 4096, 8192),
        # a short fine-tuning step from a teacher's few logits, prompts without any
        _distill("distill_train_t333", 333, 520, 1003, 8, holes=0.4, weights=True),
        # how far a validation batch is from its teacher
        _distill("distill_eval_t8192", 8192, 768, 50257, 32, grad=False),
        # fp32 training from softened logits, lists of unequal length
        _distill("distill_train_f32", 2048, 768, 50257, 20, io="f32", temperature=2.0, holes=0.05, short=0.3),
        # a training micro-batch at the widest streams, the teacher's 64 best of every token
        _distill("distill_train_t16384", 16384, 4096, 65536, 64, holes=0.05),
        # two pairs of short answers to a small model
        _prefer("prefer_train_p2", 300, 264, 1003, 2),
        # the margins of a validation set of pairs
        _prefer("prefer_eval_p12", 8192, 768, 50257, 12, grad=False),
        # a micro-batch of pairs at the widest streams, labels that may be wrong
        _prefer("prefer_train_p16", 8192, 4096, 65536, 16, smoothing=0.1, weights=True),
    ]


def _logspread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _eights(rng, lo, hi):
    return max(8, _logspread(rng, lo, hi) // 8 * 8)


def draw(rng):
    op = rng.choice(["ffn", "distill", "prefer"])
    io = rng.choice(["bf16", "bf16", "f32"])
    grad = rng.random() < 0.7
    C = _eights(rng, 64, 4096)
    if op == "ffn":
        H = _eights(rng, 64, 8192)
        most = 2.0 ** 39 if io == "bf16" else 2.0 ** 34      # T * C * H
        T = _logspread(rng, 1, max(1, min(16384, int(most / (C * H)))))
        return dict(op=op, T=T, C=C, H=H, io=io, grad=grad)
    V = _logspread(rng, 500, 65536)
    most = 2.0 ** 42 if io == "bf16" else 2.0 ** 36          # T * C * V
    T = _logspread(rng, 4, max(4, min(16384, int(most / (C * V)))))
    weights = rng.random() < 0.5
    if op == "distill":
        return dict(op=op, T=T, C=C, V=V, K=_logspread(rng, 1, 128), io=io, grad=grad, temperature=rng.choice([1.0, 1.0, 0.7, 2.0, 4.0]),
                    holes=rng.choice([0.0, 0.05, 0.4]), short=rng.choice([0.0, 0.3]), weights=weights)
    return dict(op=op, T=T, C=C, V=V, pairs=_logspread(rng, 1, max(1, min(64, T // 4))), io=io, grad=grad,
                smoothing=rng.choice([0.0, 0.1]), weights=weights)


# ---- inputs ---------------------------------------------------------------------------------


def _tokens(s, uniform, gen):
    # frequencies that fall as one over the rank, the ranks spread over the vocabulary
    T, V = s["T"], s["V"]
    rank = (uniform(T).double() * math.log(V + 1)).exp().long().clamp(1, V) - 1
    return rank, torch.randperm(V, device="cuda", generator=gen)


def _lifted(s, W, ids, normal, uniform):
    # h of which half of the tokens' logits stand out at ids
    T, C = s["T"], s["C"]
    lift = LIFT / (C * W_STD ** 2) * (uniform(T, 1) < 0.5)
    return (normal(T, C, dtype=torch.float32) + lift * W[ids].float()).to(IO[s["io"]])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    T, C, io = case["T"], case["C"], IO[case["io"]]

    def normal(*shape, std=1.0, dtype=io):
        return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, device="cuda", generator=gen)

    s = dict(case)
    if case["op"] == "ffn":
        # x as a norm leaves it
        s.update(x=normal(T, C), W_up=normal(2 * case["H"], C, std=W_STD), W_down=normal(C, case["H"], std=W_STD))
        if case["grad"]:
            s["g_y"] = normal(T, C)
        return s
    V = case["V"]
    W = normal(V, C, std=W_STD)
    rank, spread = _tokens(case, uniform, gen)
    if case["op"] == "distill":
        # a token's K likeliest next tokens have neighbouring ranks and logits that fall with their place
        K = case["K"]
        place = torch.arange(K, device="cuda")
        ids = spread[(rank.unsqueeze(1) + place) % V]
        logits = 8.0 - 1.5 * (1.0 + place).log() + normal(T, K, std=0.5, dtype=torch.float32)
        logits = logits.sort(dim=1, descending=True)[0]
        h = _lifted(case, W, ids[:, 0], normal, uniform)
        # lists that end early, and tokens that the teacher says nothing of
        count = torch.where(uniform(T) < case["short"], (uniform(T) * K).long() + 1, K)
        count = torch.where(uniform(T) < case["holes"], 0, count)
        ids = torch.where(place < count.unsqueeze(1), ids, -1)
        s.update(h=h, W=W, ids=ids, logits=logits, weight=uniform(T) / T if case["weights"] else None)
        return s
    # packed sequences, each a prompt that does not count and an answer; some rows of padding behind the last
    pairs = case["pairs"]
    share = 0.25 + uniform(2 * pairs)
    ends = (share.cumsum(0) / share.sum() * (0.97 * T)).long()
    offsets = torch.cat([torch.zeros(1, device="cuda", dtype=torch.long), ends])
    at = torch.arange(T, device="cuda")
    seq = torch.searchsorted(ends, at, right=True).clamp(max=2 * pairs - 1)
    into = (at - offsets[seq]).float() / (offsets[seq + 1] - offsets[seq]).clamp(min=1)
    ids = spread[rank]
    h = _lifted(case, W, ids, normal, uniform)
    targets = torch.where((into < 0.3) | (at >= offsets[-1]), -1, ids)
    # the reference is the same model some steps ago: its log probabilities differ by a little from this one's
    L = torch.zeros(2 * pairs, device="cuda", dtype=torch.float64)
    rows = max(1, 2 ** 28 // V)
    for t0 in range(0, T, rows):
        z = (h[t0:t0 + rows] @ W.t()).float()
        y = targets[t0:t0 + rows]
        logp = z.gather(1, y.clamp(min=0).unsqueeze(1)).squeeze(1) - z.logsumexp(dim=1)
        L.index_add_(0, seq[t0:t0 + rows], torch.where(y >= 0, logp, 0.0).double())
    reference = (L + 8.0 * normal(2 * pairs, dtype=torch.float64)).float()
    s.update(h=h, W=W, targets=targets, offsets=offsets, reference=reference,
             weight=uniform(pairs) / pairs if case["weights"] else None)
    return s


# ---- the plain forms ------------------------------------------------------------------------


def _plain_ffn(s):
    x, W_up, W_down = s["x"].float(), s["W_up"].float(), s["W_down"].float()
    gate, up = (x @ W_up.t()).chunk(2, dim=1)
    sig = 1.0 / (1.0 + (-gate).exp())
    act = gate * sig * up
    out = dict(y=(act @ W_down.t()).to(s["x"].dtype))
    if s["grad"]:
        g_y = s["g_y"].float()
        g_act = g_y @ W_down
        g_pre = torch.cat([g_act * up * sig * (1.0 + gate * (1.0 - sig)), g_act * gate * sig], dim=1)
        out.update(g_x=(g_pre @ W_up).to(s["x"].dtype), g_W_up=(g_pre.t() @ x).to(s["x"].dtype),
                   g_W_down=(g_y.t() @ act).to(s["x"].dtype))
    return out


def _softmax_parts(z):
    top = z.amax(dim=1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(dim=1, keepdim=True)
    return e, total, (top + total.log()).squeeze(1)


def _plain_distill(s):
    h, W, inv = s["h"].float(), s["W"].float(), 1.0 / s["temperature"]
    z = (h @ W.t()) * inv
    e, total, lse = _softmax_parts(z)
    there = s["ids"] >= 0
    counts = there.any(dim=1)
    at = s["ids"].clamp(min=0)
    a = torch.where(there, s["logits"] * inv, -math.inf)
    a = a - torch.where(counts, a.amax(dim=1), 0.0).unsqueeze(1)
    ea = a.exp()
    sum_a = torch.where(counts, ea.sum(dim=1), 1.0).unsqueeze(1)
    p = ea / sum_a
    terms = (a - sum_a.log()) - (z.gather(1, at) - lse.unsqueeze(1))
    out = dict(loss=torch.where(there, p * terms, 0.0).sum(dim=1), lse=lse)
    if s["grad"]:
        w = 1.0 / counts.sum().clamp(min=1).float() if s["weight"] is None else s["weight"]
        w = torch.where(counts, w * inv, 0.0).unsqueeze(1)
        g = e * (w / total)
        g.scatter_add_(1, at, -w * p)
        out.update(g_h=(g @ W).to(s["h"].dtype), g_W=(g.t() @ h).to(s["W"].dtype))
    return out


def _plain_prefer(s):
    h, W, targets, offsets = s["h"].float(), s["W"].float(), s["targets"], s["offsets"]
    z = h @ W.t()
    e, total, lse = _softmax_parts(z)
    T, n = len(targets), len(offsets) - 1
    row = torch.arange(T, device=targets.device)
    seq = (row.unsqueeze(1) >= offsets[1:]).sum(dim=1)
    counts = (targets >= 0) & (row >= offsets[0]) & (seq < n)
    seq = seq.clamp(max=n - 1)
    at = targets.clamp(min=0).unsqueeze(1)
    logp = torch.where(counts, z.gather(1, at).squeeze(1) - lse, 0.0)
    L = torch.zeros(n, device=h.device, dtype=torch.float64).index_add_(0, seq, logp.double())
    ratio = (L - s["reference"].double()).view(-1, 2)
    m = BETA * (ratio[:, 0] - ratio[:, 1])
    smooth = s["smoothing"]

    def softplus(v):
        return v.clamp(min=0.0) + (1.0 + (-v.abs()).exp()).log()

    out = dict(loss=((1.0 - smooth) * softplus(-m) + smooth * softplus(m)).float(), logp=L.float())
    if s["grad"]:
        slope = smooth / (1.0 + (-m).exp()) - (1.0 - smooth) / (1.0 + m.exp())
        slope = slope * (1.0 / len(m) if s["weight"] is None else s["weight"])
        w = torch.stack([-BETA * slope, BETA * slope], dim=1).view(-1).float()
        w = torch.where(counts, w[seq], 0.0).unsqueeze(1)
        g = e * (w / total)
        g.scatter_add_(1, at, -w)
        out.update(g_h=(g @ W).to(s["h"].dtype), g_W=(g.t() @ h).to(s["W"].dtype))
    return out


def run(s):
    if not own:
        return {"ffn": _plain_ffn, "distill": _plain_distill, "prefer": _plain_prefer}[s["op"]](s)
    import paper_2601_05732_amd as mhcl
    if s["op"] == "ffn":
        if not s["grad"]:
            return dict(y=mhcl.gated_ffn(s["x"], s["W_up"], s["W_down"]))
        y, kept = mhcl.gated_ffn(s["x"], s["W_up"], s["W_down"], keep=True)
        return dict(zip(("y", "g_x", "g_W_up", "g_W_down"),
                        (y, *mhcl.gated_ffn_grad(s["x"], s["W_up"], s["W_down"], kept, s["g_y"]))))
    if s["op"] == "distill":
        if not s["grad"]:
            return dict(zip(("loss", "lse"), mhcl.head_distill(s["h"], s["W"], s["ids"], s["logits"], temperature=s["temperature"])))
        return dict(zip(("loss", "lse", "g_h", "g_W"),
                        mhcl.head_distill_grad(s["h"], s["W"], s["ids"], s["logits"], weight=s["weight"], temperature=s["temperature"])))
    args = (s["h"], s["W"], s["targets"], s["offsets"], s["reference"])
    if not s["grad"]:
        return dict(zip(("loss", "logp"), mhcl.head_preference(*args, beta=BETA, smoothing=s["smoothing"])))
    return dict(zip(("loss", "logp", "g_h", "g_W"),
                    mhcl.head_preference_grad(*args, weight=s["weight"], beta=BETA, smoothing=s["smoothing"])))


def work(case):
    T, C, e = case["T"], case["C"], 2 if case["io"] == "bf16" else 4
    grad = bool(case["grad"])
    if case["op"] == "ffn":
        H = case["H"]
        size, flops = (2 * T * C + 3 * H * C) * e, 6 * T * C * H
        if grad:
            size, flops = size + (2 * T * C + 3 * H * C) * e, 3 * flops
        return dict(bytes=size, flops=flops)
    V = case["V"]
    size, flops = (T + V) * C * e, 2 * T * C * V
    if case["op"] == "distill":
        size += T * (case["K"] * 12 + 8 + 4 * bool(case["weights"] and grad))
    else:
        size += T * 8 + case["pairs"] * (2 * (8 + 4 + 4) + 4 + 4 * bool(case["weights"] and grad))
    if grad:
        size, flops = size + (T + V) * C * e, 3 * flops
    return dict(bytes=size, flops=flops)


# ---- the definitions in 64 bits -------------------------------------------------------------


def _exact_ffn(s):
    x, W_up, W_down = (s[k].double().requires_grad_(s["grad"]) for k in ("x", "W_up", "W_down"))
    H = W_down.shape[1]
    gate = x @ W_up[:H].t()
    y = (gate * torch.sigmoid(gate) * (x @ W_up[H:].t())) @ W_down.t()
    if not s["grad"]:
        return dict(y=y)
    g_x, g_up, g_down = torch.autograd.grad(y, [x, W_up, W_down], s["g_y"].double())
    return dict(y=y.detach(), g_x=g_x, g_W_up=g_up, g_W_down=g_down)


def _blocks(s):
    rows = max(1, 2 ** 27 // len(s["W"]))
    return [slice(t0, t0 + rows) for t0 in range(0, s["T"], rows)]


def _exact_distill(s):
    W, tau, V = s["W"].double(), s["temperature"], len(s["W"])
    held = s["ids"] >= 0
    counted = held.any(dim=1)
    out, g_W = dict(loss=[], lse=[], g_h=[]), torch.zeros_like(W)
    for b in _blocks(s):
        h, ids, on = s["h"][b].double(), s["ids"][b], held[b]
        z = (h @ W.t()) / tau
        logq = torch.log_softmax(z, dim=1)
        out["lse"].append(torch.logsumexp(z, dim=1))
        p = torch.softmax((s["logits"][b].double() / tau).masked_fill(~on, -1e300), dim=1).masked_fill(~on, 0.0)
        teacher = torch.zeros(len(h), V, dtype=torch.float64, device=h.device).scatter_add_(1, ids.clamp(min=0), p)
        out["loss"].append(torch.special.xlogy(p, p).sum(dim=1) - (teacher * logq).sum(dim=1))
        if s["grad"]:
            w = counted[b].double()
            w = w / max(1, int(counted.sum())) if s["weight"] is None else w * s["weight"][b].double()
            g = (logq.exp() - teacher) * (w / tau).unsqueeze(1)
            out["g_h"].append(g @ W)
            g_W += g.t().contiguous() @ h
    out = {k: torch.cat(v) for k, v in out.items() if v}
    if s["grad"]:
        out["g_W"] = g_W
    return out


def _exact_prefer(s):
    W, targets = s["W"].double(), s["targets"]
    T, bounds = s["T"], s["offsets"].tolist()
    n = len(bounds) - 1
    logp = torch.zeros(T, dtype=torch.float64, device=W.device)
    for b in _blocks(s):
        logq = torch.log_softmax(s["h"][b].double() @ W.t(), dim=1)
        y = targets[b]
        logp[b] = logq.gather(1, y.clamp(min=0).unsqueeze(1)).squeeze(1).masked_fill(y < 0, 0.0)
    L = torch.stack([logp[bounds[i]:bounds[i + 1]].sum() for i in range(n)]).requires_grad_()
    ratio = L - s["reference"].double()
    m = BETA * (ratio[0::2] - ratio[1::2])
    loss = -(1.0 - s["smoothing"]) * torch.nn.functional.logsigmoid(m) - s["smoothing"] * torch.nn.functional.logsigmoid(-m)
    out = dict(loss=loss.detach(), logp=L.detach())
    if not s["grad"]:
        return out
    total = loss.mean() if s["weight"] is None else (loss * s["weight"].double()).sum()
    slope, = torch.autograd.grad(total, L)
    w = torch.zeros(T, dtype=torch.float64, device=W.device)
    for i in range(n):
        w[bounds[i]:bounds[i + 1]] = -slope[i]
    w = w.masked_fill(targets < 0, 0.0)
    g_h, g_W = [], torch.zeros_like(W)
    for b in _blocks(s):
        h, y = s["h"][b].double(), targets[b]
        g = torch.softmax(h @ W.t(), dim=1)
        g.scatter_add_(1, y.clamp(min=0).unsqueeze(1), -torch.ones(len(y), 1, dtype=torch.float64, device=W.device))
        g *= w[b].unsqueeze(1)
        g_h.append(g @ W)
        g_W += g.t().contiguous() @ h
    return dict(out, g_h=torch.cat(g_h), g_W=g_W)


def exact(case, seed):
    s = prepare(case, seed)
    return {"ffn": _exact_ffn, "distill": _exact_distill, "prefer": _exact_prefer}[case["op"]](s)
