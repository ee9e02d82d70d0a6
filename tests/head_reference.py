"""The head's losses in 64 bits with, for each result, the largest error that its roundings allow: helpers of the GPU tests.

Roundings that count, for operands in bf16 or fp32:
  * a sum of products over K: 2^-24 of the sum of their sizes for each of the ceil(K / 32) additions to the fp32 accumulator, six times
    as many for fp32 operands, and 2^-23 for the products of their parts that are left out; for a logit at most e_z in a row, and with a
    factor on the logits 2^-23 of the largest besides (the factor's rounding and the product's);
  * lse: e_z and 2^-22 of itself; a token's log probability: 2 e_z and 2^-22 of its parts;
  * a probability, relative: 2 e_z, and 2^-21 for each unit of |z - lse| and |lse| that goes through an exponential in fp32;
  * g, the gradient on a logit: the probability's error, for bf16 also 2^-11 of it (numerators of 10 bits; none below 2^-63), and its
    rounding, finfo.eps / 2 (fp32: twice that, for the weight's product);
  * g_h, g_W: those errors times |W|, |h|, that of the sum of |g| |W|, |g| |h|, and the rounding of the result.
"""
import torch

BF, F = torch.bfloat16, torch.float32


def summed(K, io):
    return (-(-K // 32) + 1) * 2.0 ** -24 if io is BF else (6 * -(-K // 32) + 3) * 2.0 ** -24


def last(io):
    return 2.0 ** -8 if io is BF else 2.0 ** -23


class Logits:
    """z = h W^T * inv of a block of rows, their lse and probabilities q, and the errors of each."""

    def __init__(self, h, W, inv=1.0):
        self.x, self.W = h.double(), W.double()
        io, bf = h.dtype, h.dtype is BF
        self.z = (self.x @ self.W.t()) * inv
        self.e_z = summed(h.shape[1], io) * inv * (self.x.abs() @ self.W.abs().t()).amax(dim=1)
        if inv != 1.0:
            self.e_z += 2.0 ** -23 * self.z.abs().amax(dim=1)
        self.lse = torch.logsumexp(self.z, dim=1)
        self.e_lse = self.e_z + 2.0 ** -22 * (1 + self.lse.abs())
        away = self.z - self.lse.unsqueeze(1)
        self.q = torch.exp(away)
        rel = 2 * self.e_z.unsqueeze(1) + 2.0 ** -21 * (1 + away.abs() + self.lse.abs().unsqueeze(1)) + (2.0 ** -11 if bf else 0.0)
        self.e_q = self.q * rel + 2.0 ** -63


class Gradients:
    """g_h and g_W of blocks of g, and their errors."""

    def __init__(self, h, W):
        self.W, self.T, self.io = W.double(), len(h), h.dtype
        self.g_h, self.e_h = [], []
        self.g_W, self.e_W = torch.zeros_like(self.W), torch.zeros_like(self.W)

    def add(self, x, g, e_g):
        """rows x of h (64 bits) with the gradients g on their logits; rows of g that are 0 read nothing of x."""
        e_g = e_g + last(self.io) * g.abs()
        x = x.masked_fill(~(g != 0).any(dim=1, keepdim=True), 0.0)
        self.g_h.append(g @ self.W)
        self.e_h.append((e_g + summed(len(self.W), self.io) * g.abs()) @ self.W.abs())
        self.g_W += g.t().contiguous() @ x
        self.e_W += (e_g + summed(self.T, self.io) * g.abs()).t().contiguous() @ x.abs()

    def results(self):
        g_h, e_h = torch.cat(self.g_h), torch.cat(self.e_h)
        return dict(g_h=(g_h, e_h + last(self.io) * g_h.abs()), g_W=(self.g_W, self.e_W + last(self.io) * self.g_W.abs()))


def within(got, ref, bound, what):
    assert got.shape == ref.shape
    over = (got.double() - ref).abs() / bound.clamp(min=1e-45)
    assert bool((over <= 1).all()), f"{what}: {float(over.max()):.3f} of the bound"


def distill(h, W, ids, logits, weight, tau, rows=1024):
    """{name: (result, largest error)}; weight [T] or None.  The teacher's probabilities, of logits a / tau: 2^-21 of the largest |a / tau| (the
    difference from the largest one is at most twice that, and has three roundings of 2^-24: its own, the factor's, the product's) and 2^-20 of themselves (exp, a sum of at most ten additions, a division);
    their logarithms as much and 2^-21 of their own."""
    held = (ids >= 0) & (logits > -float("inf"))
    counts = held.any(dim=1)
    w = torch.full((len(h),), 1.0 / max(1, int(counts.sum())), device=h.device, dtype=torch.float64) if weight is None else weight.double()
    w = torch.where(counts, w, 0.0)
    out = {k: [] for k in ("loss", "e_loss", "lse", "e_lse")}
    grads = Gradients(h, W)
    for t0 in range(0, len(h), rows):
        b = slice(t0, t0 + rows)
        L = Logits(h[b], W, 1.0 / tau)
        on, at = held[b], ids[b].long().clamp(min=0)
        a = (logits[b].double() / tau).masked_fill(~on, -1e300)
        p = torch.softmax(a, dim=1).masked_fill(~on, 0.0)
        top = a.abs().masked_fill(~on, 0.0).amax(dim=1, keepdim=True)
        log_p = torch.where(p > 0, p, 1.0).log()
        rel_p = 2.0 ** -21 * top + 2.0 ** -20
        z = L.z.gather(1, at)
        log_q = z - L.lse.unsqueeze(1)
        terms = log_p - log_q
        e = (p * rel_p * terms.abs() + p * (rel_p + 2 * L.e_z.unsqueeze(1) + 2.0 ** -21 * (1 + z.abs() + L.lse.abs().unsqueeze(1) + log_p.abs()))
             + 2.0 ** -20 * (p * terms).abs())
        out["loss"].append((p * terms).sum(dim=1))
        out["e_loss"].append(e.sum(dim=1))
        out["lse"].append(L.lse)
        out["e_lse"].append(L.e_lse)
        teacher = torch.zeros_like(L.q).scatter_add_(1, at, p)
        e_teacher = torch.zeros_like(L.q).scatter_add_(1, at, p * rel_p)
        v = (w[b] / tau).unsqueeze(1)
        on = v != 0
        grads.add(L.x, ((L.q - teacher) * v).masked_fill(~on, 0.0), ((L.e_q + e_teacher + 2.0 ** -21 * (L.q + teacher)) * v.abs()).masked_fill(~on, 0.0))
    out = {k: torch.cat(v) for k, v in out.items()}
    return dict(loss=(out["loss"], out["e_loss"]), lse=(out["lse"], out["e_lse"]), **grads.results())


def preference(h, W, targets, offsets, reference, weight, beta, smoothing, rows=1024):
    """{name: (result, largest error)}.  A pair's margin has beta times the errors of its log probabilities, its loss that, and the tokens' weights
    a quarter of it; each 2^-23 of itself."""
    beta, smoothing = (float(torch.tensor(v, dtype=F)) for v in (beta, smoothing))
    bounds = offsets.tolist()
    n = len(bounds) - 1
    ce, e_ce = (torch.zeros(len(h), dtype=torch.float64, device=h.device) for _ in range(2))
    for t0 in range(0, len(h), rows):
        b = slice(t0, t0 + rows)
        L = Logits(h[b], W)
        y = targets[b].long()
        z_y = L.z.gather(1, y.clamp(min=0).unsqueeze(1)).squeeze(1)
        ce[b] = torch.where(y >= 0, L.lse - z_y, 0.0)
        e_ce[b] = torch.where(y >= 0, 2 * L.e_z + 2.0 ** -22 * (1 + L.lse.abs() + z_y.abs()), 0.0)
    seq = [slice(bounds[i], bounds[i + 1]) for i in range(n)]
    logp = -torch.stack([ce[s].sum() for s in seq]) if n else ce[:0]
    e_logp = torch.stack([e_ce[s].sum() for s in seq]) if n else ce[:0]
    ratio = logp - (0.0 if reference is None else reference.double())
    m = beta * (ratio[0::2] - ratio[1::2])
    e_m = abs(beta) * (e_logp[0::2] + e_logp[1::2])
    soft = torch.nn.functional.softplus
    loss = (1 - smoothing) * soft(-m) + smoothing * soft(m)
    slope = smoothing * torch.sigmoid(m) - (1 - smoothing) * torch.sigmoid(-m)
    v = torch.full_like(m, 1.0 / max(1, len(m))) if weight is None else weight.double()
    w, e_w = (torch.zeros(len(h), dtype=torch.float64, device=h.device) for _ in range(2))
    for i, s in enumerate(seq):
        w[s] = (-beta if i % 2 == 0 else beta) * slope[i // 2] * v[i // 2]
        e_w[s] = abs(beta) * v[i // 2].abs() * 0.25 * e_m[i // 2] + 2.0 ** -23 * w[s].abs()
    there = targets >= 0
    w, e_w = torch.where(there, w, 0.0), torch.where(there, e_w, 0.0)
    grads = Gradients(h, W)
    for t0 in range(0, len(h), rows):
        b = slice(t0, t0 + rows)
        L = Logits(h[b], W)
        hit = torch.nn.functional.one_hot(targets[b].long().clamp(min=0), len(W)).double()
        on = (w[b] != 0).unsqueeze(1)
        g = ((L.q - hit) * w[b].unsqueeze(1)).masked_fill(~on, 0.0)
        grads.add(L.x, g, (L.e_q * w[b].abs().unsqueeze(1) + (L.q + hit) * e_w[b].unsqueeze(1)).masked_fill(~on, 0.0))
    return dict(loss=(loss, 1.01 * e_m + 2.0 ** -23 * loss + 1e-30), logp=(logp, e_logp + 2.0 ** -23 * logp.abs()), **grads.results())
