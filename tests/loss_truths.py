"""Plain 64-bit forms of the losses over a layer's outputs, and the error bounds that
follow from how the library computes them (torch only, no code of the library; on
whatever device the inputs are)."""
from __future__ import annotations

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}    # one rounding
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # spacing near zero
EPS = 2.0 ** -24


def logits(F, X, bias, temperature=1.0):
    z = F.double() @ X.double()
    if bias is not None:
        z = z + bias.double()[:, None]
    return z / temperature


def teacher(top, index, kn, temperature):
    """(q with zeros where an entry does not count, the columns that have any, the
    columns with an index beyond the classes)."""
    v = top.double() / temperature
    counts = (index >= 0) & (top.double() != -torch.inf)
    v = torch.where(counts, v, -torch.inf)
    best = v.max(0).values
    e = torch.where(counts, torch.exp(v - torch.where(best.abs() < torch.inf, best, 0.0)), 0.0)
    some = counts.any(0)
    return e / torch.where(some, e.sum(0), 1.0), some, (counts & (index >= kn)).any(0)


def targets(case, kn, t, device):
    """(entries' classes [k, t], their weights q, which columns count, which are
    invalid, T)."""
    if "labels" in case:
        y = case["labels"].long()
        keep = y != case["ignore"]
        bad = keep & ((y < 0) | (y >= kn))
        return torch.where(keep & ~bad, y, 0)[None], (keep & ~bad).double()[None], keep, bad, 1.0
    q, some, bad = teacher(case["top"], case["index"], kn, case["temperature"])
    return case["index"].long().clamp(0, max(kn - 1, 0)), q, some, bad, case["temperature"]


def forward(F, X, bias, case):
    """(loss, lse) of the definition."""
    kn, t = F.shape[0], X.shape[1]
    at, q, keep, bad, T = targets(case, kn, t, F.device)
    z = logits(F, X, bias, T)
    lse = torch.logsumexp(z, 0)
    per = torch.where(q > 0, q * (torch.log(torch.where(q > 0, q, 1.0)) - (z.gather(0, at) - lse)), 0.0)
    loss = torch.where(keep, T * T * per.sum(0), 0.0)
    return torch.where(bad, torch.nan, loss), lse


def slopes(F, X, bias, case, g):
    """dZ of the definition; columns that do not count, or with g = 0, are zero."""
    kn, t = F.shape[0], X.shape[1]
    at, q, keep, bad, T = targets(case, kn, t, F.device)
    z = logits(F, X, bias, T)
    d = torch.exp(z - torch.logsumexp(z, 0))
    d.scatter_add_(0, at, -q)
    w = torch.where(keep, g.double() * T, 0.0)
    return torch.where(w == 0, 0.0, d * w)


def backward(F, X, bias, case, g):
    d = slopes(F, X, bias, case, g)
    counted = torch.where((d != 0).any(0), X.double(), 0.0)
    return F.double().t() @ d, d @ counted.t(), d.sum(1)


def logit_bound(F, X, bias, T):
    """fp32 sums of ci products and the bias, and the division by T."""
    sums = F.double().abs() @ X.double().abs() + (0 if bias is None else bias.double().abs()[:, None])
    return 1.001 * (F.shape[1] + 6) * EPS * sums / T


def forward_bound(F, X, bias, case):
    """Bounds of (loss, lse).  The exponentials' arguments are off by the logits'
    error and by two roundings of a difference of at most the column's spread; the
    exponential by 2^-22; a sum runs through at most 256 additions; then a logarithm
    and an addition.  The targets' weights by as much, each times its logarithm."""
    kn, t = F.shape[0], X.shape[1]
    at, q, _, _, T = targets(case, kn, t, F.device)
    z, ez = logits(F, X, bias, T), logit_bound(F, X, bias, T)
    finite = torch.where(z.abs() < torch.inf, z, 0.0)
    lse = torch.logsumexp(z, 0)
    spread = finite.max(0).values - finite.min(0).values
    el = ez.max(0).values + 4 * EPS * spread + 4 * EPS + 256 * EPS + 4 * EPS * (lse.abs() + finite.abs().max(0).values)
    if "labels" in case:
        return el + ez.gather(0, at)[0] + 4 * EPS * (lse.abs() + z.gather(0, at)[0].abs()), el
    v = case["top"].double() / T
    v = torch.where(v.abs() < torch.inf, v, 0.0)
    eq = 4 * EPS * (v.max(0).values - v.min(0).values) + (case["top"].shape[0] + 16) * EPS          # relative, of q
    log_q = torch.log(torch.where(q > 0, q, 1.0)).abs()
    miss = (log_q + (z.gather(0, at) - lse).abs())
    per = q * (el + ez.gather(0, at) + eq * (1 + miss) + 8 * EPS * (miss + lse.abs() + z.gather(0, at).abs()))
    return T * T * (per.sum(0) + (case["top"].shape[0] + 8) * EPS * (q * miss).sum(0)), el


def backward_bound(F, X, bias, case, g, dtype):
    """Bounds of dX, dF, dbias: p by the errors of its exponent, the weights as above,
    a subtraction and two products; one rounding of dZ to the type (not for dbias;
    16-bit types: times a factor, below which 2^-39 of the largest g T is lost);
    fp32 sums; one rounding of each result."""
    kn, t = F.shape[0], X.shape[1]
    at, q, keep, _, T = targets(case, kn, t, F.device)
    d = slopes(F, X, bias, case, g)
    z, ez = logits(F, X, bias, T), logit_bound(F, X, bias, T)
    lse = torch.logsumexp(z, 0)
    p = torch.exp(z - lse)
    _, el = forward_bound(F, X, bias, case)
    w = torch.where(keep, g.double().abs() * T, 0.0)
    far = torch.where(z.abs() < torch.inf, (z - lse).abs(), 0.0)
    e = p * (ez + el + 4 * EPS * far + 16 * EPS + 4 * EPS * lse.abs())
    top = 0.0 if "labels" in case else case["top"].double() / T
    eq = 16 * EPS if "labels" in case else 4 * EPS * (torch.where(top.abs() < torch.inf, top, 0.0)).abs().max() * 2 + (q.shape[0] + 32) * EPS
    e = w * e.scatter_add(0, at, q * eq) + 8 * EPS * (d.abs() + w * p)
    u = UNIT[dtype]
    held = e + u * (d.abs() + e) + (TINY[dtype] if dtype == torch.float32 else w.max() * 2.0 ** -39)
    held = torch.where(w == 0, 0.0, held)
    big = d.abs() + held
    Fa, Xa = F.double().abs(), torch.where(w == 0, 0.0, X.double().abs())
    eX = Fa.t() @ held + 1.001 * (kn + 16) * EPS * (Fa.t() @ big)
    eF = held @ Xa.t() + 1.001 * (t + 16) * EPS * (big @ Xa.t())
    eb = e.sum(1) + 1.001 * (t + 16) * EPS * (d.abs() + e).sum(1)
    want = backward(F, X, bias, case, g)
    return tuple(e_ + u * (r.abs() + e_) + TINY[dtype] for e_, r in zip((eX, eF, eb), want))
