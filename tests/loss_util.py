"""References in 64 bits for the loss of a linear layer and its gradients, and the bounds that the results are held to.

A logit is an fp32 sum of K products and a bias: off by (K + 8) 2^-24 times the sum of their magnitudes, `dz` below, largest over a row's classes.  lse moves by no
more than its logits do; beside that its sum of N exponentials is off by a unit for each addition on the longest way (at most 64 + N / 64 of them here) and by the
exponentials' own arithmetic, F = 16 units and a unit for each binary digit of their argument's size (|z - top| 2^-24, weighed by e^-|z - top| no more than one), and it is rounded once.  A probability p = exp(z - lse) is off by p times (the
logit's error, lse's, 2^-24 |z - lse| and F)."""
import torch

from layers_util import E, F, TINY, U, d64


def logits(a, w, bias):
    """(z, the bound of its error)"""
    a, w = d64(a), d64(w)
    b = d64(bias) if bias is not None else torch.zeros(w.shape[0], dtype=torch.float64)
    return a @ w.t() + b, (a.shape[1] + 8) * E * (a.abs() @ w.abs().t() + torch.where(torch.isfinite(b), b.abs(), 0.0))


def counts(labels, weight, classes, rows):
    labels = labels[:rows].cpu().long()
    has = (labels >= 0) & (labels < classes)
    w = torch.ones(rows, dtype=torch.float64) if weight is None else d64(weight)[:rows]
    return labels.clamp(0, classes - 1), has, torch.where(has, w, 0.0)


def loss(a, w, labels, bias=None, weight=None, rows=None):
    """{name: (value, bound)} of lse, row_loss, total and loss over the first `rows` rows."""
    rows = a.shape[0] if rows is None else rows
    z, err = logits(a[:rows], w, bias)
    n = z.shape[1]
    at, has, weights = counts(labels, weight, n, rows)
    lse = torch.logsumexp(z, 1)
    finite = torch.where(torch.isfinite(z), err, 0.0).amax(1)
    lse_err = finite + E * (64 + n / 64 + 20) + F
    picked = z.gather(1, at[:, None])[:, 0]
    each = torch.where(has, lse - picked, 0.0)
    each_err = torch.where(has, lse_err + err.gather(1, at[:, None])[:, 0] + E * (picked.abs() + each.abs()), 0.0)  # (the logit is held in 32 bits, and so is the difference)
    on = weights != 0
    total = weights[on].sum()
    mean, mean_err = torch.zeros((), dtype=torch.float64), torch.zeros((), dtype=torch.float64)
    if total != 0:
        mean = (weights[on] * each[on]).sum() / total
        mean_err = (weights[on].abs() * (each_err[on] + E * each[on].abs())).sum() / total.abs() + 4 * E * mean.abs()
    return {"lse": (lse, lse_err + E * lse.abs()), "row_loss": (each, each_err), "total": (total.reshape(1), E * total.abs().reshape(1)), "loss": (mean.reshape(1), mean_err.reshape(1))}


def gradients(a, w, labels, kind, bias=None, weight=None, rows=None, dloss=1.0, mean=True):
    """((da, bound), (dw, bound), (dbias, bound)).  dz / (dloss / total) is held in `kind`, rounded once, for fp16 scaled so that the largest weight is at the top of its range."""
    rows = a.shape[0] if rows is None else rows
    z, err = logits(a[:rows], w, bias)
    n = z.shape[1]
    at, has, weights = counts(labels, weight, n, rows)
    total = weights.sum() if mean else torch.ones((), dtype=torch.float64)
    g = dloss / total if total != 0 else torch.zeros((), dtype=torch.float64)
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(z - lse)
    size = torch.where(torch.isfinite(z), (z - lse).abs(), 0.0)
    p_err = p * (torch.where(torch.isfinite(z), err, 0.0) + err.amax(1, keepdim=True) + E * (64 + n / 64 + 20 + size + lse.abs()) + 2 * F)
    dz = p.clone()
    dz[torch.arange(rows), at] -= has.double()
    dz = torch.where(weights[:, None] != 0, dz * weights[:, None], 0.0)
    top = weights.abs().max() if rows else torch.zeros(())
    err32 = p_err * weights[:, None].abs() + 2 * E * dz.abs() + torch.where(weights[:, None] != 0, 2 * E * weights[:, None].abs() * p, 0.0)
    held = err32 if kind == torch.float32 else err32 + U[kind] * dz.abs() + (top * 2.0**-38 if kind == torch.float16 else 2.0**-133)
    a, w = d64(a)[:rows], d64(w)
    u, out = U[kind], []
    for left, left_err, right, k in ((dz, held, w, n), (dz.t(), held.t(), a, rows)):
        want = g * (left @ right)
        b = g.abs() * (left_err @ right.abs() + (k + 8) * E * (left.abs() @ right.abs())) + 4 * E * want.abs()
        out.append((want, b * (1 + u) + u * want.abs() + TINY[kind]))
    out.append((g * dz.sum(0), g.abs() * (err32.sum(0) + (rows + 8) * E * dz.abs().sum(0)) + 4 * E * (g * dz.sum(0)).abs()))
    return out
