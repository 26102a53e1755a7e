"""References in 64 bits for the dense operators (numpy / torch on the host), and the bounds that their results are held to.

A result is rounded to its type once (unit roundoff u: 2^-24, 2^-11, 2^-8), after fp32 sums of at most K terms whose error is at most
K 2^-24 times the sum of the terms' magnitudes, whatever the order.  `F` = 16 units of fp32 covers an activation's own arithmetic
(a few operations and a library exp or erf of one or two units each), relative to its input's magnitude: |act(z)| <= |z|, and its slope's
bound is taken relative to 1 + |z|."""
import math

import numpy as np
import torch

U = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
TINY = {torch.float32: 2.0**-149, torch.float16: 2.0**-24, torch.bfloat16: 2.0**-133}
E = 2.0**-24
F = 16 * E


def philox(c, k):
    """Philox4x32-10 on numpy uint64 arrays of 32-bit words."""
    u = np.uint64
    low = u(0xFFFFFFFF)
    c = [np.asarray(x, dtype=u) for x in c]
    k = [u(k[0]), u(k[1])]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ k[0], b & low, (a >> u(32)) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + u(0x9E3779B9)) & low, (k[1] + u(0xBB67AE85)) & low]
    return c


def kept(p, key, layer, ids, cols):
    """Which cells a mask keeps: bool [len(ids), cols]."""
    ids = np.asarray(ids, dtype=np.int64).astype(np.uint32).astype(np.uint64)[:, None]
    c = np.arange(cols, dtype=np.uint64)[None, :]
    words = philox([ids + 0 * c, c // np.uint64(8) + 0 * ids, np.uint64(layer) + 0 * (c + ids), np.uint64(1) + 0 * (c + ids)],
                   (key & 0xFFFFFFFF, key >> 32 & 0xFFFFFFFF))
    which = (np.arange(cols) // 2) % 4
    word = np.choose(which[None, :], words)
    bits = np.where(np.arange(cols)[None, :] % 2 == 1, word >> np.uint64(16), word & np.uint64(0xFFFF))
    return torch.from_numpy(bits >= np.uint64(math.floor(p * 65536 + 0.5)))


def drop(x, mask, ids=None):
    """`x` (64 bits, host) through a mask given as (p, key, layer); dropped cells are 0 whatever they are."""
    if mask is None or mask[0] == 0:
        return x
    p, key, layer = mask
    t = math.floor(p * 65536 + 0.5)
    if t == 65536:
        return torch.zeros_like(x)
    k = kept(p, key, layer, range(x.shape[0]) if ids is None else ids, x.shape[1])
    return torch.where(k, x * (65536 / (65536 - t)), torch.zeros_like(x))


def act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        g = torch.sigmoid(z)
        return g + z * g * (1 - g)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def d64(t):
    return t.detach().cpu().double()


def check(got, want, bound, what=""):
    """Every element within its bound (infinities and NaN in the same places)."""
    got = d64(got)
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    fine = torch.isfinite(want)
    rest = ~fine & ~torch.isnan(want)
    assert torch.equal(got[rest], want[rest]), f"{what}: infinities"
    err, bound = (got - want).abs()[fine], bound.expand_as(want)[fine]
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {err.numel()} off, worst {float((err / bound).max()):.3g} bounds"


def linear(a, w, bias, residual, name, mask, kind, scale_a=None, scale_w=None, ids=None):
    """(y, its bound, z, its bound) in 64 bits."""
    a, w = d64(a), d64(w)
    if scale_a is not None:
        a = a * d64(scale_a)[:, None]
    if scale_w is not None:
        w = w * d64(scale_w)[:, None]
    b = d64(bias) if bias is not None else torch.zeros(w.shape[0], dtype=torch.float64)
    z = a @ w.t() + b
    size = a.abs() @ w.abs().t() + b.abs()
    z_err = (a.shape[1] + 8) * E * size  # the scales' products and the bias are five operations more
    v, v_err = act(z, name), 1.2 * z_err + (F * z.abs() if name != "none" else 0)  # (no activation is steeper than 1.13)
    y, grown = drop(v, mask, ids), 1.0
    if mask is not None and 0 < mask[0] < 1:
        grown = 65536 / (65536 - math.floor(mask[0] * 65536 + 0.5))
    y_err = grown * (v_err + 2 * E * v.abs())
    if residual is not None:
        y = y + d64(residual)
        y_err = y_err + E * y.abs()
    u, tiny = U[kind], TINY[kind]
    return y, y_err * (1 + u) + u * y.abs() + tiny, z, z_err * (1 + u) + u * z.abs() + tiny


def linear_grads(dy, a, w, z, name, mask, kind, rows=None, ids=None):
    """((da, bound), (dw, bound), (dbias, bound)) in 64 bits, over the first `rows` rows."""
    n = dy.shape[0] if rows is None else rows
    dy, a, w = d64(dy)[:n], d64(a)[:n], d64(w)
    s = slope(d64(z)[:n], name) if name != "none" else torch.ones_like(dy)
    zs = d64(z)[:n].abs() if name != "none" else torch.zeros_like(dy)
    dz = drop(dy * s, mask, None if ids is None else ids[:n])
    live = drop(dy, mask, None if ids is None else ids[:n]).abs()
    err32 = live * (F * (1 + zs) + 2 * E)
    u = U[kind]
    exact = name in ("none", "relu")
    err = err32 if exact else err32 + u * dz.abs() + TINY[kind]  # dz is an operand in the type
    out = []
    for left, left_err, right, k in ((dz, err, w, dz.shape[1]), (dz.t(), err.t(), a, n)):
        want = left @ right
        b = left_err @ right.abs() + (k + 8) * E * (left.abs() @ right.abs())
        out.append((want, b * (1 + u) + u * want.abs() + TINY[kind]))
    out.append((dz.sum(0), err32.sum(0) + (n + 8) * E * dz.abs().sum(0)))
    return out
