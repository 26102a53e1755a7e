"""The Newton-Schulz steps in 64 bits, and what their result may be off by.

The steps grow small singular values by up to 3.4 each, and with them what is off in the matrix: a bound that holds for every matrix is far above what any of them shows.  So the tolerance is the error
of the documented arithmetic itself, carried through the steps for the matrix at hand, in 64 bits: every value that is held between products is rounded as it is held (two fp16 planes: 22 bits; one plane as an operand of
a bfloat16 result's products), and every sum of K products is disturbed by a random sum of K / 16 roundings to fp32 (the matrix instructions round once for 16 products), each of 2^-24 of the sum's size.  A result's
distance from the exact one may be `SLACK` times what that leaves (in length; a single cell's `CELL` times its share), and its own rounding."""
import math

import torch

E, SLACK, CELL = 2.0**-24, 4.0, 40.0
U = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
MUON = (3.4445, -4.7750, 2.0315)


def _triples(coefficients, steps):
    return [coefficients] * steps if isinstance(coefficients[0], float) else list(coefficients)


def single(rows, cols, steps, kind):
    """Whether the products' operands are single fp16 planes."""
    return kind == torch.bfloat16 and min(rows, cols) >= 256 and steps <= 6


def exact(g, steps=5, coefficients=MUON, eps=1e-7):
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x = x / (x.pow(2).sum().sqrt() + eps)
    for a, b, c in _triples(coefficients, steps):
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def emulated(g, kind, steps=5, coefficients=MUON, eps=1e-7):
    """The steps with the roundings of their documented arithmetic."""
    one = single(*g.shape, steps, kind)
    gen = torch.Generator(device=g.device).manual_seed(1)

    def high(v, top):
        scale = 2.0 ** (14 - math.ceil(math.log2(top))) if top > 0 else 1.0
        return (v * scale).half().double() / scale

    def pair(v, top):
        h = high(v, top)
        return h + high(v - h, top)

    def product(x, top_x, y, top_y):
        if one:
            x, y = high(x, top_x), high(y, top_y)
        size = x.abs() @ y.abs()
        rounds = max(1.0, x.shape[1] * (1 if one else 3) / 16) ** 0.5
        return x @ y + size * (E * rounds) * torch.randn(size.shape, dtype=torch.float64, device=g.device, generator=gen)

    held = high if one else pair
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x, top = pair(x / (x.pow(2).sum().sqrt() + eps), 1.0), 1.0  # (top: the largest that a singular value can be, which the planes' exponent goes by)
    for a, b, c in _triples(coefficients, steps):
        v = torch.linspace(0, top, 10001, dtype=torch.float64)
        top_b, top_x = float((b * v**2 + c * v**4).abs().max()), float((a * v + b * v**3 + c * v**5).abs().max())
        s = held(product(x, top, x.t().contiguous(), top), top * top)
        x = pair(a * x + product(held(b * s + c * product(s, top * top, s, top * top), top_b), top_b, x, top), top_x)
        top = top_x
    return x.t() if tall else x


def check(got, g, kind, steps=5, coefficients=MUON, eps=1e-7, what=""):
    want = exact(g, steps, coefficients, eps)
    off = (emulated(g, kind, steps, coefficients, eps) - want).norm()
    err = got.double() - want
    cells, length = want.numel() ** 0.5, want.norm()
    assert float(err.norm()) <= float(SLACK * off + U[kind] * length + 1e-30), (what, float(err.norm() / length), float(off / length))
    worst = (err.abs() - U[kind] * want.abs()).max()
    assert float(worst) <= float(CELL * off / cells + 2.0**-24 * length / cells + 1e-30), (what, float(worst), float(off / cells))
