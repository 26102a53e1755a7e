"""The Newton-Schulz steps in 64 bits, and what their result may be off by.

The steps grow small singular values by up to 3.4 each, and with them what is off in the matrix: a bound that holds for every matrix is far above what any of them shows.  So the tolerance is the error
of the documented arithmetic itself, carried through the steps for the matrix at hand, in 64 bits: every value that is held between products is rounded as it is held (two fp16 planes: 22 bits; one plane as an operand of
a bfloat16 result's products), and every sum of K products is disturbed by a random sum of K / 16 roundings to fp32 (the matrix instructions round once for 16 products), each of 2^-24 of the sum's size.  A result's
distance from the exact one may be `SLACK` times what that leaves (in length; a single cell's `CELL` times its share), and its own rounding."""
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

    def high(v):
        return (v * 2.0**13).half().double() * 2.0**-13

    def pair(v):
        h = high(v)
        return h + high(v - h)

    def product(x, y):
        if one:
            x, y = high(x), high(y)
        size = x.abs() @ y.abs()
        rounds = max(1.0, x.shape[1] * (1 if one else 3) / 16) ** 0.5
        return x @ y + size * (E * rounds) * torch.randn(size.shape, dtype=torch.float64, device=g.device, generator=gen)

    held = high if one else pair
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x = pair(x / (x.pow(2).sum().sqrt() + eps))
    for a, b, c in _triples(coefficients, steps):
        s = held(product(x, x.t().contiguous()))
        x = pair(a * x + product(held(b * s + c * product(s, s)), x))
    return x.t() if tall else x


def check(got, g, kind, steps=5, coefficients=MUON, eps=1e-7, what=""):
    want = exact(g, steps, coefficients, eps)
    off = (emulated(g, kind, steps, coefficients, eps) - want).norm()
    err = got.double() - want
    cells, length = want.numel() ** 0.5, want.norm()
    assert float(err.norm()) <= float(SLACK * off + U[kind] * length + 1e-30), (what, float(err.norm() / length), float(off / length))
    worst = (err.abs() - U[kind] * want.abs()).max()
    assert float(worst) <= float(CELL * off / cells + 2.0**-24 * length / cells + 1e-30), (what, float(worst), float(off / cells))
