"""Activations and their slopes cell by cell, where results are fp32: against 64 bits, relative to each value, over both tails."""
import math

import pytest
import torch

from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

E = 2.0**-24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _cells(kind):
    """Cells over -40 .. 40, dense around 0, as values of `kind`."""
    z = torch.cat((torch.linspace(-40, 40, 40001, dtype=torch.float64), torch.linspace(-6, 6, 24001, dtype=torch.float64), torch.logspace(-6, 0, 301, dtype=torch.float64)))
    return torch.cat((z, -z[-301:], torch.zeros(1, dtype=torch.float64))).to(kind)


def _silu(z):
    """(value, its bound, slope, its bound) at 64 bits.  exp is right to a unit in the last place (2 E) and its argument exact; the sum, the quotient
    and the product round once each; a factor of two for good measure.  The slope is g (1 + z (1 - g)): its sum cancels, so that bound goes by the terms.
    Below z = -87 (where exp(-z) leaves fp32) nothing is asked: the cells end at -40."""
    g = 1 / (1 + torch.exp(-z))
    v, s = z * g, g * (1 + z * (1 - g))
    return v, 12 * E * v.abs(), s, 16 * E * g * (1 + z.abs())


def _gelu(z):
    """The same for z Phi(z).  With x = -z / sqrt 2 rounded twice (3 E relative), erfc(x) moves by its condition number, up to z^2 + 2, and is itself
    right to 16 units in the last place (32 E), what the function's specification (OpenCL's) allows; exp(-z^2 / 2) in the slope moves by z^2 / 2 times
    the 2 E of its argument.  fp32 ends at 1e-45: a floor of 1e-37 where products go below the normal range."""
    phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    bell = z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    v, s = z * phi, phi + bell
    tail = (3 * (z * z + 2) + 40) * E
    return v, tail * v.abs() + 1e-37, s, tail * phi + (z * z + 12) * E * bell.abs() + 1e-37


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("large", [False, True])
def test_activations_of_fp32_results(act, large):
    """in = 1 and a weight of 1: z is the operand itself.  `large`: through the large tiles (in = 8, seven columns of zeros)."""
    z = _cells(torch.float32)
    want, bound = {"silu": _silu, "gelu": _gelu}[act](z.double())[:2]
    if large:
        a = torch.zeros(z.numel(), 8, device="cuda")
        w = torch.zeros(160, 8, device="cuda")
        a[:, 3], w[:, 3] = z.cuda(), 1.0
    else:
        a, w = z.cuda()[:, None], torch.ones(3, 1, device="cuda")
    y = layers.linear(a, w, act=act).double().cpu()
    err = (y - want[:, None]).abs()
    bad = ~(err <= bound[:, None])
    assert not bad.any(), f"{int(bad.any(1).sum())} cells, worst {float((err / bound[:, None]).nan_to_num(0).max()):.3g} bounds at z = {float(z[(err / bound[:, None]).nan_to_num(0).amax(1).argmax()]):.4g}"


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes_in_fp32_sums(act, kind):
    """One row of ones: the bias gradient (fp32 whatever the operands are) is the slope itself."""
    z = _cells(kind)
    z = z[: z.numel() // 8 * 8]
    want, bound = {"silu": _silu, "gelu": _gelu}[act](z.double())[2:]
    for i in range(0, z.numel(), 32768):
        part = z[i: i + 32768].cuda()[None]
        dy, a, w = torch.ones_like(part), torch.ones(1, 1, device="cuda", dtype=kind), torch.ones(part.shape[1], 1, device="cuda", dtype=kind)
        got = layers.linear_backward(dy, a, w, preact=part, act=act, need=(False, False, True))[2].double().cpu()
        at = slice(i, i + part.shape[1])
        err = (got - want[at]).abs()
        bad = ~(err <= bound[at])
        assert not bad.any(), f"{int(bad.sum())} cells, worst {float((err / bound[at]).nan_to_num(0).max()):.3g} bounds at z = {float(z[at][(err / bound[at]).nan_to_num(0).argmax()]):.4g}"
