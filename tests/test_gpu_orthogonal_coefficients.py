"""Coefficients of every kind against the steps in 64 bits: a bfloat16 result is off by no more than stated with the operator."""
import zlib

import pytest
import torch

import orthogonal_util as O
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
STATED = 4.0e-3  # of the length of as many singular values of one, beside a bfloat16 result's own rounding

# triples for each step that take small singular values up faster, with a factor of 1.01 against rounding
FAST = [(8.28721201814563, -23.595886519098837, 17.300387312530933), (4.107059111542203, -2.9478499167379106, 0.5448431082926601), (3.9486908534822946, -2.908902115962949, 0.5518191394370137),
        (3.3184196573706015, -2.488488024314874, 0.51004894012372), (2.300652019954817, -1.6689039845747493, 0.4188073119525673)]
SAFE = [(a / 1.01, b / 1.01**3, c / 1.01**5) for a, b, c in FAST]
SETS = {"default": [O.MUON] * 5, "default 4": [O.MUON] * 4, "default 6": [O.MUON] * 6, "fast": FAST, "safe": SAFE, "safe 3": SAFE[:3], "cubic 6": [(1.5, -0.5, 0.0)] * 6, "quintic 6": [(2.0, -1.5, 0.5)] * 6}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _gen(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def _matrix(what, rows, cols):
    g = _gen(what, rows, cols)
    noise = torch.randn(rows, cols, device="cuda", generator=g)
    if what == "one direction":
        return torch.randn(rows, 1, device="cuda", generator=g) * torch.randn(1, cols, device="cuda", generator=g) + 0.05 * noise
    if what == "even":  # all singular values alike
        return (torch.linalg.qr(noise.t().double())[0].t() if rows <= cols else torch.linalg.qr(noise.double())[0]).float().contiguous()
    return noise


@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("what", ["noise", "one direction", "even"])
@pytest.mark.parametrize("size", [(256, 256), (256, 1500), (700, 300), (400, 400)], ids=str)
def test_a_result_of_16_bits_is_as_near_as_stated(size, what, name):
    """Its error has two parts, the products' (STATED) and its own rounding, which have nothing to do with each other: over 65536 cells and more their lengths add up as sides of a right angle, to within
    three standard deviations of what their directions have in common, 3 / 256 of either."""
    m, k = _matrix(what, *size).to(BF16), SETS[name]
    want = O.exact(m, len(k), k)
    rounding = float((want.bfloat16().double() - want).norm())
    off = float((layers.orthogonalize(m, coefficients=k, steps=len(k)).double() - want).norm())
    assert off <= 1.012 * (STATED**2 * min(size) + rounding**2) ** 0.5, off / min(size) ** 0.5


def test_an_update_of_16_bits_is_as_near_as_stated():
    for name in ("default 6", "safe"):
        k, (rows, cols) = SETS[name], (300, 700)
        g, m = _matrix("noise", rows, cols), torch.zeros(rows, cols, device="cuda")
        w = torch.zeros(rows, cols, device="cuda", dtype=BF16)
        layers.muon_step(w, m, g, lr=1.0, momentum=0.0, nesterov=False, scale=1.0, steps=len(k), coefficients=k)
        want = -O.exact(g, len(k), k)
        rounding = float((want.bfloat16().double() - want).norm())
        assert float((w.double() - want).norm()) <= 1.012 * (STATED**2 * rows + rounding**2) ** 0.5
