"""Steps whose singular values become very small before they grow again, against the steps in 64 bits."""
import zlib

import pytest
import torch

import orthogonal_util as O
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


SMALL = [[(1e-5, 0.0, 0.0), (1e5, -5e14, 0.0)], [(1e-7, 0.0, 0.0), (1e7, -5e20, 0.0), (1.5, -0.5, 0.0)], [(0.0, 0.0, 1e-4), (1e4, -3e11, 0.0), (3.0, -3.0, 1.0)]]


@pytest.mark.parametrize("k", SMALL, ids=["1e-5", "1e-7", "1e-4 of the fifth"])
@pytest.mark.parametrize("kind", [F32, BF16], ids=str)
@pytest.mark.parametrize("size", [(40, 60), (300, 260)], ids=str)
def test_steps_through_very_small_values(size, kind, k):
    """What is held between products keeps its 22 bits wherever the largest of it is."""
    g = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(size).encode()))
    m = (torch.randn(size[0], 1, device="cuda", generator=g) * torch.randn(1, size[1], device="cuda", generator=g) + 0.05 * torch.randn(size, device="cuda", generator=g)).to(kind)
    O.check(layers.orthogonalize(m, coefficients=k, steps=len(k)), m, kind, len(k), k)
