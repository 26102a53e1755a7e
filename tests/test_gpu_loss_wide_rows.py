"""Up to four rows as long as the kernel for a few rows takes them: four of 16 KB are all of the LDS that a launch has, and one element more goes another way."""
import zlib

import pytest
import torch

import layers_util as R
import loss_util as L
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


@pytest.mark.parametrize("kind", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("more", [-8, 0, 8])
def test_rows_of_16_kilobytes(rows, more, kind):
    k, n = 16384 // kind.itemsize + more, 333
    g = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((rows, more, str(kind))).encode()))
    a, w = (torch.randn(m, k, device="cuda", generator=g).mul(s).to(kind) for m, s in ((rows, 2.0), (n, k**-0.5)))
    labels = torch.randint(0, n, (rows,), device="cuda", generator=g)
    bias = torch.randn(n, device="cuda", generator=g)
    want = L.loss(a, w, labels, bias)
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, row_loss=True)
    for name in ("lse", "row_loss", "total", "loss"):
        R.check(getattr(r, name), *want[name], name)
    live = torch.tensor([rows - 1], dtype=torch.int32, device="cuda")
    some = layers.linear_cross_entropy(a, w, labels, bias=bias, rows=live, row_loss=True)
    assert torch.equal(some.lse[: rows - 1], r.lse[: rows - 1]) and torch.equal(some.row_loss[: rows - 1], r.row_loss[: rows - 1])
