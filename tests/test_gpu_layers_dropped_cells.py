"""Gradients of a product where the activation's stored input is not finite, in cells that dropout left out."""
import pytest
import torch

import layers_util as R
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

KINDS = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_a_dropped_cell_has_no_gradient_whatever_its_input_is(act, kind):
    rows, k, n, mask = 130, 40, 203, (0.5, 31337, 4)
    g = torch.Generator(device="cuda").manual_seed(5)
    keep = R.kept(*mask, range(rows), n).cuda()
    a, w = torch.randn(rows, k, device="cuda", generator=g).to(kind), torch.randn(n, k, device="cuda", generator=g).to(kind)
    dy, z = torch.randn(rows, n, device="cuda", generator=g).to(kind), torch.randn(rows, n, device="cuda", generator=g).to(kind)
    drop = layers.Dropout(*mask)
    want = layers.linear_backward(dy, a, w, preact=torch.where(keep, z, 0), act=act, dropout=drop)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for dy_too in (False, True):
            got = layers.linear_backward(torch.where(keep, dy, bad) if dy_too else dy, a, w, preact=torch.where(keep, z, bad), act=act, dropout=drop)
            for x, y, what in zip(got, want, ("da", "dw", "dbias")):
                assert torch.equal(x, y), (what, bad, dy_too)
