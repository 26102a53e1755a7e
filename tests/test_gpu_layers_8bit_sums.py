"""Sums of 8-bit operands whose products differ by orders of magnitude - one large column in eight, as a few channels of a hidden layer
are - at every kernel's sizes: they are held to what an fp32 sum of the same terms may lose, like the sums of any other type."""
import pytest
import torch

import layers_util as R
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


# a few rows, one tile or a few, many large tiles, operands that lie anyhow; sums shorter and longer than 512 terms
SIZES = [(1, 512, 16), (4, 504, 8), (300, 640, 257), (20000, 320, 264), (20000, 1024, 264), (9000, 4112, 2064), (20001, 1030, 257), (2000, 511, 40)]


@pytest.mark.parametrize("kind", ["one large in eight", "large ones that cancel", "large ones anywhere"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_large_columns_take_nothing_from_the_small_ones(size, kind):
    """2^-13 of 448 is a value of the type too, and 448 times 1 one product; the bound is layers_util's, (in + 8) 2^-24 of the terms' sum."""
    rows, k, n = size
    g = torch.Generator(device="cuda").manual_seed(rows + k)
    column = torch.arange(k, device="cuda")
    large = column % 8 == 5 if kind != "large ones anywhere" else torch.rand(k, device="cuda", generator=g) < 0.125
    sign = torch.where(column // 8 % 2 == 0, 1.0, -1.0) if kind == "large ones that cancel" else torch.ones(k, device="cuda")
    row = torch.where(large, 448.0 * sign, 448.0 * 2.0**-13)
    a = row.expand(rows, k).contiguous()
    a[1::2] *= 0.5  # (rows that differ, or a wrong row would not show)
    a[2::3, : k // 2] = 0
    w = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, 0.5)[:, None].expand(n, k).contiguous()
    a, w = a.to(F8), w.to(F8)
    some = torch.cat((torch.arange(min(rows, 300)), torch.arange(max(rows - 300, 0), rows))).unique()
    y = layers.linear(a, w, out_dtype=torch.float32)
    want = R.linear(a[some.cuda()].float(), w.float(), None, None, "none", None, torch.float32)
    R.check(y[some.cuda()], want[0], want[1])


def test_every_value_of_the_type_is_multiplied_exactly():
    """Each of the 256 codes against 1, alone in its row: the value itself, not a number where the code is that."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(F8)
    for rows, k, n in ((256, 16, 16), (256, 1024, 16), (20480, 1024, 264), (8192, 4096, 2048), (20224, 1030, 257)):
        a = torch.zeros(rows, k, device="cuda").to(F8)
        w = torch.zeros(n, k, device="cuda").to(F8)
        at = torch.arange(rows, device="cuda") * 37 % k
        a.view(torch.uint8)[torch.arange(rows, device="cuda"), at] = torch.arange(rows, device="cuda").remainder(256).to(torch.uint8)
        w[:] = torch.ones(1, device="cuda").to(F8)
        y = layers.linear(a, w, out_dtype=torch.float32)
        want = codes.float()[torch.arange(rows, device="cuda") % 256]
        assert torch.equal(torch.isnan(y), torch.isnan(want)[:, None].expand(rows, n))
        assert torch.equal(torch.nan_to_num(y, nan=0.0), torch.nan_to_num(want, nan=0.0)[:, None].expand(rows, n).contiguous())
