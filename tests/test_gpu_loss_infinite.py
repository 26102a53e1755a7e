"""Rows of the loss whose logits hold an infinity or no number: lse, row_loss and the gradients are what the formulas give in IEEE arithmetic.  lse = log sum exp z is NaN where a logit is NaN, else
+infinity where one is that, else -infinity where nothing is finite; row_loss = lse - z[label]; exp(z - lse) is 0 for a finite z below an infinite lse and no number for an infinite one."""
import zlib

import pytest
import torch

from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
INF, NAN = float("inf"), float("nan")
SIZES = [  # rows, in, classes, elements between rows: few rows, few tiles, tiles that are narrow, of chunks, large, and of rows that lie anyhow
    (1, 64, 700, 0), (4, 128, 333, 0), (200, 64, 40, 0), (300, 64, 1003, 0), (70000, 264, 64, 0), (4097, 264, 2100, 0), (9000, 1032, 2064, 0), (30000, 133, 129, 1)]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _inputs(size, kind, *key):
    rows, k, n, pad = size
    g = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((size, str(kind), key)).encode()))
    a, w = ((torch.randn(m, k + pad, device="cuda", generator=g) * s).to(kind)[:, :k] for m, s in ((rows, 1.0), (n, k**-0.5)))
    return a, w, torch.randint(0, n, (rows,), device="cuda", generator=g), torch.randn(n, device="cuda", generator=g)


def _same_kind(got, want, what):
    """Not a number, +infinity and -infinity in the same places."""
    for name, of in (("NaN", torch.isnan), ("+infinity", torch.isposinf), ("-infinity", torch.isneginf)):
        assert torch.equal(of(got), of(want)), f"{what}: {name} at {of(got).nonzero().flatten()[:5].tolist()}, wanted at {of(want).nonzero().flatten()[:5].tolist()}"


@pytest.mark.parametrize("kind", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_classes_of_infinite_logits(size, kind):
    """Biases of +infinity (the one of class `up`), of NaN beside it, and of -infinity everywhere."""
    rows, _, n, _ = size
    a, w, labels, bias = _inputs(size, kind)
    up, bad = n // 2 + 1, n // 3
    labels[: rows // 2] = up
    plain = layers.linear_cross_entropy(a, w, labels, bias=bias, row_loss=True)
    assert bool(torch.isfinite(plain.lse).all()) and bool(torch.isfinite(plain.row_loss).all())
    bias[up] = INF
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, row_loss=True)
    at = labels == up
    _same_kind(r.lse, torch.full_like(r.lse, INF), "lse")
    _same_kind(r.row_loss, torch.where(at, NAN, INF), "row_loss")
    db = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, need=(False, False, True))[2]
    want = -torch.bincount(labels, minlength=n).float()  # (no probability beside the infinite one)
    want[up] = NAN
    assert torch.equal(torch.isnan(db), torch.isnan(want)) and torch.equal(db[torch.isfinite(want)], want[torch.isfinite(want)])
    bias[bad] = NAN
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, row_loss=True)
    assert bool(torch.isnan(r.lse).all()) and bool(torch.isnan(r.row_loss).all())
    r = layers.linear_cross_entropy(a, w, labels, bias=torch.full_like(bias, -INF), row_loss=True)
    _same_kind(r.lse, torch.full_like(r.lse, -INF), "lse")
    assert bool(torch.isnan(r.row_loss).all())


@pytest.mark.parametrize("kind", [F32, BF16], ids=str)
@pytest.mark.parametrize("size", SIZES[2:], ids=str)
def test_rows_of_infinite_logits(size, kind):
    """Products beyond fp32's range in some rows: the others keep their values."""
    rows, _, n, _ = size
    a, w, labels, bias = _inputs(size, kind, "rows")
    w[:, 0] = 0
    up, down = 7, n - 2
    w[up, 0], w[down, 0] = 30.0, -30.0
    good = layers.linear_cross_entropy(a, w, labels, bias=bias, row_loss=True)
    assert bool(torch.isfinite(good.lse).all())
    lse, each = good.lse.clone(), good.row_loss.clone()
    for i, (value, label, top, loss) in enumerate([(3e38, 5, INF, INF), (3e38, up, INF, NAN), (3e38, down, INF, INF), (-3e38, up, INF, INF), (-3e38, down, INF, NAN), (NAN, 5, NAN, NAN)]):
        for m in (3 + 8 * i, rows - 2 - 8 * i):
            a[m, 0] = value
            labels[m] = label
            lse[m], each[m] = top, loss
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, row_loss=True)
    _same_kind(r.lse, lse, "lse")
    _same_kind(r.row_loss, each, "row_loss")
    fine = torch.isfinite(lse)
    assert torch.equal(r.lse[fine], good.lse[fine]) and torch.equal(r.row_loss[fine], good.row_loss[fine])
    assert not bool(torch.isfinite(r.loss).any())
