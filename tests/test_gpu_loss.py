"""The loss of a linear layer over many classes on the GPU against its definition in 64 bits (loss_util), at the sizes, strides, labels, masks and counts where it can go
wrong; its gradients against the formula's, against differentiation and against differences."""
import zlib

import pytest
import torch

import layers_util as R
import loss_util as L
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
KINDS = [F32, F16, BF16]
SENTINEL = 77.0


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _gen(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))  # (the same in every process)


def _matrix(g, rows, cols, kind, pad=0, shift=0, scale=1.0):
    flat = (torch.randn(rows * (cols + pad) + shift, device="cuda", generator=g) * scale).to(kind)
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def _buffer(rows, cols, kind, pad=0):
    whole = torch.full((rows + 2, cols + pad), SENTINEL, device="cuda").to(kind)
    return whole, whole[1:-1, :cols]


def _untouched(whole, rows, cols, what):
    ok = torch.full_like(whole[:1, :1].float(), SENTINEL).to(whole.dtype)
    for part in (whole[:1], whole[1 + rows:], whole[:, cols:]):
        assert bool((part == ok).all()), f"{what}: something was written outside"


def _inputs(g, rows, k, n, kind, pad=0, shift=0, missing=0.2, wide=True):
    a, w = _matrix(g, rows, k, kind, pad, shift, 2.0), _matrix(g, n, k, kind, pad, shift, k**-0.5)
    labels = torch.randint(0, n, (rows,), device="cuda", generator=g)
    none = torch.rand(rows, device="cuda", generator=g) < missing
    labels = torch.where(none, torch.where(torch.arange(rows, device="cuda") % 2 == 0, -1, n + 3), labels)
    return a, w, labels if wide else labels.int(), torch.randn(n, device="cuda", generator=g), torch.rand(rows, device="cuda", generator=g) + 0.5


def _check_loss(r, want, live, what=""):
    for name in ("lse", "row_loss"):
        if getattr(r, name) is not None:
            R.check(getattr(r, name)[:live], *want[name], f"{name} {what}")
    for name in ("total", "loss"):
        R.check(getattr(r, name), *want[name], f"{name} {what}")


SIZES = [  # rows, in, classes, pad, shift
    (1, 1, 1, 0, 0), (1, 1, 2, 0, 0), (1, 256, 512, 0, 0), (1, 1024, 5003, 0, 0), (2, 7, 5, 1, 1), (3, 301, 47, 2, 0), (16, 128, 33, 0, 0), (17, 64, 64, 0, 0), (31, 40, 8, 0, 0),
    (65, 1000, 129, 8, 0), (64, 128, 128, 0, 0), (127, 96, 255, 8, 8), (257, 200, 257, 0, 0), (300, 602, 41, 0, 1), (611, 256, 16, 0, 0), (515, 33, 1000, 3, 1), (700, 512, 3001, 0, 0),
    (2500, 256, 4099, 0, 0), (4097, 264, 2100, 0, 0), (5, 32768, 9, 0, 0)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_loss(size, kind):
    rows, k, n, pad, shift = size
    g = _gen(size, str(kind))
    a, w, labels, bias, weight = _inputs(g, rows, k, n, kind, pad, shift)
    for i, (b, v) in enumerate([(None, None), (bias, weight)]):
        whole, lse = _buffer(1, rows, F32)
        r = layers.linear_cross_entropy(a, w, labels if i else labels.int(), bias=b, weight=v, row_loss=True, lse=lse.reshape(-1))
        _check_loss(r, L.loss(a, w, labels, b, v), rows, str(i))
        _untouched(whole, 1, rows, "lse")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradients(size, kind):
    rows, k, n, pad, shift = size
    g = _gen(size, str(kind), "gradients")
    a, w, labels, bias, weight = _inputs(g, rows, k, n, kind, pad, shift)
    for i, (b, v) in enumerate([(None, None), (bias, weight)]):
        r = layers.linear_cross_entropy(a, w, labels, bias=b, weight=v)
        whole_a, da = _buffer(rows, k, kind, pad)
        whole_w, dw = _buffer(n, k, kind, pad)
        dloss = torch.tensor([-3.0], device="cuda") if i else None
        got = layers.linear_cross_entropy_backward(a, w, labels if i else labels.int(), r.lse, bias=b, weight=v, total=r.total if i == 0 else None, dloss=dloss, da=da, dw=dw)
        want = L.gradients(a, w, labels, kind, b, v, dloss=-3.0 if i else 1.0, mean=i == 0)
        for x, (y, bound), what in zip(got, want, ("da", "dw", "dbias")):
            R.check(x, y, bound, f"{what} {i}")
        _untouched(whole_a, rows, k, "da")
        _untouched(whole_w, n, k, "dw")
