"""Every kernel of the products at sizes that the library's rules send to it (layers_routes), against the definitions in 64 bits: results of every
type, activation, dropout, residual and the stored input together, a device's count below the capacity."""
import pytest
import torch

import layers_routes as S
import layers_util as R
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

KIND = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}
SENTINEL = 77.0


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _matrix(g, rows, cols, kind, pad=0, scale=1.0):
    return (torch.randn(rows, cols + pad, device="cuda", generator=g) * scale).to(kind)[:, :cols]


def _watched(rows, cols, kind):
    """An output among sentinels, a row before and behind it."""
    whole = torch.full((rows + 2, cols), SENTINEL, device="cuda").to(kind)
    return whole, whole[1:-1]


def _untouched(whole, live):
    ok = torch.full((1,), SENTINEL, device="cuda").to(whole.dtype)
    assert bool((whole[:1] == ok).all()) and bool((whole[1 + live:] == ok).all())


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", S.FORWARD, ids=str)
def test_forward(case, out):
    T, rows, k, n, pad, epilogue, _ = case
    g, kind = torch.Generator(device="cuda").manual_seed(rows + n), KIND[out]
    a = _matrix(g, rows, k, KIND[T], pad, 60.0 if T == "f8" else 1.0)
    w = _matrix(g, n, k, KIND[T], pad, 60.0 if T == "f8" else k**-0.5)
    scales = {"scale_a": torch.rand(rows, device="cuda", generator=g) * 0.01 + 1e-4, "scale_w": torch.rand(n, device="cuda", generator=g) * 0.01 + 1e-4} if T == "f8" else {}
    live = rows - rows // 11
    dev = torch.tensor([live], dtype=torch.int32, device="cuda")
    some = torch.cat((torch.arange(min(300, live)), torch.arange(max(live - 300, 0), live))).unique()
    at = some.cuda()
    rowed = {"scale_a": scales["scale_a"][at], "scale_w": scales["scale_w"]} if scales else {}
    whole_y, y = _watched(rows, n, kind)
    if epilogue == "light":
        layers.linear(a, w, rows=dev, out=y, out_dtype=kind, **scales)
        want = R.linear(a[at], w, None, None, "none", None, kind, **rowed)
    else:
        mask, bias, r = (0.3, 77, 5), torch.randn(n, device="cuda", generator=g), _matrix(g, rows, n, kind, pad)
        whole_z, z = _watched(rows, n, kind)
        layers.linear(a, w, bias=bias, act="gelu", dropout=layers.Dropout(*mask), residual=r, rows=dev, out=y, preact=z, out_dtype=kind, **scales)
        want = R.linear(a[at], w, bias, r[at], "gelu", mask, kind, ids=some.tolist(), **rowed)
        R.check(z[at], want[2], want[3], "z")
        _untouched(whole_z, live)
    R.check(y[at], want[0], want[1], "y")
    _untouched(whole_y, live)


@pytest.mark.parametrize("case", S.BACKWARD, ids=str)
def test_backward(case):
    T, O, rows, k, n, pad, *_ = case
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    a, w = _matrix(g, rows, k, KIND[T], pad), _matrix(g, n, k, KIND[T], pad, k**-0.5)
    dy, z = _matrix(g, rows, n, KIND[O], pad), _matrix(g, rows, n, KIND[O], pad)
    for act, mask, live in (("silu", None, rows), ("gelu", (0.25, 9, 9), rows - rows // 11)):
        dev = torch.tensor([live], dtype=torch.int32, device="cuda")
        whole_a, da = _watched(rows, k, KIND[T])
        whole_w, dw = _watched(n, k, KIND[T])
        db = layers.linear_backward(dy, a, w, preact=z, act=act, dropout=layers.Dropout(*mask) if mask else None, rows=dev, da=da, dw=dw)[2]
        for got, (want, bound), what in zip((da[:live], dw, db), R.linear_grads(dy, a, w, z, act, mask, KIND[T], rows=live), ("da", "dw", "dbias")):
            R.check(got, want, bound, f"{what} {act}")
        _untouched(whole_a, live)
        _untouched(whole_w, n)
