"""Matrices whose cells lie more than 2^32 elements apart, read and written by every operator, and results large enough to go past the caches."""
import pytest
import torch

import layers_util as R
from paper_2605_29346_amd import layers, zg
from test_gpu_layers import _check_norm, _check_norm_grad

pytestmark = pytest.mark.gpu

F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
FAR = 2**32 + 16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()
    yield
    torch.cuda.empty_cache()


def test_few_rows_far_apart():
    store = torch.empty(2 * FAR + 1024, dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    cols = 40

    def far(i, fill=True):  # the ith matrix, 3 rows
        t = torch.as_strided(store, (3, cols), (FAR, 1), 8 + i * 48)
        t.copy_(torch.randn(3, cols, device="cuda", generator=g)) if fill else t.fill_(77)
        return t

    x, r, dy, dh = (far(i) for i in range(4))
    y, h, dx, dr = (far(i, False) for i in range(4, 8))
    near_x, near_r, near_dy, near_dh = (t.clone() for t in (x, r, dy, dh))
    gain, mask = torch.randn(cols, device="cuda", generator=g), (0.25, 9, 1)
    drop = layers.Dropout(*mask)
    out = layers.rms_norm(x, gain=gain, residual=r, dropout=drop, y=y, h=h)
    _check_norm(near_x, gain, near_r, mask, BF16, y, h, out.rstd)
    y8 = torch.as_strided(store.view(torch.uint8), (3, cols), (2 * FAR, 1), 2 * (8 + 8 * 48)).view(F8)
    out8 = layers.rms_norm(x, gain=gain, residual=r, dropout=drop, out_dtype=F8, y=y8)
    _check_norm(near_x, gain, near_r, mask, BF16, y8, out8.h, out8.rstd, scale=out8.scale)
    near_h = h.clone()
    _, _, dgain = layers.rms_norm_backward(dy, h, out.rstd, gain=gain, dh=dh, dropout=drop, dx=dx, dr=dr)
    _check_norm_grad(near_dy, near_h, out.rstd, gain, near_dh, mask, BF16, dx, dr, dgain)
    layers.dropout(x, drop, residual=r, out=y)
    want = R.drop(R.d64(near_x), mask) + R.d64(near_r)
    R.check(y, want, 4 * R.U[BF16] * want.abs() + 4 * R.E * R.d64(near_x).abs() + R.TINY[BF16], "dropout")
    w = (torch.randn(cols, cols, device="cuda", generator=g) * cols**-0.5).to(BF16)
    layers.linear(x, w, act="silu", residual=r, dropout=drop, out=y, preact=h)
    want = R.linear(near_x, w, None, near_r, "silu", mask, BF16)
    R.check(y, want[0], want[1], "y")
    R.check(h, want[2], want[3], "z")
    near_z = h.clone()
    _, dw, db = layers.linear_backward(dy, x, w, preact=h, act="silu", dropout=drop, da=dx)
    for got, (want, bound), what in zip((dx, dw, db), R.linear_grads(near_dy, near_x, w, near_z, "silu", mask, BF16), ("da", "dw", "dbias")):
        R.check(got, want, bound, what)
    for t, near in ((x, near_x), (r, near_r), (dy, near_dy), (dh, near_dh)):
        assert torch.equal(t, near)


@pytest.mark.parametrize("kind", [F32, BF16], ids=str)
@pytest.mark.parametrize("shift", [0, 1])
def test_large_tiles_over_wide_rows(kind, shift):
    """20000 rows 2^18 elements apart, the matrices beside each other in them: in whole chunks, and one element further on."""
    rows, k, n, pitch = 20000, 272, 264, 1 << 18
    store = torch.empty(rows, pitch, dtype=kind, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    at = [shift + 1024 * i for i in range(7)]
    a, r, dy = (store[:, at[i]: at[i] + c] for i, c in ((0, k), (1, n), (2, n)))
    y, z, da = (store[:, at[i]: at[i] + c] for i, c in ((3, n), (4, n), (5, k)))
    for t in (a, r, dy):
        t.copy_(torch.randn(t.shape, device="cuda", generator=g))
    w = (torch.randn(n, k, device="cuda", generator=g) * k**-0.5).to(kind)
    mask, live = (0.25, 9, 1), rows - 100
    drop, dev = layers.Dropout(*mask), torch.tensor([live], dtype=torch.int32, device="cuda")
    y[live:], z[live:], da[live:] = 77, 77, 77
    layers.linear(a, w, act="silu", residual=r, dropout=drop, rows=dev, out=y, preact=z)
    some = torch.cat((torch.arange(300), torch.arange(live - 3500, live - 3000), torch.arange(live - 300, live)))
    want = R.linear(a[some.cuda()], w, None, r[some.cuda()], "silu", mask, kind, ids=some.tolist())
    R.check(y[some.cuda()], want[0], want[1], "y")
    R.check(z[some.cuda()], want[2], want[3], "z")
    _, dw, db = layers.linear_backward(dy, a, w, preact=z, act="silu", dropout=drop, rows=dev, da=da)
    grads = R.linear_grads(dy, a, w, z, "silu", mask, kind, rows=live)
    for got, (want, bound), what in zip((da[:live], dw, db), grads, ("da", "dw", "dbias")):
        R.check(got, want, bound, what)
    assert all(bool((t[live:] == 77).all()) for t in (y, z, da))


@pytest.mark.parametrize("kind", [F32, BF16], ids=str)
def test_norm_gradients_past_the_caches(kind):
    """More than 32 MB of results, the device's count below the capacity: rows of the beginning, the middle and the end, and the gain's whole sum."""
    rows, cols, mask = 40000, 1000, (0.25, 9, 1)
    g = torch.Generator(device="cuda").manual_seed(3)
    dy, h, dh = (torch.randn(rows, cols, device="cuda", generator=g).to(kind) for _ in range(3))
    rstd, gain = torch.rand(rows, device="cuda", generator=g) + 0.5, 1 + 0.5 * torch.randn(cols, device="cuda", generator=g)
    live = rows - 77
    dev = torch.tensor([live], dtype=torch.int32, device="cuda")
    dx, dr = torch.full_like(dy, 77), torch.full_like(dy, 77)
    _, _, dgain = layers.rms_norm_backward(dy, h, rstd, gain=gain, dh=dh, dropout=layers.Dropout(*mask), rows=dev, dx=dx, dr=dr)
    some = torch.cat((torch.arange(200), torch.arange(rows // 2, rows // 2 + 200), torch.arange(live - 200, live)))
    at = some.cuda()
    _check_norm_grad(dy[at], h[at], rstd[at], gain, dh[at], mask, kind, dx[at], dr[at], None, ids=some.tolist())
    terms = R.d64(dy[:live]) * R.d64(h[:live]) * R.d64(rstd[:live])[:, None]
    R.check(dgain, terms.sum(0), (live + 8) * R.E * terms.abs().sum(0), "dgain")
    assert bool((dx[live:] == 77).all()) and bool((dr[live:] == 77).all())
