"""The dense operators on the GPU against their definitions in 64 bits (layers_util), at the sizes, strides, masks and counts where they
can go wrong; gradients against the formula's and against differences."""
import math
import zlib

import pytest
import torch

import layers_util as R
from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, F16, BF16, F8 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
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
    """Random rows inside wider ones, starting `shift` elements into the storage."""
    flat = (torch.randn(rows * (cols + pad) + shift, device="cuda", generator=g) * scale).to(kind)
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def _buffer(rows, cols, kind, pad=0):
    """An output whose surroundings are watched: a row before and behind, `pad` columns beside."""
    whole = torch.full((rows + 2, cols + pad), SENTINEL, device="cuda").to(kind)
    return whole, whole[1:-1, :cols]


def _untouched(whole, rows, cols, what):
    ok = torch.full_like(whole[:1, :1].float(), SENTINEL).to(whole.dtype)
    for part in (whole[:1], whole[1 + rows:], whole[:, cols:]):
        assert bool((part == ok).all()), f"{what}: something was written outside"


LINEAR = [  # rows, in, out, pad, shift
    (1, 1, 1, 0, 0), (1, 256, 512, 0, 0), (1, 2048, 33, 0, 0), (2, 7, 5, 1, 1), (3, 301, 47, 2, 0), (16, 1024, 16, 0, 0), (17, 64, 64, 0, 0), (31, 40, 8, 0, 0),
    (33, 1000, 130, 8, 0), (63, 65, 127, 1, 3), (64, 128, 128, 0, 0), (65, 72, 129, 0, 0), (127, 96, 255, 8, 8), (128, 512, 256, 0, 0), (130, 8, 100, 3, 5),
    (257, 200, 257, 0, 0), (300, 602, 41, 0, 1), (515, 33, 64, 0, 0), (1025, 256, 320, 0, 0), (700, 2048, 384, 0, 0), (5, 32768, 9, 0, 0)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", LINEAR, ids=str)
def test_linear(size, kind):
    rows, k, n, pad, shift = size
    g = _gen(size, str(kind))
    a, w = _matrix(g, rows, k, kind, pad, shift), _matrix(g, n, k, kind, pad, shift, k**-0.5)
    bias, r = torch.randn(n, device="cuda", generator=g), _matrix(g, rows, n, kind, pad, shift)
    acts = ["none", "relu", "silu", "gelu"]
    for i, (act, mask, res) in enumerate([("none", None, None), (acts[n % 4], (0.3, 12345678901, 7), r), ("gelu", (0.5, 99, 1), None), ("silu", None, r)]):
        whole_y, y = _buffer(rows, n, kind, pad)
        whole_z, z = _buffer(rows, n, kind, pad)
        layers.linear(a, w, bias=None if i == 0 else bias, act=act, dropout=layers.Dropout(*mask) if mask else None, residual=res, out=y, preact=z)
        want = R.linear(a, w, None if i == 0 else bias, res, act, mask, kind)
        R.check(z, want[2], want[3], f"z {act}")
        R.check(y, want[0], want[1], f"y {act}")
        _untouched(whole_y, rows, n, "y")
        _untouched(whole_z, rows, n, "z")


@pytest.mark.parametrize("out_kind", KINDS)
@pytest.mark.parametrize("size", [(1, 64, 16), (3, 17, 5), (16, 1024, 130), (100, 333, 47), (128, 256, 128), (300, 640, 257), (1100, 128, 512)], ids=str)
def test_linear_8bit(size, out_kind):
    rows, k, n = size
    g = _gen(size, str(out_kind), "f8")
    a, w = _matrix(g, rows, k, F8, 3, 1, 60.0), _matrix(g, n, k, F8, 0, 0, 60.0)
    sa, sw = torch.rand(rows, device="cuda", generator=g) * 0.05 + 1e-3, torch.rand(n, device="cuda", generator=g) * 0.05 + 1e-3
    bias, r = torch.randn(n, device="cuda", generator=g), _matrix(g, rows, n, out_kind, 1)
    for scales in ((sa, sw), (None, None)):
        if out_kind == F16 and scales[0] is None:  # sums beyond the type's range
            continue
        y, z = layers.linear(a, w, bias=bias, act="silu", residual=r, scale_a=scales[0], scale_w=scales[1], out_dtype=out_kind, save=True)
        want = R.linear(a, w, bias, r, "silu", None, out_kind, *scales)
        R.check(z, want[2], want[3], "z")
        R.check(y, want[0], want[1], "y")


# enough rows and columns for the large tiles: of operands in whole 16-byte chunks (the two sizes of tiles; widths that end inside a step, inside a
# tile and inside a lane's eight columns) and of operands that lie anyhow
LARGE = [(20000, 264, 264, 0, 0), (33000, 72, 520, 8, 0), (17000, 1096, 1032, 0, 0), (9000, 2056, 2049, 8, 0), (33333, 301, 47, 2, 0), (20001, 130, 257, 1, 1)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_linear_in_large_tiles(size, kind):
    rows, k, n, pad, shift = size
    g = _gen(size, str(kind), "large")
    a, w = _matrix(g, rows, k, kind, pad, shift), _matrix(g, n, k, kind, pad, shift, k**-0.5)
    bias, r = torch.randn(n, device="cuda", generator=g), _matrix(g, rows, n, kind, pad, shift)
    mask = (0.3, 12345678901, 7)
    live = rows - 300
    dev = torch.tensor([live], dtype=torch.int32, device="cuda")
    whole_y, y = _buffer(rows, n, kind, pad)
    whole_z, z = _buffer(rows, n, kind, pad)
    some = torch.cat((torch.arange(0, 700), torch.arange(live - 700, live)))  # rows of the first and the last tiles, every column
    want = R.linear(a[some.cuda()], w, bias, r[some.cuda()], "silu", None, kind)
    layers.linear(a, w, bias=bias, act="silu", residual=r, rows=dev, out=y, preact=z)
    R.check(z[some.cuda()], want[2], want[3], "z")
    R.check(y[some.cuda()], want[0], want[1], "y")
    _untouched(whole_y, live, n, "y")
    _untouched(whole_z, live, n, "z")
    # with dropout, and plain: the same cells as small calls on the same rows give
    ids = torch.arange(rows, dtype=torch.int32, device="cuda")
    at = slice(live - 256, live)
    for drop, act in ((mask, "gelu"), (None, "none")):
        big = layers.linear(a, w, act=act, dropout=layers.Dropout(*drop) if drop else None)
        small = layers.linear(a[at], w, act=act, dropout=layers.Dropout(*drop, ids[at]) if drop else None)
        want = R.linear(a[at], w, None, None, act, drop, kind, ids=range(live - 256, live))
        R.check(big[at], want[0], want[1], f"large {act}")
        R.check(small, want[0], want[1], f"small {act}")


@pytest.mark.parametrize("out_kind", KINDS)
@pytest.mark.parametrize("size", [(40000, 528, 272), (9000, 4112, 2064), (33000, 80, 520)], ids=str)
def test_linear_8bit_in_large_tiles(size, out_kind):
    rows, k, n = size
    g = _gen(size, str(out_kind), "f8 large")
    a, w = _matrix(g, rows, k, F8, 0, 0, 60.0), _matrix(g, n, k, F8, 0, 0, 60.0)
    sa, sw = torch.rand(rows, device="cuda", generator=g) * 0.01 + 1e-4, torch.rand(n, device="cuda", generator=g) * 0.01 + 1e-4
    y = layers.linear(a, w, act="relu", scale_a=sa, scale_w=sw, out_dtype=out_kind)
    some = torch.cat((torch.arange(0, 300), torch.arange(rows - 300, rows)))
    want = R.linear(a[some.cuda()], w, None, None, "relu", None, out_kind, sa[some.cuda()], sw)
    R.check(y[some.cuda()], want[0], want[1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(20000, 264, 264), (9000, 1032, 2056), (30011, 130, 257)], ids=str)
def test_linear_gradients_in_large_tiles(size, kind):
    rows, k, n = size
    g = _gen(size, str(kind), "large back")
    a, w, dy, z = _matrix(g, rows, k, kind), _matrix(g, n, k, kind, 0, 0, k**-0.5), _matrix(g, rows, n, kind), _matrix(g, rows, n, kind)
    for act, mask, live in (("none", None, rows), ("relu", (0.25, 9, 9), rows - 777)):
        dev = torch.tensor([live], dtype=torch.int32, device="cuda")
        whole, da = _buffer(rows, k, kind)
        _, dw, db = layers.linear_backward(dy, a, w, preact=z, act=act, dropout=layers.Dropout(*mask) if mask else None, rows=dev, da=da)
        grads = R.linear_grads(dy, a, w, z, act, mask, kind, rows=live)
        for got, (want, bound), what in zip((da[:live], dw, db), grads, ("da", "dw", "dbias")):
            R.check(got, want, bound, f"{what} {act}")
        _untouched(whole, live, k, "da")


@pytest.mark.parametrize("out_kind", KINDS)
@pytest.mark.parametrize("kind", KINDS)
def test_linear_result_in_another_type(kind, out_kind):
    g = _gen(str(kind), str(out_kind))
    a, w, bias = _matrix(g, 150, 90, kind), _matrix(g, 70, 90, kind, 0, 0, 0.1), torch.randn(70, device="cuda", generator=g)
    r = _matrix(g, 150, 70, out_kind)
    y, z = layers.linear(a, w, bias=bias, act="relu", residual=r, out_dtype=out_kind, save=True)
    want = R.linear(a, w, bias, r, "relu", None, out_kind)
    R.check(y, want[0], want[1])
    R.check(z, want[2], want[3])
    dy = _matrix(g, 150, 70, out_kind)
    for got, (want, bound) in zip(layers.linear_backward(dy, a, w, preact=z, act="gelu"), R.linear_grads(dy, a, w, z, "gelu", None, kind)):
        R.check(got, want, bound)


COUNTS = [0, 1, 5, 64, 129, 300, 100000]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("count", COUNTS)
def test_the_count_on_the_device_bounds_every_operator(count, kind):
    """Rows beyond the count hold NaN in every input: nothing of them arrives anywhere, and no output row of theirs is written."""
    rows, k, n = 300, 72, 40
    live = min(count, rows)
    g = _gen(count, str(kind))
    dev = torch.tensor([count], dtype=torch.int32, device="cuda")

    def poisoned(c):
        t = _matrix(g, rows, c, kind, 1)
        t[live:] = float("nan")
        return t

    a, w, bias, r, dy, z = poisoned(k), _matrix(g, n, k, kind, 0, 0, 0.1), torch.randn(n, device="cuda", generator=g), poisoned(n), poisoned(n), poisoned(n)
    mask = (0.25, 42, 3)
    drop = layers.Dropout(*mask)
    whole, y = _buffer(rows, n, kind, 2)
    layers.linear(a, w, bias=bias, act="silu", dropout=drop, residual=r, rows=dev, out=y)
    want = R.linear(a[:live], w, bias, r[:live], "silu", mask, kind)
    R.check(y[:live], want[0], want[1], "linear")
    _untouched(whole, live, n, "linear")

    whole, da = _buffer(rows, k, kind, 2)
    _, dw, db = layers.linear_backward(dy, a, w, preact=z, act="gelu", dropout=drop, rows=dev, da=da)
    grads = R.linear_grads(dy, a, w, z, "gelu", mask, kind, rows=live)
    for got, (want, bound), what in zip((da[:live], dw, db), grads, ("da", "dw", "dbias")):
        R.check(got, want, bound, what)
    _untouched(whole, live, k, "da")

    whole, out = _buffer(rows, n, kind, 2)
    layers.dropout(dy, drop, residual=r, rows=dev, out=out)
    want = R.drop(R.d64(dy[:live]), mask) + R.d64(r[:live])
    R.check(out[:live], want, 4 * R.U[kind] * want.abs() + 4 * R.E * R.d64(dy[:live]).abs() + R.TINY[kind], "dropout")
    _untouched(whole, live, n, "dropout")

    gain = torch.randn(n, device="cuda", generator=g)
    whole_y, y = _buffer(rows, n, kind, 2)
    whole_h, h = _buffer(rows, n, kind, 2)
    rstd = torch.full((rows,), SENTINEL, device="cuda")
    layers.rms_norm(dy, gain=gain, residual=r, dropout=drop, rows=dev, y=y, h=h, rstd=rstd)
    _check_norm(dy[:live], gain, r[:live], mask, kind, y[:live], h[:live], rstd[:live])
    _untouched(whole_y, live, n, "y")
    _untouched(whole_h, live, n, "h")
    assert bool((rstd[live:] == SENTINEL).all())

    whole_x, dx = _buffer(rows, n, kind, 2)
    whole_r, dr = _buffer(rows, n, kind, 2)
    rstd[live:] = float("nan")
    dgain = layers.rms_norm_backward(dy, r, rstd, gain=gain, dh=z, dropout=drop, rows=dev, dx=dx, dr=dr)[2]
    _check_norm_grad(dy[:live], r[:live], rstd[:live], gain, z[:live], mask, kind, dx[:live], dr[:live], dgain)
    _untouched(whole_x, live, n, "dx")
    _untouched(whole_r, live, n, "dr")


BACK = [(1, 1, 1, 0, 0), (1, 256, 64, 0, 0), (2, 33, 7, 1, 1), (17, 64, 130, 0, 0), (64, 64, 64, 8, 0), (100, 200, 47, 0, 1), (129, 257, 65, 3, 2),
        (300, 128, 384, 0, 0), (1000, 100, 100, 0, 0), (4099, 72, 40, 0, 0), (2048, 512, 256, 0, 0), (70, 1030, 1029, 0, 0)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", BACK, ids=str)
def test_linear_gradients(size, kind):
    rows, k, n, pad, shift = size
    g = _gen(size, str(kind), "back")
    a, w = _matrix(g, rows, k, kind, pad, shift), _matrix(g, n, k, kind, pad, shift, k**-0.5)
    dy, z = _matrix(g, rows, n, kind, pad, shift), _matrix(g, rows, n, kind, pad, shift)
    for act, mask in (("none", None), ("relu", None), (["silu", "gelu"][n % 2], (0.4, 5 << 40, 2)), ("none", (0.1, 3, 0))):
        whole_a, da = _buffer(rows, k, kind, pad)
        whole_w, dw = _buffer(n, k, kind, pad)
        db = layers.linear_backward(dy, a, w, preact=z, act=act, dropout=layers.Dropout(*mask) if mask else None, da=da, dw=dw)[2]
        for got, (want, bound), what in zip((da, dw, db), R.linear_grads(dy, a, w, z, act, mask, kind), ("da", "dw", "dbias")):
            R.check(got, want, bound, f"{what} {act}")
        _untouched(whole_a, rows, k, "da")
        _untouched(whole_w, n, k, "dw")


def test_only_the_gradients_that_are_asked_for():
    g = _gen("need")
    a, w, dy, z = _matrix(g, 90, 24, BF16), _matrix(g, 40, 24, BF16), _matrix(g, 90, 40, BF16), _matrix(g, 90, 40, BF16)
    every = layers.linear_backward(dy, a, w, preact=z, act="silu")
    for need in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        some = layers.linear_backward(dy, a, w, preact=z, act="silu", need=need)
        for asked, x, y in zip(need, some, every):
            assert torch.equal(x, y) if asked else x is None
    x, _, none = layers.rms_norm_backward(dy, z, torch.ones(90, device="cuda"), need_dgain=False)
    assert none is None and torch.equal(x, layers.rms_norm_backward(dy, z, torch.ones(90, device="cuda"))[0])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 0, 1), (70, 601, 1, 0), (129, 512, 0, 0), (40, 2500, 3, 2), (5, 32768, 0, 0)], ids=str)
@pytest.mark.parametrize("p", [0.0, 2.0**-20, 0.1, 0.5, 0.99, 1.0])
def test_dropout(size, kind, p):
    rows, cols, pad, shift = size
    g = _gen(size, str(kind), p)
    x, r = _matrix(g, rows, cols, kind, pad, shift), _matrix(g, rows, cols, kind, pad, shift)
    ids = torch.randint(-2**31, 2**31 - 1, (rows,), device="cuda", generator=g, dtype=torch.int32)
    for with_ids, res in ((None, None), (ids, r)):
        whole, y = _buffer(rows, cols, kind, pad)
        layers.dropout(x, layers.Dropout(p, -5, 2**32 - 1, with_ids), residual=res, out=y)
        want = R.drop(R.d64(x), (p, 2**64 - 5, 2**32 - 1), None if with_ids is None else with_ids.cpu().numpy())
        err = 2 * R.E * want.abs()
        want = want if res is None else want + R.d64(res)
        R.check(y, want, (err + R.E * want.abs()) * 1.01 + R.U[kind] * want.abs() + R.TINY[kind])
        _untouched(whole, rows, cols, "y")
    same = x.clone()
    layers.dropout(same, layers.Dropout(p, -5, 2**32 - 1), out=same)  # in place
    assert torch.equal(same, layers.dropout(x, layers.Dropout(p, -5, 2**32 - 1)))


def test_dropped_cells_are_zero_whatever_they_are():
    rows, cols, mask = 50, 203, (0.5, 31337, 4)
    keep = R.kept(*mask, range(rows), cols).cuda()
    x = torch.randn(rows, cols, device="cuda")
    for bad in (float("nan"), float("inf"), -float("inf"), -3.4e38):
        y = layers.dropout(torch.where(keep, x, bad), layers.Dropout(*mask))
        assert torch.equal(y, torch.where(keep, 2 * x, 0.0))
        h = layers.rms_norm(torch.where(keep, x, bad), dropout=layers.Dropout(*mask)).h
        assert torch.equal(h, torch.where(keep, 2 * x, 0.0))
        # behind a product: a bias makes the dropped cells whatever they are
        w, z = torch.zeros(cols, 8, device="cuda"), torch.zeros(rows, 8, device="cuda")
        y = layers.linear(z, w, bias=torch.full((cols,), bad, device="cuda"), dropout=layers.Dropout(*mask))
        assert bool((y[~keep] == 0).all()) and not bool((y[keep] == 0).any())


def _check_norm(x, gain, r, mask, kind, y, h, rstd, eps=1e-6, ids=None, scale=None):
    cols = x.shape[1]
    want_h = R.drop(R.d64(x), mask, ids)
    err = 2 * R.E * want_h.abs() if mask else torch.zeros_like(want_h)
    if r is not None:
        want_h = want_h + R.d64(r)
        err = err + R.E * want_h.abs()
    if h is not None:
        R.check(h, want_h, err * 1.01 + R.U[kind] * want_h.abs() + R.TINY[kind], "h")
    ms = want_h.pow(2).mean(1)
    want_rstd = (ms + eps).rsqrt()
    # the mean square is off by (cols + 4) units and by what its terms are; the square root halves that
    ms_err = (cols + 4) * R.E * ms + 2 * (err * want_h.abs()).mean(1)
    rstd_err = want_rstd * (0.5 * ms_err / (ms + eps) + 4 * R.E)
    R.check(rstd, want_rstd, rstd_err, "rstd")
    g = R.d64(gain) if gain is not None else torch.ones(cols, dtype=torch.float64)
    want = want_h * want_rstd[:, None] * g
    y_err = (err * want_rstd[:, None] + want_h.abs() * rstd_err[:, None]) * g.abs() + 3 * R.E * want.abs()
    if scale is None:
        R.check(y, want, y_err * 1.01 + R.U[kind] * want.abs() + R.TINY[kind], "y")
        return
    top = want.abs().amax(1) / 448 if x.shape[0] else torch.zeros(0, dtype=torch.float64)
    want_scale = torch.where(top > 0, top, torch.ones_like(top))
    R.check(scale, want_scale, y_err.amax(1) / 448 + 4 * R.E * want_scale, "scale")
    # four significant bits, steps of 2^-9 at the bottom
    rounded = R.d64(scale)[:, None] * R.d64(y.float())
    R.check(rounded, want, y_err + (2.0**-4 * 1.001) * want.abs() + 2.0**-10 * 1.001 * want_scale[:, None], "y (8 bits)")


NORM = [(1, 1, 0, 0), (1, 1024, 0, 0), (2, 7, 1, 1), (9, 64, 0, 0), (33, 65, 3, 1), (5, 128, 0, 0), (17, 129, 0, 0), (30, 256, 8, 0), (7, 300, 1, 0), (11, 512, 0, 0),
        (10, 601, 1, 3), (130, 1024, 0, 0), (6, 1030, 0, 1), (3, 2048, 0, 0), (4, 2049, 0, 0), (2, 4097, 1, 0), (3, 8192, 0, 0), (2, 8199, 0, 0), (2, 16384, 0, 0),
        (1025, 40, 0, 0), (5000, 96, 0, 0)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", NORM, ids=str)
def test_norm(size, kind):
    rows, cols, pad, shift = size
    g = _gen(size, str(kind), "norm")
    x, r = _matrix(g, rows, cols, kind, pad, shift), _matrix(g, rows, cols, kind, pad, shift, 3.0)
    gain = 1 + 0.5 * torch.randn(cols, device="cuda", generator=g)
    ids = torch.randint(0, 2**31 - 1, (rows,), device="cuda", generator=g, dtype=torch.int32)
    for res, gn, mask, with_ids in ((None, None, None, None), (r, gain, None, None), (r, gain, (0.2, 8, 1), ids), (None, gain, (0.5, 1 << 50, 0), None)):
        drop = layers.Dropout(*mask, with_ids) if mask else None
        whole, y = _buffer(rows, cols, kind, pad)
        out = layers.rms_norm(x, gain=gn, residual=res, dropout=drop, y=y)
        host_ids = None if with_ids is None else with_ids.cpu().numpy()
        _check_norm(x, gn, res, mask, kind, out.y, out.h, out.rstd, ids=host_ids)
        _untouched(whole, rows, cols, "y")
        out = layers.rms_norm(x, gain=gn, residual=res, dropout=drop, out_dtype=F8)
        _check_norm(x, gn, res, mask, kind, out.y, out.h, out.rstd, ids=host_ids, scale=out.scale)


def test_norm_in_other_types_and_in_place():
    g = _gen("types")
    x, r = _matrix(g, 60, 200, F32), _matrix(g, 60, 200, F32)
    for kind in (F16, BF16):
        out = layers.rms_norm(x, residual=r, out_dtype=kind)
        want = R.d64(x) + R.d64(r)
        want = want * (want.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt()
        R.check(out.y, want, (220 * R.E + R.U[kind]) * 1.01 * want.abs() + 4 * R.E + R.TINY[kind])
    ref = layers.rms_norm(x, residual=r)
    stream = r.clone()
    out = layers.rms_norm(x, residual=stream, h=stream)  # the residual stream is updated where it lies
    assert torch.equal(stream, ref.h) and torch.equal(out.y, ref.y)


def test_norm_of_special_rows():
    x = torch.randn(6, 100, device="cuda")
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, 5] = float("inf")
    x[3] = 1e-30
    x[4] = 1e18
    out = layers.rms_norm(x, eps=1e-6)
    assert bool((out.y[0] == 0).all()) and abs(float(out.rstd[0]) - 1000) < 1e-3
    assert bool(torch.isnan(out.y[1]).all()) and bool(torch.isnan(out.y[2, 5])) and bool((out.y[2, :5] == 0).all())
    assert bool((out.y[3].abs() < 2e-27).all()) and bool(torch.allclose(out.y[4], torch.ones(100, device="cuda"), rtol=1e-5))
    eight = layers.rms_norm(x, eps=1e-6, out_dtype=F8)
    assert float(eight.scale[0]) == 1 and bool((eight.y[0].float() == 0).all())
    assert float(eight.scale[1]) == 1 and bool(torch.isnan(eight.y[1].float()).all())
    assert bool((eight.y[4].float() == 448).all())
    assert bool(torch.isnan(layers.rms_norm(x[:1], eps=0.0).y).all())  # 0 / 0, as the formula says


def _check_norm_grad(dy, h, rstd, gain, dh, mask, kind, dx, dr, dgain, ids=None):
    dy, h, s = R.d64(dy), R.d64(h), R.d64(rstd)[:, None]
    cols = dy.shape[1]
    g = R.d64(gain) if gain is not None else torch.ones(cols, dtype=torch.float64)
    gy = dy * g
    dot = (gy * h).mean(1, keepdim=True)
    want = s * (gy - h * dot * s * s)
    err = s * (2 * R.E * gy.abs() + h.abs() * s * s * ((cols + 8) * R.E * (gy * h).abs().mean(1, keepdim=True))) + 6 * R.E * (s * gy.abs() + (h * dot * s**3).abs())
    if dh is not None:
        want = want + R.d64(dh)
        err = err + R.E * want.abs()
    if dr is not None:
        R.check(dr, want, err * 1.01 + R.U[kind] * want.abs() + R.TINY[kind], "dr")
    t = math.floor(mask[0] * 65536 + 0.5) if mask else 0
    grown = 65536 / (65536 - t)
    dropped = R.drop(want, mask, ids)
    R.check(dx, dropped, (err * grown + 2 * R.E * dropped.abs()) * 1.01 + R.U[kind] * dropped.abs() + R.TINY[kind], "dx")
    if dgain is not None:
        terms = dy * h * s
        R.check(dgain, terms.sum(0), (dy.shape[0] + 8) * R.E * terms.abs().sum(0), "dgain")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", NORM, ids=str)
def test_norm_gradients(size, kind):
    rows, cols, pad, shift = size
    g = _gen(size, str(kind), "norm grad")
    dy, h, dh = (_matrix(g, rows, cols, kind, pad, shift) for _ in range(3))
    rstd = torch.rand(rows, device="cuda", generator=g) + 0.5
    gain = 1 + 0.5 * torch.randn(cols, device="cuda", generator=g)
    for gn, d, mask in ((None, None, None), (gain, dh, None), (gain, dh, (0.3, 77, 9)), (gain, None, (0.5, 1, 1))):
        whole, dx = _buffer(rows, cols, kind, pad)
        _, dr, dgain = layers.rms_norm_backward(dy, h, rstd, gain=gn, dh=d, dropout=layers.Dropout(*mask) if mask else None, dx=dx)
        _check_norm_grad(dy, h, rstd, gn, d, mask, kind, dx, dr, dgain)
        _untouched(whole, rows, cols, "dx")
    ref = layers.rms_norm_backward(dy, h, rstd, gain=gain, dh=dh)
    for name, t in (("dh", dh.clone()), ("dy", dy.clone())):  # in place
        a, b = (dy, t) if name == "dh" else (t, dh)
        layers.rms_norm_backward(a, h, rstd, gain=gain, dh=b, dx=t)
        assert torch.equal(t, ref[0])


def _along(f, x, direction, c, eps):
    """Difference quotient of sum(c f(x)) along a direction, of fourth order: a step in a weight moves a cell by that many times the length
    of a whole row of a."""
    def at(t):
        return (f(x + t * eps * direction).double() * c.double()).sum()

    return float(8 * (at(1) - at(-1)) - (at(2) - at(-2))) / (12 * eps)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_gradients_against_differences(act):
    """f32, eps 2^-6: a cell moves by up to 2^-6 times the length of a row (about 7), the quotient is off by the fourth power of that / 30 times a
    fifth derivative and by rounding over eps, both far below the 1 % of the gradient's size along the direction that is asked for."""
    g = _gen("differences", act)
    rows, k, n, eps = 60, 48, 40, 2.0**-6
    a, w, bias = _matrix(g, rows, k, F32), _matrix(g, n, k, F32, 0, 0, k**-0.5), torch.randn(n, device="cuda", generator=g)
    c, drop = _matrix(g, rows, n, F32), layers.Dropout(0.25, 9, 2)
    _, z = layers.linear(a, w, bias=bias, act=act, dropout=drop, save=True)
    grads = layers.linear_backward(c, a, w, preact=z, act=act, dropout=drop)
    f = [lambda v: layers.linear(v, w, bias=bias, act=act, dropout=drop), lambda v: layers.linear(a, v, bias=bias, act=act, dropout=drop),
         lambda v: layers.linear(a, w, bias=v, act=act, dropout=drop)]
    for fn, x, grad in zip(f, (a, w, bias), grads):
        d = torch.randn(x.shape, device="cuda", generator=g)
        got = float((grad.double() * d.double()).sum())
        assert abs(got - _along(fn, x, d, c, eps)) < 0.01 * float(grad.double().norm()), act
    x, r, gain = _matrix(g, rows, n, F32), _matrix(g, rows, n, F32), torch.randn(n, device="cuda", generator=g)
    ch = _matrix(g, rows, n, F32)
    out = layers.rms_norm(x, gain=gain, residual=r, dropout=drop)
    dx, dr, dgain = layers.rms_norm_backward(c, out.h, out.rstd, gain=gain, dh=ch, dropout=drop)

    def norm(x, r, gain):
        o = layers.rms_norm(x, gain=gain, residual=r, dropout=drop)
        return torch.cat((o.y, o.h), 1)

    both = torch.cat((c, ch), 1)
    for fn, v, grad in ((lambda v: norm(v, r, gain), x, dx), (lambda v: norm(x, v, gain), r, dr), (lambda v: norm(x, r, v), gain, dgain)):
        d = torch.randn(v.shape, device="cuda", generator=g)
        assert abs(float((grad.double() * d.double()).sum()) - _along(fn, v, d, both, eps)) < 0.01 * float(grad.double().norm())


def test_special_values_pass_through_a_product():
    for kind in KINDS:
        a, w = torch.ones(70, 40, device="cuda", dtype=kind), torch.ones(50, 40, device="cuda", dtype=kind)
        a[3, 7], a[5, 39], a[6, 0] = float("inf"), float("nan"), -float("inf")
        w[:, 1:39] = 0.5
        y = layers.linear(a, w).float()
        assert bool(torch.isinf(y[3]).all()) and bool((y[3] > 0).all()) and bool(torch.isnan(y[5]).all()) and bool((y[6] == -float("inf")).all())
        others = [i for i in range(70) if i not in (3, 5, 6)]
        assert bool(torch.isfinite(y[others]).all())
        y = layers.linear(a, w, act="relu").float()
        assert bool(torch.isnan(y[5]).all()) and bool((y[6] == 0).all())


def test_offsets_beyond_32_bits():
    """Rows 2^32 elements apart."""
    far = 2**32 + 16
    store = torch.empty(2 * far + 64, dtype=BF16, device="cuda")
    a = torch.as_strided(store, (3, 40), (far, 1), 8)
    a.copy_(torch.randn(3, 40, device="cuda"))
    g = _gen("far")
    w = _matrix(g, 24, 40, BF16)
    want = R.linear(a, w, None, None, "none", None, BF16)
    R.check(layers.linear(a, w), want[0], want[1])
    dy = _matrix(g, 3, 24, BF16)
    dw = layers.linear_backward(dy, a, w)[1]
    want, bound = R.linear_grads(dy, a, w, None, "none", None, BF16)[1]
    R.check(dw, want, bound)
    y = torch.as_strided(store, (3, 40), (far, 1), 0)
    out = layers.rms_norm(a.clone(), y=torch.as_strided(store, (3, 40), (far, 1), 8))
    _check_norm(y.new_tensor(0).expand(0, 40), None, None, None, BF16, out.y[:0], None, out.rstd[:0])
    assert torch.equal(layers.dropout(out.y, layers.Dropout(0.5, 3)), layers.dropout(out.y.contiguous(), layers.Dropout(0.5, 3)))
    del store


def test_many_rows():
    """More rows than a launch's other dimensions hold, against the same rows in small calls."""
    rows, k, n = 300_001, 16, 24
    g = _gen("many")
    a, w = _matrix(g, rows, k, BF16), _matrix(g, n, k, BF16)
    y = layers.linear(a, w, act="relu")
    at = slice(rows - 1000, rows)
    assert torch.equal(y[at], layers.linear(a[at], w, act="relu"))
    assert torch.equal(layers.rms_norm(a).y[at], layers.rms_norm(a[at]).y)
    ids = torch.arange(rows, dtype=torch.int32, device="cuda")
    assert torch.equal(layers.dropout(a, layers.Dropout(0.3, 5))[at], layers.dropout(a[at], layers.Dropout(0.3, 5, 0, ids[at])))


def test_more_workgroups_than_a_grids_first_dimension_takes():
    rows, cols = 70_000_003, 8
    g = _gen("rows")
    x = torch.empty(rows, cols, device="cuda", dtype=BF16).normal_(generator=g)
    w = _matrix(g, 8, cols, BF16)
    at = slice(rows - 5000, rows)
    for part in (at, slice(0, 5000), slice(67_108_864 - 2500, 67_108_864 + 2500)):
        assert torch.equal(layers.linear(x, w, act="relu")[part], layers.linear(x[part], w, act="relu"))
        assert torch.equal(layers.rms_norm(x).y[part], layers.rms_norm(x[part]).y)
    ids = torch.arange(rows, dtype=torch.int32, device="cuda")
    assert torch.equal(layers.dropout(x, layers.Dropout(0.3, 5))[at], layers.dropout(x[at], layers.Dropout(0.3, 5, 0, ids[at])))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(5, 40, 24), (700, 301, 47), (20000, 264, 264), (9000, 2056, 520)], ids=str)
def test_a_result_in_the_residuals_place(size, kind):
    rows, k, n = size
    g = _gen(size, str(kind), "in place")
    a, w, r = _matrix(g, rows, k, kind), _matrix(g, n, k, kind, 0, 0, k**-0.5), _matrix(g, rows, n, kind, 8)
    want = layers.linear(a, w, act="silu", residual=r)
    whole = torch.full((rows, n + 8), SENTINEL, device="cuda").to(kind)
    y = whole[:, :n]
    y.copy_(r)
    layers.linear(a, w, act="silu", residual=y, out=y)
    assert torch.equal(y, want) and bool((whole[:, n:] == torch.tensor(SENTINEL, device="cuda").to(kind)).all())
    x = _matrix(g, rows, n, kind)
    want = layers.dropout(x, layers.Dropout(0.5, 1), residual=r)
    y.copy_(r)
    assert torch.equal(layers.dropout(x, layers.Dropout(0.5, 1), residual=y, out=y), want)


def test_same_bits_every_time():
    g = _gen("bits")
    a, w, dy, z = _matrix(g, 5000, 130, F32), _matrix(g, 70, 130, F32), _matrix(g, 5000, 70, F32), _matrix(g, 5000, 70, F32)
    first = layers.linear_backward(dy, a, w, preact=z, act="gelu")
    norm = layers.rms_norm_backward(dy, z, z.square().mean(1).rsqrt())
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(first, layers.linear_backward(dy, a, w, preact=z, act="gelu")))
        assert all(torch.equal(x, y) for x, y in zip(norm, layers.rms_norm_backward(dy, z, z.square().mean(1).rsqrt())) if x is not None)


def test_on_another_stream():
    g = _gen("stream")
    a, w, dy = _matrix(g, 3000, 256, BF16), _matrix(g, 128, 256, BF16), _matrix(g, 3000, 128, BF16)
    want = (layers.linear(a, w), *layers.linear_backward(dy, a, w), layers.rms_norm(dy).y)
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(), zg.new_stream()):
        for _ in range(3):
            got = (layers.linear(a, w, stream=stream), *layers.linear_backward(dy, a, w, stream=stream), layers.rms_norm(dy, stream=stream).y)
            torch.cuda.ExternalStream(stream).synchronize() if isinstance(stream, int) else stream.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_recorded_into_a_graph():
    """A small training step of all operators, captured and replayed with new inputs and a new row count, against the eager calls."""
    g = _gen("graph")
    rows, k, n = 600, 96, 64
    x, w, dy = _matrix(g, rows, k, BF16), _matrix(g, n, k, BF16, 0, 0, 0.1), _matrix(g, rows, n, BF16)
    bias, live = torch.randn(n, device="cuda", generator=g), torch.tensor([rows], dtype=torch.int32, device="cuda")
    drop = layers.Dropout(0.2, 11, 1)

    def step():
        y, z = layers.linear(x, w, bias=bias, act="silu", dropout=drop, rows=live, save=True, out=bufs[0], preact=bufs[1])
        o = layers.rms_norm(y, residual=dy, dropout=drop, rows=live, y=bufs[2], h=bufs[3], rstd=rstd)
        dx, dr, dgain = layers.rms_norm_backward(dy, o.h, o.rstd, dropout=drop, rows=live, dx=bufs[4], dr=bufs[5])
        return [y, z, o.y, dx, dr, dgain, *layers.linear_backward(dx, x, w, preact=z, act="silu", dropout=drop, rows=live, da=bufs[6])]

    bufs = [torch.zeros(rows, c, dtype=BF16, device="cuda") for c in (n, n, n, n, n, n, k)]
    rstd = torch.zeros(rows, device="cuda")
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i, count in enumerate((600, 37, 0, 599, 600)):
        x.copy_(torch.randn(rows, k, device="cuda", generator=g))
        live.fill_(count)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        want = step()
        torch.cuda.synchronize()
        for j, (p, q) in enumerate(zip(got, want)):
            assert torch.equal(p, q), (i, j)


def test_refusals_of_the_binding():
    x, w = torch.zeros(8, 16, device="cuda"), torch.zeros(4, 16, device="cuda")
    bad = [lambda: layers.linear(x, w[:, :8]), lambda: layers.linear(x, w.half()), lambda: layers.linear(x, w, act="tanh"),
           lambda: layers.linear(x, w, bias=torch.zeros(5, device="cuda")), lambda: layers.linear(x, w, bias=torch.zeros(4, device="cuda").half()),
           lambda: layers.linear(x.t(), w), lambda: layers.linear(x, w, residual=x), lambda: layers.linear(x, w, out=torch.zeros(8, 4)),
           lambda: layers.linear(x, w, rows=torch.zeros(1, device="cuda")), lambda: layers.linear(x, w, dropout=layers.Dropout(0.5, 1, 0, torch.zeros(8))),
           lambda: layers.rms_norm(x, gain=torch.ones(8, device="cuda")), lambda: layers.dropout(x.expand(8, 16)[:, ::2], None),
           lambda: layers.linear_backward(x, x, w), lambda: layers.rms_norm_backward(x, x, torch.ones(4, device="cuda"))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        layers.linear(x.double(), w.double())
    with pytest.raises(zg.ZgError):
        layers.dropout(x, layers.Dropout(1.5, 1))
    with pytest.raises(zg.ZgError):
        layers.linear(x, w, scale_a=torch.ones(8, device="cuda"))
    with pytest.raises(zg.ZgError):
        layers.linear_backward(torch.zeros(8, 4, device="cuda"), x, w, act="silu")  # the activation's input is missing
