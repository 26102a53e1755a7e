"""Results that take the place of an operand, where a call allows it, and matrices that lie between each other's rows: the same values as from
separate memory."""
import pytest
import torch

from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

KINDS = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _rand(g, rows, cols, kind):
    return torch.randn(rows, cols, device="cuda", generator=g).to(kind)


@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("size", [(1, 40), (5, 129), (700, 72), (300, 2100), (9, 9000)], ids=str)
def test_norm_and_dropout(size, kind):
    g = torch.Generator(device="cuda").manual_seed(size[0])
    x, r, dy, dh = (_rand(g, *size, kind) for _ in range(4))
    gain, drop = torch.randn(size[1], device="cuda", generator=g), layers.Dropout(0.25, 7, 1)
    want = layers.rms_norm(x, gain=gain, residual=r, dropout=drop)
    for y_in, h_in in (("x", None), ("r", None), ("x", "r"), ("r", "x"), (None, "x"), (None, "r")):
        t = {"x": x.clone(), "r": r.clone(), None: None}
        got = layers.rms_norm(t["x"], gain=gain, residual=t["r"], dropout=drop, y=t[y_in], h=t[h_in])
        assert torch.equal(got.y, want.y) and torch.equal(got.h, want.h) and torch.equal(got.rstd, want.rstd), (y_in, h_in)
    h, rstd = want.h, want.rstd
    want = layers.rms_norm_backward(dy, h, rstd, gain=gain, dh=dh, dropout=drop)
    for dx_in, dr_in in (("dy", None), ("h", None), ("dh", None), ("dy", "dh"), ("dh", "h"), (None, "dy")):
        t = {"dy": dy.clone(), "h": h.clone(), "dh": dh.clone(), None: None}
        got = layers.rms_norm_backward(t["dy"], t["h"], rstd, gain=gain, dh=t["dh"], dropout=drop, dx=t[dx_in], dr=t[dr_in])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (dx_in, dr_in)
    want = layers.dropout(x, drop, residual=r)
    for name in ("x", "r"):
        t = {"x": x.clone(), "r": r.clone()}
        assert torch.equal(layers.dropout(t["x"], drop, residual=t["r"], out=t[name]), want)


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_matrices_between_each_others_rows(kind):
    rows, n = 300, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    whole = torch.zeros(rows, 5 * n, device="cuda", dtype=kind)
    a, r, y, z, da = (whole[:, i * n: (i + 1) * n] for i in range(5))
    a.copy_(_rand(g, rows, n, kind)), r.copy_(_rand(g, rows, n, kind))
    w, drop = _rand(g, n, n, kind), layers.Dropout(0.25, 7, 1)
    want = layers.linear(a.clone(), w, act="silu", residual=r.clone(), dropout=drop, save=True)
    layers.linear(a, w, act="silu", residual=r, dropout=drop, out=y, preact=z)
    assert torch.equal(y, want[0]) and torch.equal(z, want[1])
    grads = layers.linear_backward(r.clone(), a.clone(), w, preact=z.clone(), act="silu", dropout=drop)
    assert all(torch.equal(p, q) for p, q in zip(layers.linear_backward(r, a, w, preact=z, act="silu", dropout=drop, da=da), grads))
    norm = layers.rms_norm(a.clone(), residual=r.clone())
    got = layers.rms_norm(a, residual=r, y=y, h=z)
    assert torch.equal(got.y, norm.y) and torch.equal(got.h, norm.h)
    # an operand that a call does not read does not count
    only = layers.linear_backward(r, a, w, need=(True, False, False))[0]
    place = a.clone()
    assert torch.equal(layers.linear_backward(r, place, w, need=(True, False, False), da=place)[0], only)
    # rows of one matrix in front of another's in the same memory
    both = torch.cat((a, torch.zeros_like(a)))
    assert torch.equal(layers.dropout(both[:rows], drop, out=both[rows:]), layers.dropout(a, drop))


def test_the_binding_says_what_lies_on_what():
    x, w = torch.zeros(8, 16, device="cuda"), torch.zeros(16, 16, device="cuda")
    for call in (lambda: layers.linear(x, w, out=x), lambda: layers.linear_backward(x, x.clone(), w, da=x), lambda: layers.dropout(x[1:], None, out=x[:-1]),
                 lambda: layers.rms_norm(x, y=x, h=x)):
        with pytest.raises(zg.ZgError, match="lies on"):
            call()
