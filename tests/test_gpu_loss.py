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


ROUTES = [  # sizes that the library's rules send to the kernels that those above do not reach (test_step_routes)
    (100, 64, 5000, 0, 0), (70000, 264, 64, 0, 0), (99000, 64, 47, 0, 0), (30000, 133, 129, 1, 0), (8193, 133, 257, 1, 0), (700, 133, 2100, 0, 1), (3001, 301, 1303, 3, 0), (9000, 1032, 2064, 0, 0), (4500, 1032, 3080, 0, 0)]
SIZES = [  # rows, in, classes, pad, shift
    (1, 1, 1, 0, 0), (1, 1, 2, 0, 0), (1, 256, 512, 0, 0), (1, 1024, 5003, 0, 0), (2, 7, 5, 1, 1), (3, 301, 47, 2, 0), (16, 128, 33, 0, 0), (17, 64, 64, 0, 0), (31, 40, 8, 0, 0),
    (65, 1000, 129, 8, 0), (64, 128, 128, 0, 0), (127, 96, 255, 8, 8), (257, 200, 257, 0, 0), (300, 602, 41, 0, 1), (611, 256, 16, 0, 0), (515, 33, 1000, 3, 1), (700, 512, 3001, 0, 0),
    (2500, 256, 4099, 0, 0), (4097, 264, 2100, 0, 0), (5, 32768, 9, 0, 0), (2, 64, 4001, 0, 0), (4, 520, 331, 8, 0), (20000, 96, 47, 0, 0), (9001, 264, 64, 0, 0)]


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


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", ROUTES, ids=str)
def test_other_kernels(size, kind):
    rows, k, n, pad, shift = size
    g = _gen(size, str(kind), "routes")
    a, w, labels, bias, weight = _inputs(g, rows, k, n, kind, pad, shift)
    weight = weight if pad else None
    live = rows - rows // 11
    dev = torch.tensor([live], dtype=torch.int32, device="cuda")
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight, rows=dev, row_loss=True)
    _check_loss(r, L.loss(a, w, labels, bias, weight, live), live)
    whole_a, da = _buffer(rows, k, kind)
    whole_w, dw = _buffer(n, k, kind)
    db = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total, rows=dev, da=da, dw=dw)[2]
    for x, (y, bound), what in zip((da[:live], dw, db), L.gradients(a, w, labels, kind, bias, weight, live), ("da", "dw", "dbias")):
        R.check(x, y, bound, what)
    _untouched(whole_a, live, k, "da")
    _untouched(whole_w, n, k, "dw")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(300, 64, 70, 260), (1, 128, 900, 1), (5000, 264, 64, 4567), (2100, 520, 2056, 2001), (700, 33, 47, 300)], ids=str)
def test_rows_beyond_the_devices_count_are_left_alone(size, kind):
    rows, k, n, live = size
    g = _gen(size, str(kind), "live")
    a, w, labels, bias, weight = _inputs(g, rows, k, n, kind)
    a[live:] = float("nan")
    labels[live:] = 0
    weight[live:] = float("nan")
    for count in (live, 0, rows + 7 if live == rows else live // 2):
        dev = torch.tensor([count], dtype=torch.int32, device="cuda")
        n_live = min(count, rows)
        lse, each = torch.full((rows,), SENTINEL, device="cuda"), torch.full((rows,), SENTINEL, device="cuda")
        whole, da = _buffer(rows, k, kind)
        r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight, rows=dev, lse=lse, row_loss=each)
        assert bool((lse[n_live:] == SENTINEL).all()) and bool((each[n_live:] == SENTINEL).all())
        got = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total, rows=dev, da=da)
        _untouched(whole, n_live, k, "da")
        if n_live == 0:
            assert float(r.loss) == 0 and float(r.total) == 0 and not got[1].any() and not got[2].any()
            continue
        _check_loss(r, L.loss(a, w, labels, bias, weight, n_live), n_live)
        want = L.gradients(a, w, labels, kind, bias, weight, n_live)
        for x, (y, bound), what in zip((da[:n_live], got[1], got[2]), want, ("da", "dw", "dbias")):
            R.check(x, y, bound, what)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(40, 64, 50), (3, 64, 1000), (600, 264, 64), (2300, 128, 2056), (70, 33, 129)], ids=str)
def test_classes_that_are_masked_out(size, kind):
    """A bias of -infinity takes a class out, whole runs of them too; of the type's lowest value as well, and where all have that, they are even."""
    rows, k, n = size
    g = _gen(size, str(kind), "mask")
    a, w, labels, bias, _ = _inputs(g, rows, k, n, kind, missing=0.0)
    keep = torch.zeros(n, dtype=torch.bool, device="cuda")
    keep[torch.randint(0, n, (max(1, n // 20),), device="cuda", generator=g)] = True
    keep[n - 1] = True
    choice = keep.nonzero()[:, 0]
    labels = choice[torch.randint(0, choice.numel(), (rows,), device="cuda", generator=g)]
    for low in (-float("inf"), torch.finfo(torch.float32).min):
        masked = torch.where(keep, bias, low)
        r = layers.linear_cross_entropy(a, w, labels, bias=masked, row_loss=True)
        want = L.loss(a, w[keep], (keep.cumsum(0) - 1)[labels], masked[keep])
        _check_loss(r, want, rows, str(low))
        da, dw, db = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=masked, total=r.total)
        (wa, ba), (ww, bw), (wb, bb) = L.gradients(a, w[keep], (keep.cumsum(0) - 1)[labels], kind, masked[keep])
        R.check(da, wa, ba, "da")
        R.check(dw[keep], ww, bw, "dw")
        R.check(db[keep], wb, bb, "dbias")
        assert not dw[~keep].any() and not db[~keep].any()
    # everything at the lowest value: there is no room for log n beside it, in 32 bits or 64, and nothing overflows
    lowest = torch.full((n,), torch.finfo(torch.float32).min, device="cuda")
    r = layers.linear_cross_entropy((a * 1e-3).to(kind), w, labels, bias=lowest)
    assert float(((r.lse - lowest[0]) / lowest[0]).abs().max()) <= 2.0**-23
    got = layers.linear_cross_entropy_backward((a * 1e-3).to(kind), w, labels, r.lse, bias=lowest, total=r.total)
    assert all(bool(torch.isfinite(x).all()) for x in got)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [40, 700])
def test_what_is_not_finite_stays_in_its_row(n, kind):
    rows, k = 200, 64
    g = _gen(n, str(kind), "nan")
    a, w, labels, bias, weight = _inputs(g, rows, k, n, kind, missing=0.0)
    a[3], a[50, 7], a[120, 1] = float("nan"), float("inf"), -float("inf")
    labels[3] = -1
    weight[50] = 0
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[[3, 50, 120]] = False
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight, row_loss=True)
    want = L.loss(a[good], w, labels[good], bias, weight[good])
    R.check(r.lse[good], *want["lse"], "lse")
    R.check(r.row_loss[good], *want["row_loss"], "row_loss")
    assert bool(torch.isnan(r.lse[3])) and float(r.row_loss[3]) == 0  # (no label: no loss, whatever the logits are)
    assert not bool(torch.isfinite(r.loss))  # row 120 counts
    da, _, db = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=None)
    assert not da[3].any() and not da[50].any() and bool(torch.isnan(da[120]).any())
    (wa, ba), _, _ = L.gradients(a[good], w, labels[good], kind, bias, weight[good], mean=False)
    R.check(da[good], wa, ba, "da")
    labels[120] = -1
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight)
    R.check(r.loss, *want["loss"], "loss")
    db = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=None, need=(False, False, True))[2]
    R.check(db, *L.gradients(a[good], w, labels[good], kind, bias, weight[good], mean=False)[2], "dbias")


@pytest.mark.parametrize("kind", KINDS)
def test_a_row_without_any_class_is_not_a_number(kind):
    g = _gen(str(kind), "none")
    a, w, labels, _, _ = _inputs(g, 9, 32, 70, kind, missing=0.0)
    r = layers.linear_cross_entropy(a, w, labels, bias=torch.full((70,), -float("inf"), device="cuda"), row_loss=True)
    assert bool((r.lse == -float("inf")).all()) and bool(torch.isnan(r.row_loss).all()) and bool(torch.isnan(r.loss).all())


def test_large_logits_and_weights_of_every_size():
    g = _gen("large")
    for kind, scale, size in ((F32, 300.0, 1e-30), (BF16, 300.0, 1e30), (F16, 300.0, 1e-6), (F16, 300.0, 3e4)):
        a, w, labels, bias, weight = _inputs(g, 333, 96, 500, kind, missing=0.1)
        a = (a * scale / 10).to(kind)
        weight = weight * size * (10.0 ** torch.randint(-3, 3, (333,), device="cuda", generator=g))
        r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight, row_loss=True)
        _check_loss(r, L.loss(a, w, labels, bias, weight), 333)
        got = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total)
        for x, (y, bound), what in zip(got, L.gradients(a, w, labels, kind, bias, weight), ("da", "dw", "dbias")):
            R.check(x, y, bound, f"{what} {kind} {size}")


def test_gradients_against_differentiation_and_differences():
    g = _gen("differences")
    a, w, labels, bias, weight = _inputs(g, 60, 24, 37, F32, missing=0.2)
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight)
    got = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total)
    A, W, B = (t.double().cpu().requires_grad_() for t in (a, w, bias))
    has = ((labels >= 0) & (labels < 37)).cpu()
    each = torch.nn.functional.cross_entropy(A @ W.t() + B, torch.where(has, labels.cpu(), 0), reduction="none")
    counts = torch.where(has, weight.double().cpu(), 0.0)
    ((counts * each).sum() / counts.sum()).backward()
    want = L.gradients(a, w, labels, F32, bias, weight)
    for x, p, (_, bound), what in zip(got, (A, W, B), want, ("da", "dw", "dbias")):
        R.check(x, p.grad, bound + 1e-15, what)
    # along a direction of W: the loss' own central difference, whose error is h^2 times a third derivative (the loss is smooth, |z| moves by less than 0.1) and the loss' rounding over 2 h
    d = torch.randn(37, 24, device="cuda", generator=g) * 24**-0.5
    h = 2.0**-6
    up, down = (layers.linear_cross_entropy(a, w + s * h * d, labels, bias=bias, weight=weight).loss for s in (1, -1))
    slope = float((got[1].double() * d.double()).sum())
    noise = 2 * float(L.loss(a, w, labels, bias, weight)["loss"][1]) / (2 * h)
    assert abs(float(up.double() - down.double()) / (2 * h) - slope) <= h * h * 4.0 + noise


def test_pieces_of_the_classes():
    """More classes than one piece of dZ holds: 2^29 bytes are 4096 classes of 65536 fp16 rows; dA is joined out of several parts, twice over."""
    rows, k, n = 65_600, 40, 25_003
    g = _gen("pieces")
    a, w, labels, bias, _ = _inputs(g, rows, k, n, BF16, missing=0.5)
    r = layers.linear_cross_entropy(a, w, labels, bias=bias)
    da, dw, db = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, total=r.total)
    # the same in fp32 by torch, piece by piece of the rows (references of 64 bits for 1.6e9 cells would take minutes on the host)
    A, W = a.double(), w.double()
    wa, ww, wb, lse = torch.zeros_like(A), torch.zeros_like(W), torch.zeros(n, dtype=torch.float64, device="cuda"), torch.empty(rows, dtype=torch.float64, device="cuda")
    has = (labels >= 0) & (labels < n)
    for i in range(0, rows, 4100):
        s = slice(i, min(rows, i + 4100))
        z = A[s] @ W.t().contiguous() + bias.double()
        lse[s] = torch.logsumexp(z, 1)
        p = torch.exp(z - lse[s, None])
        p[torch.arange(z.shape[0], device="cuda"), labels[s].clamp(0, n - 1)] -= 1
        p *= has[s, None] / has.sum()
        wa[s] = p @ W
        ww += p.t().contiguous() @ A[s]
        wb += p.sum(0)
    assert float((r.lse.double() - lse).abs().max()) < 1e-5
    for x, y, what, u in ((da, wa, "da", 2.0**-8), (dw, ww, "dw", 2.0**-8), (db, wb, "dbias", 2.0**-20)):
        # two roundings (dZ and the result) of random sign, half a step each at most: 2 u of the length, and 8 u of the largest for any cell
        assert float((x.double() - y).norm() / y.norm()) < 2 * u, what
        assert float((x.double() - y).abs().max() / y.abs().max()) < 8 * u, what


def test_one_call_gives_the_same_bits_each_time_on_any_stream_and_in_a_graph():
    g = _gen("bits")
    rows, k, n = 3000, 128, 1003
    a, w, labels, bias, weight = _inputs(g, rows, k, n, BF16)
    live = torch.tensor([rows], dtype=torch.int32, device="cuda")

    def both(stream=None):
        r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight, rows=live, stream=stream)
        return (r.loss, r.total, r.lse, *layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total, rows=live, stream=stream))

    want = [t.clone() for t in both()]
    for got in (both(), both(torch.cuda.Stream())):
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    other = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first = both()
    with torch.cuda.graph(other):
        second = both()
    for count in (rows, 1500, rows, 0, rows):
        live.fill_(count)
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        eager = both()
        torch.cuda.synchronize()
        for x, y, z in zip(first, second, eager):
            if x.dim() and x.shape[0] == rows:
                x, y, z = x[:count], y[:count], z[:count]
            assert torch.equal(x, z) and torch.equal(y, z)


def test_cells_more_than_2_to_the_32_elements_apart():
    """Rows 2^22 elements apart, 1100 of them: the last ones' offsets pass 2^32."""
    g = _gen("far")
    rows, k, n, ld = 1100, 64, 1100, 1 << 22
    store = torch.empty(rows * ld, dtype=BF16, device="cuda")
    far = store.view(rows, ld)
    a, w = far[:, :k], far[:, 1024:1024 + k]
    a.copy_(torch.randn(rows, k, device="cuda", generator=g))
    w.copy_(torch.randn(n, k, device="cuda", generator=g) * k**-0.5)
    da, dw = far[:, 2048:2048 + k], far[:, 4096:4096 + k]
    labels = torch.randint(0, n, (rows,), device="cuda", generator=g)
    r = layers.linear_cross_entropy(a, w, labels, row_loss=True)
    near = (a.contiguous(), w.contiguous())
    _check_loss(r, L.loss(*near, labels), rows)
    layers.linear_cross_entropy_backward(a, w, labels, r.lse, total=r.total, da=da, dw=dw, need=(True, True, False))
    want = L.gradients(*near, labels, BF16)
    R.check(da, *want[0], "da")
    R.check(dw, *want[1], "dw")


def test_needs_are_served_one_by_one_and_nothing_else_is_written():
    g = _gen("needs")
    a, w, labels, bias, weight = _inputs(g, 300, 64, 130, BF16)
    r = layers.linear_cross_entropy(a, w, labels, bias=bias)
    whole = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, total=r.total)
    for i in range(3):
        need = tuple(j == i for j in range(3))
        got = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, total=r.total, need=need)
        assert all((x is None) != wanted for x, wanted in zip(got, need)) and torch.equal(got[i], whole[i])
    assert layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, total=r.total, need=(False, False, False)) == (None, None, None)


def test_no_rows():
    w = torch.randn(40, 16, device="cuda")
    r = layers.linear_cross_entropy(torch.empty(0, 16, device="cuda"), w, torch.empty(0, dtype=torch.int64, device="cuda"), row_loss=True)
    assert float(r.loss) == 0 and float(r.total) == 0 and r.lse.numel() == 0
    da, dw, db = layers.linear_cross_entropy_backward(torch.empty(0, 16, device="cuda"), w, torch.empty(0, dtype=torch.int64, device="cuda"), r.lse, total=r.total)
    assert da.shape == (0, 16) and not dw.any() and not db.any()


@pytest.mark.parametrize("kind", KINDS)
def test_rows_beyond_the_count_of_operands_that_lie_anyhow(kind):
    """At a size where such operands are copied first: what lies behind the count, in A and in the workspace, is nobody's operand."""
    rows, k, n, live = 3001, 301, 1303, 2777
    g = _gen("anyhow", str(kind))
    a, w, labels, bias, weight = _inputs(g, rows, k, n, kind, 3)
    a[live:] = float("nan")
    weight[live:] = float("nan")
    dev = torch.tensor([live], dtype=torch.int32, device="cuda")
    full = torch.full((1 << 24,), float("nan"), device="cuda")  # (torch's next allocations of this size are likely to have these values)
    del full
    r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight, rows=dev, row_loss=True)
    _check_loss(r, L.loss(a, w, labels, bias, weight, live), live)
    got = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total, rows=dev)
    for x, (y, bound), what in zip((got[0][:live], got[1], got[2]), L.gradients(a, w, labels, kind, bias, weight, live), ("da", "dw", "dbias")):
        R.check(x, y, bound, what)


@pytest.mark.parametrize("rows", [1, 3, 200])
@pytest.mark.parametrize("kind", KINDS)
def test_probabilities_stay_probabilities(rows, kind):
    """Logits of millions, off by ones: the loss and its gradients need not add them up in one order, and exp(Z - lse) could be any power of e.  It is held to one: no gradient is infinite, none of a
    bias larger than the rows' number.  lse itself may be given, too, with the rounding of another kernel."""
    g = _gen("probabilities", rows)
    a, w = (torch.randn(m, 1024, device="cuda", generator=g).mul(300).to(kind) for m in (rows, 900))
    labels = torch.randint(0, 900, (rows,), device="cuda", generator=g)
    lse = layers.linear_cross_entropy(a, w, labels).lse
    for off in (0.0, 5.0):
        da, dw, db = layers.linear_cross_entropy_backward(a, w, labels, lse - off)
        assert bool(torch.isfinite(da).all()) and bool(torch.isfinite(dw).all())
        assert float(db.abs().max()) <= rows
    small = layers.linear_cross_entropy(a * 2.0**-10, w, labels).lse  # (of thousands)
    assert float(layers.linear_cross_entropy_backward(a * 2.0**-10, w, labels, small - 5.0)[2].abs().max()) <= rows
