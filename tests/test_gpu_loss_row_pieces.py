"""Gradients over so many rows that dZ is made of pieces of them: the weights' gradient is a sum over the pieces, dA is of each, counts end in any of them."""
import zlib

import pytest
import torch

from paper_2605_29346_amd import layers, zg
from test_gpu_step_workspace import Guarded

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SENTINEL = 77.0
# rows, in, classes, elements between rows, type -> pieces of the rows, pieces of the classes (test_step_row_pieces asks the library for them)
SIZES = [
    (240_007, 40, 4100, 0, BF16, 4, 2),    # dW of many parts, dA of a few
    (240_007, 37, 4100, 3, F16, 4, 2),     # rows that lie anyhow, copied piece by piece
    (120_011, 40, 5003, 0, F32, 2, 2),
    (240_007, 2312, 4100, 0, BF16, 4, 2),  # dA's parts are large; dW of one part
    (240_007, 264, 4096, 8, BF16, 4, 1),   # one piece of the classes
    (7_600_001, 16, 64, 0, F32, 4, 1),     # few classes
]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _reference(a, w, labels, bias, weight, live, mean=True):
    """lse and the gradients in 64 bits (products of a few thousand rows at a time, in 64 bits)."""
    rows, k = a.shape
    n = w.shape[0]
    W, wa, ww, wb = w.double(), torch.zeros(live, k, dtype=torch.float64, device="cuda"), torch.zeros(n, k, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    Wt = W.t().contiguous()
    lse = torch.empty(live, dtype=torch.float64, device="cuda")
    has = ((labels >= 0) & (labels < n))[:live]
    counts = torch.where(has, weight[:live].double() if weight is not None else 1.0, 0.0)
    total = counts.sum() if mean else 1.0
    step = max(512, min(1 << 16, (1 << 25) // n))
    for i in range(0, live, step):
        s = slice(i, min(live, i + step))
        z = a[s].double() @ Wt
        if bias is not None:
            z += bias.double()
        lse[s] = torch.logsumexp(z, 1)
        p = z.sub_(lse[s, None]).exp_()
        p[torch.arange(p.shape[0], device="cuda"), labels[s].clamp(0, n - 1)] -= 1
        p *= (counts[s] / total)[:, None]
        wa[s] = p @ W
        ww += p.t().contiguous() @ a[s].double()
        wb += p.sum(0)
    return lse, wa, ww, wb


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_row_pieces(size):
    rows, k, n, pad, kind, _, _ = size
    g = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(size).encode()))
    a, w = (torch.randn(m, k + pad, device="cuda", generator=g).mul_(s).to(kind)[:, :k] for m, s in ((rows, 2.0), (n, k**-0.5)))
    labels = torch.randint(0, n, (rows,), device="cuda", generator=g)
    labels[torch.rand(rows, device="cuda", generator=g) < 0.2] = -1
    bias = torch.randn(n, device="cuda", generator=g)
    weight = torch.rand(rows, device="cuda", generator=g) + 0.5 if pad else None
    # all rows; a count that ends inside a piece, at the end of one, in the first, and nowhere
    for live in (None, rows - rows // 9, 65536, 4099, 0):
        dev = torch.tensor([live], dtype=torch.int32, device="cuda") if live is not None else None
        m = rows if live is None else min(live, rows)
        if m == 65536 and k > 1000:
            continue
        r = layers.linear_cross_entropy(a, w, labels, bias=bias, weight=weight, rows=dev)
        da = torch.full((rows, k), SENTINEL, dtype=kind, device="cuda")
        _, dw, db = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total, rows=dev, da=da)
        assert bool((da[m:] == SENTINEL).all())
        if m == 0:
            assert not dw.any() and not db.any()
            continue
        _, wa, ww, wb = _reference(a, w, labels, bias, weight, m)
        u = {F32: 2.0**-24, F16: 2.0**-11, BF16: 2.0**-8}[kind]
        for x, y, what, e in ((da[:m], wa, "da", u), (dw, ww, "dw", u), (db, wb, "dbias", 2.0**-24)):
            # Two roundings to the type (dZ, the result) of random sign: 2 u of the length, 8 u of the largest for a cell.  Beside them probabilities made of fp32 logits of K terms, off by (K + 8) 2^-24 of the
            # sum of their magnitudes at most, and by its root for errors of random sign; 2^-18 of the length covers sums of 2^12 terms, and fp32's own.
            # fp16 below 2^-14, where a mean over 240000 rows has its gradients, has steps of 2^-24: a cell is off by half of one beside that, whatever it is.
            err, tiny = x.double() - y, 2.0**-25 if x.dtype == F16 else 0.0
            assert float(err.norm()) < (2 * e + 2.0**-18) * float(y.norm()) + tiny * y.numel() ** 0.5, (what, live)
            assert float(err.abs().max()) < (8 * e + 2.0**-16) * float(y.abs().max()) + tiny, (what, live)
        for i in range(3):  # each of them alone has the same bits
            need = tuple(j == i for j in range(3))
            got = layers.linear_cross_entropy_backward(a, w, labels, r.lse, bias=bias, weight=weight, total=r.total, rows=dev, need=need)[i]
            assert torch.equal(got[:m] if i == 0 else got, (da[:m], dw, db)[i]) or i == 2, (need, live)


def test_in_a_graph_with_counts_that_change():
    rows, k, n = 240_007, 40, 4100
    g = torch.Generator(device="cuda").manual_seed(5)
    a, w = (torch.randn(m, k, device="cuda", generator=g).mul_(s).to(BF16) for m, s in ((rows, 2.0), (n, k**-0.5)))
    labels = torch.randint(0, n, (rows,), device="cuda", generator=g)
    live = torch.tensor([rows], dtype=torch.int32, device="cuda")

    def both():
        r = layers.linear_cross_entropy(a, w, labels, rows=live)
        return (r.lse, *layers.linear_cross_entropy_backward(a, w, labels, r.lse, total=r.total, rows=live))

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for count in (rows, 70_001, 0, 65536, rows):
        live.fill_(count)
        graph.replay()
        torch.cuda.synchronize()
        eager = both()
        torch.cuda.synchronize()
        for x, y in zip(captured, eager):
            if x.shape[0] == rows:
                x, y = x[:count], y[:count]
            assert torch.equal(x, y)


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_nothing_is_written_behind_the_workspace(size, monkeypatch):
    rows, k, n, pad, kind, _, _ = size
    a, w = (torch.randn(m, k + pad, device="cuda").to(kind)[:, :k] for m in (rows, n))
    labels = torch.randint(0, n, (rows,), device="cuda")
    weight = torch.rand(rows, device="cuda")
    r = layers.linear_cross_entropy(a, w, labels, weight=weight)
    guarded = Guarded()
    monkeypatch.setattr(layers.torch, "empty", guarded)
    for live in (None, torch.tensor([rows // 2 + 3], dtype=torch.int32, device="cuda")):
        layers.linear_cross_entropy_backward(a, w, labels, r.lse, weight=weight, total=r.total, rows=live)
        guarded.check(str(live))
