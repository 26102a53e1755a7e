"""The loss, its gradients, orthogonalised matrices and the update write nothing behind the workspace that they ask for, and nothing behind their results: each allocation of a call has a megabyte
of a pattern behind it, more than the longest row of sums at these sizes."""
import math

import pytest
import torch

from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
BEHIND, PATTERN = 1 << 20, 0xA5
ROWS = [1, 3, 4, 15, 16, 17, 31, 33, 48, 49, 79, 127, 200, 300, 515, 700, 2100]  # halves of tiles of 32 rows that there are, and those that there are not
WIDTHS = [(1024, 900), (64, 47), (33, 129), (520, 2056)]  # of a row, classes


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


class Guarded:
    def __init__(self):
        self.made, self.empty = [], torch.empty

    def __call__(self, *shape, dtype, device):
        shape = shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape
        size = math.prod(shape) * dtype.itemsize
        whole = torch.full((size + BEHIND,), PATTERN, dtype=torch.uint8, device=device)
        self.made.append((whole, size))
        return whole[:size].view(dtype).view(shape)

    def check(self, what):
        assert self.made
        for whole, size in self.made:
            assert bool((whole[size:] == PATTERN).all()), f"{what}: something was written behind {size} bytes"
        self.made.clear()


@pytest.fixture
def guarded(monkeypatch):
    g = Guarded()
    monkeypatch.setattr(layers.torch, "empty", g)
    return g


@pytest.mark.parametrize("kind", [F32, F16, BF16])
@pytest.mark.parametrize("widths", WIDTHS, ids=str)
def test_loss_and_gradients(guarded, widths, kind):
    k, n = widths
    g = torch.Generator(device="cuda").manual_seed(k)
    for rows in ROWS:
        a, w = (torch.randn(m, k, device="cuda", generator=g).to(kind) for m in (rows, n))
        labels = torch.randint(0, n, (rows,), device="cuda", generator=g)
        weight = torch.rand(rows, device="cuda", generator=g)
        for live in (None, torch.tensor([(rows + 1) // 2], dtype=torch.int32, device="cuda")):
            r = layers.linear_cross_entropy(a, w, labels, weight=weight, rows=live, row_loss=True)
            guarded.check(f"loss {rows} {live}")
            for need in ((True, True, True), (False, False, True)):
                layers.linear_cross_entropy_backward(a, w, labels, r.lse, weight=weight, total=r.total, rows=live, need=need)
                guarded.check(f"gradients {rows} {live} {need}")


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("size", [(1, 1), (7, 5), (64, 384), (384, 64), (65, 33), (31, 500), (100, 1000), (255, 255), (600, 1201), (1201, 600), (700, 2003), (1025, 1100)], ids=str)
def test_matrices_and_the_update(guarded, size, kind):
    g = torch.Generator(device="cuda").manual_seed(size[0])
    x, w, m = (torch.randn(size, device="cuda", generator=g) for _ in range(3))
    layers.orthogonalize(x.to(kind))
    guarded.check("orthogonalize")
    layers.muon_step(w.to(kind), m, x.to(kind), lr=0.1)
    guarded.check("update")
