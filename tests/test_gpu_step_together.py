"""The loss and the update together, as a training step has them: on a plan's mini-batch through the training module, and as a head and its update captured into one graph."""
import pytest
import torch

import orthogonal_util as O
from paper_2605_29346_amd import layers, train, zg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def test_an_update_on_a_plans_mini_batch():
    """Two steps of the training module: the hidden layers' weights against the update in 64 bits of the same gradients, the others' against theirs."""
    plan, model, labels, rows, fused, pool = train.make()
    ids = plan.view_S()[: plan.out.x_row_cap]
    momentum = {name: m.double() for name, m in model.momentum.items()}
    for i in range(2):
        plan.step(pool.batch_for(i).cuda(), 77 + i)
        y = labels[ids.clamp(0, labels.numel() - 1).long()]
        loss, grads = model.step(fused, y, ids, rows, 77 + i)
        before = {name: p.double() for name, p in model.params.items()}
        model.update(grads, 0.3, 0.02)
        assert bool(torch.isfinite(loss))
        for name, p in model.params.items():
            g = grads[name].double()
            if name in momentum:
                momentum[name] = m = 0.95 * momentum[name] + g
                u = (0.95 * m + g).float()
                s = 0.02 * max(1.0, p.shape[0] / p.shape[1]) ** 0.5
                want = before[name] - s * O.exact(u)
                off = s * (O.emulated(u, torch.float32) - O.exact(u)).norm()
                # beside the products' error: u's rounding to fp32 (a relative 2^-24 of each cell, grown by no more than 3.9 a step: 900) and w's own
                bound = O.SLACK * off + 900 * 2.0**-23 * s + 2.0**-23 * want.norm()
                assert float((p.double() - want).norm()) <= float(bound), name
            else:
                want = before[name] - 0.3 * g
                assert float((p.double() - want).abs().max()) <= 2.0**-22 * float(want.abs().max() + g.abs().max()), name


def test_the_loop_runs_with_both_updates():
    for muon in (None, 0.02):
        losses = train.train(8, muon=muon)
        assert len(losses) == 8 and all(x == x and abs(x) < 1e3 for x in losses)


def test_a_head_and_its_update_in_one_graph():
    """Loss, gradients and update of a head captured once and replayed, against the same calls one by one; the graph's workspaces are its own."""
    g = torch.Generator(device="cuda").manual_seed(3)
    a = torch.randn(900, 128, device="cuda", generator=g).bfloat16()
    y = torch.randint(0, 300, (900,), device="cuda", generator=g, dtype=torch.int32)
    start = torch.randn(300, 128, device="cuda", generator=g) * 128**-0.5

    def step(w, m):
        half = w.bfloat16()
        r = layers.linear_cross_entropy(a, half, y)
        _, dw, _ = layers.linear_cross_entropy_backward(a, half, y, r.lse, total=r.total, need=(False, True, False))
        layers.muon_step(w, m, dw, lr=0.05)
        return r.loss

    w, m = start.clone(), torch.zeros_like(start)
    graph = torch.cuda.CUDAGraph()
    step(w, m)
    with torch.cuda.graph(graph):
        loss = step(w, m)
    w.copy_(start), m.zero_()
    ew, em = start.clone(), torch.zeros_like(start)
    for _ in range(4):
        graph.replay()
        eager = step(ew, em)
        torch.cuda.synchronize()
        assert torch.equal(loss, eager) and torch.equal(w, ew) and torch.equal(m, em)
    # the same on another stream and under another current stream, memory handed over as torch expects
    side = torch.cuda.Stream()
    sw, sm = start.clone(), torch.zeros_like(start)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(4):
            step(sw, sm)
    torch.cuda.synchronize()
    assert torch.equal(sw, ew) and torch.equal(sm, em)
