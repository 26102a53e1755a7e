"""A small training loop on device-resident mini-batches: a plan's step, then a GraphSAGE layer and a pre-norm residual block on the rows it leaves, all
with the library's operators and no host read of any size.

    python -m paper_2605_29346_amd.train [--steps 100] [--hidden 256] [--optimizer muon]

The plan (`ZG_PLAN_FUSED_INPUT`) leaves [features | neighbor mean] of the innermost frontier D_{H-1} as one fp32 matrix; the model classifies the
vertices of that frontier:

    x = drop(relu([X | mean] W1^T + b1))                     fp32 operands, bfloat16 result
    h = drop(silu(norm(x; g1) W2^T + b2)) + x
    loss = mean cross entropy of norm(h; g2) W3^T + b3       bfloat16 operands, the logits are not kept

and updates its weights by their gradients, or (`--optimizer muon`) the hidden layers' by their orthogonalised momentum.
The frontier's size stays on the device (`rows`), and the masks go by vertex ids, so a vertex is dropped alike wherever it stands in a batch."""
from __future__ import annotations

import argparse
from typing import Optional

import torch

from . import layers, zg
from . import workloads as W


class Model:
    """Parameters in fp32, their gradients, and the buffers of a step (`cap` rows of capacity)."""

    def __init__(self, cap: int, width: int, hidden: int, classes: int, p: float = 0.1, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, k):
            return torch.randn(n, k, device="cuda", generator=gen) * k**-0.5

        self.p = p
        self.params = {"W1": weight(hidden, width), "b1": torch.zeros(hidden, device="cuda"), "g1": torch.ones(hidden, device="cuda"),
                       "W2": weight(hidden, hidden), "b2": torch.zeros(hidden, device="cuda"), "g2": torch.ones(hidden, device="cuda"),
                       "W3": weight(classes, hidden), "b3": torch.zeros(classes, device="cuda")}
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.buf = {name: torch.zeros(cap, hidden, **bf) for name in ("x", "z1", "y1", "t", "z2", "y2", "h")}
        self.lse = torch.zeros(cap, device="cuda")
        self.momentum = {name: torch.zeros_like(self.params[name]) for name in ("W1", "W2")}

    def step(self, fused, labels, ids, rows, key: int):
        """Loss (a device scalar) and gradients by parameter for one mini-batch: `fused` [cap, width] fp32, `labels` [cap] int64, `ids` [cap] int32,
        `rows` the frontier's size on the device."""
        P, B = self.params, self.buf
        w2, w3 = P["W2"].bfloat16(), P["W3"].bfloat16()
        d1, d2 = (layers.Dropout(self.p, key, layer, ids) for layer in (1, 2))
        layers.linear(fused, P["W1"], bias=P["b1"], act="relu", dropout=d1, rows=rows, out_dtype=torch.bfloat16, out=B["x"], preact=B["z1"])
        n1 = layers.rms_norm(B["x"], gain=P["g1"], rows=rows, y=B["y1"])
        layers.linear(n1.y, w2, bias=P["b2"], act="silu", rows=rows, out=B["t"], preact=B["z2"])
        n2 = layers.rms_norm(B["t"], gain=P["g2"], residual=B["x"], dropout=d2, rows=rows, y=B["y2"], h=B["h"])
        r = layers.linear_cross_entropy(n2.y, w3, labels, bias=P["b3"], rows=rows, lse=self.lse)

        g = {}
        dy2, g["W3"], g["b3"] = layers.linear_cross_entropy_backward(n2.y, w3, labels, r.lse, bias=P["b3"], total=r.total, rows=rows)
        dt, dx, g["g2"] = layers.rms_norm_backward(dy2, n2.h, n2.rstd, gain=P["g2"], dropout=d2, rows=rows)
        dy1, g["W2"], g["b2"] = layers.linear_backward(dt, n1.y, w2, preact=B["z2"], act="silu", rows=rows)
        dx, _, g["g1"] = layers.rms_norm_backward(dy1, B["x"], n1.rstd, gain=P["g1"], dh=dx, rows=rows)
        _, g["W1"], g["b1"] = layers.linear_backward(dx, fused, P["W1"], preact=B["z1"], act="relu", dropout=d1, rows=rows, need=(False, True, True))
        return r.loss[0], g

    def update(self, grads, lr: float, muon: Optional[float] = None):
        """Steps of `lr` against the gradients; with `muon`, the hidden layers' weights take steps of that size along their orthogonalised momentum instead."""
        for name, g in grads.items():
            if muon is not None and name in self.momentum:
                layers.muon_step(self.params[name], self.momentum[name], g, lr=muon)
            else:
                self.params[name].sub_(g.to(torch.float32), alpha=lr)


def make(workload: str = "tiny", fanouts=(5, 5), batch: int = 64, hidden: int = 256, classes: int = 16):
    """(plan, model, labels of every vertex, rows, fused input, seed pool): what the loop below runs on."""
    cfg = W.CONFIGS[workload]
    graph = cfg.build_graph()
    feat = W.feature_table(graph.num_nodes, cfg.dim, cfg.feat_seed).cuda()
    dg = zg.Graph(graph.offsets.cuda(), graph.indices.cuda())
    plan = zg.Plan(dg, fanouts, batch, zg.make_envelope(zg.ENV_MAX, flags=zg.PLAN_FUSED_INPUT), feat_dim=cfg.dim)
    plan.bind_features(feat)
    H = plan.num_hops
    fused = plan.view_X()
    if fused.shape[1] != 2 * cfg.dim:  # (a width that is a multiple of four leaves no columns between the halves)
        raise ValueError("the workload's feature width is not a multiple of four")
    rows = plan.view_counts()[0][H - 1: H]
    gen = torch.Generator(device="cuda").manual_seed(1)
    labels = (feat @ torch.randn(cfg.dim, classes, device="cuda", generator=gen)).argmax(1)
    model = Model(int(plan.out.x_row_cap), 2 * cfg.dim, hidden, classes)
    return plan, model, labels, rows, fused, W.SeedPool(graph, batch, cfg.feat_seed)


def train(steps: int, lr: float = 0.3, muon: Optional[float] = None, **kw):
    """Runs the loop and returns its losses (read at the end); `lr` and `muon` as in `Model.update`."""
    plan, model, labels, rows, fused, pool = make(**kw)
    ids = plan.view_S()[: plan.out.x_row_cap]
    losses = []
    for i in range(steps):
        plan.step(pool.batch_for(i).cuda(), 1000 + i)
        y = labels[ids.clamp(0, labels.numel() - 1).long()]
        loss, grads = model.step(fused, y, ids, rows, 1000 + i)
        model.update(grads, lr, muon)
        losses.append(loss)
    return torch.stack(losses).cpu().tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--lr", type=float, default=0.3)
    ap.add_argument("--optimizer", choices=("sgd", "muon"), default="sgd")
    ap.add_argument("--muon-lr", type=float, default=0.02)
    a = ap.parse_args()
    losses = train(a.steps, a.lr, a.muon_lr if a.optimizer == "muon" else None, hidden=a.hidden)
    for i in range(0, len(losses), 10):
        print(f"step {i}: loss {losses[i]:.4f}")
    print(f"last: loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
