"""Performance cases of what closes a training step: the loss of a linear layer over many classes, and the update of a layer's weights.

`linear_cross_entropy` is the softmax cross entropy of A W^T + bias against a class for each row, a mean over the rows that have one, made without keeping
the logits, with its gradients; `orthogonalize` brings the singular values of a matrix near one by Newton-Schulz products, and `muon_step` is the weights'
update that uses it: momentum, orthogonalised, behind a weight decay.

`own` chooses between the plain forms below (elementary torch operations in 32 bits, rounded once; products in 64 bits where an orthogonalised
matrix is returned in 32, whose small singular values grow by 3.4 in each of five steps, the errors of 32-bit sums with them) and the library's kernels.
`exact` has the same values in 64 bits from the definitions.  Feature widths, batches and vertex counts are those of the benchmark's workloads; hidden widths and
class counts are generic."""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
STEP = (3.4445, -4.7750, 2.0315)  # x -> a x + b x^3 + c x^5 on the singular values
EPS = 1e-7
RATE = 0.02


def _loss(name, dtype, rows, k, n, **more):
    return {"name": name, "op": "loss", "dtype": dtype, "rows": rows, "in": k, "out": n, "bias": True, "weight": False, "labelled": 1.0, "count": 0, "pad": 0, **more}


def _orth(name, dtype, rows, cols, **more):
    return {"name": name, "op": "orthogonalize", "dtype": dtype, "out": dtype, "rows": rows, "cols": cols, "steps": 5, "pad": 0, **more}


def _muon(name, dtype, rows, cols, **more):
    return {"name": name, "op": "muon", "dtype": dtype, "grad": dtype, "rows": rows, "cols": cols, "steps": 5, "nesterov": True, "decay": 0.1, "pad": 0, **more}


def listed():
    return [
        # serving: how likely one vertex's class is, out of fifty thousand
        _loss("loss_one_row", "bf16", 1, 1024, 50_021, bias=False),
        # the training loop on the smallest workload: the frontier of a batch of 64 as many rows as the device says, sixteen classes; loss and gradients
        _loss("loss_small_step", "bf16", 2_304, 256, 16, op="loss_step", count=611),
        # node classification over a wide frontier: few and odd classes, fp32, labels on some of the vertices only; loss and gradients
        _loss("loss_frontier_step", "f32", 98_765, 256, 47, op="loss_step", labelled=0.3),
        # predicting a vertex out of all of the medium graph's for each seed of a batch
        _loss("loss_vertices", "bf16", 4_096, 256, 250_000),
        # a large vocabulary in training
        _loss("loss_vocabulary", "bf16", 16_384, 1024, 131_072, bias=False),
        # its gradients, over half as many classes
        _loss("loss_gradients", "bf16", 16_384, 1024, 65_536, op="loss_backward"),
        # gradients where nothing is even: odd widths, rows that start anywhere, weighted rows, some without a label
        _loss("loss_gradients_ragged", "f16", 4_099, 301, 10_007, op="loss_backward", weight=True, labelled=0.9, pad=1),
        # a hidden layer's weights, the smallest update
        _orth("orthogonal_small", "bf16", 256, 256),
        # a wide layer's gradient
        _orth("orthogonal_wide", "bf16", 1_024, 4_096),
        # an odd and tall one in 32 bits, rows that start anywhere
        _orth("orthogonal_tall_f32", "f32", 1_201, 600, pad=3),
        # the update of a layer kept in 32 bits, its gradient in 16
        _muon("muon_f32", "f32", 1_024, 2_048, grad="bf16"),
        # the update of the largest layer
        _muon("muon_large", "bf16", 4_096, 4_096),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))

    op = rng.choice(["loss", "loss", "loss_backward", "loss_backward", "loss_step", "orthogonalize", "orthogonalize", "muon", "muon"])
    dtype, pad = rng.choice(["f32", "bf16", "f16"]), rng.choice([0, 0, 1, 8])
    if op.startswith("loss"):
        rows = log(1, 131_072)
        case = {"op": op, "dtype": dtype, "rows": rows, "in": log(1, 2048), "out": log(2, 262_144), "bias": rng.random() < 0.6, "weight": rng.random() < 0.3,
                "labelled": rng.choice([1.0, 1.0, 0.9, 0.3]), "count": rng.choice([0, 0, rng.randint(0, rows)]), "pad": pad}
    else:
        case = {"op": op, "dtype": dtype, "rows": log(1, 4096), "cols": log(1, 4096), "steps": rng.choice([5, 5, 5, 4, 6]), "pad": pad}
        if op == "orthogonalize":
            case["out"] = rng.choice([dtype, "f32", "bf16"])
        else:
            case |= {"grad": rng.choice([dtype, "f32", "bf16"]), "nesterov": rng.random() < 0.7, "decay": rng.choice([0.0, 0.1])}
    alike = [c for c in listed() if c["op"][:4] == op[:4]]
    while _cost(case) > max(map(_cost, alike)) or (op[:4] == "loss" and _cells(case) > max(map(_cells, alike))):  # no more than the largest one of its kind
        long = "rows" if case["rows"] >= case.get("cols", 0) else "cols"
        case[long] -= -(-case[long] // 8)
        if "count" in case:
            case["count"] = min(case["count"], case["rows"])
    return case


def _cells(case):
    return case["rows"] * case["out"]


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"].startswith("loss"):
        m, k, n = case["count"] or case["rows"], case["in"], case["out"]
        rows, read = 4 * m * (2 + case["weight"]), e * (m * k + n * k) + 4 * n * case["bias"]
        forward = {"bytes": read + rows + 4 * m, "flops": 2.0 * m * k * n}
        if case["op"] == "loss":
            return forward
        backward = {"bytes": 2 * read + rows + 4 * m, "flops": 6.0 * m * k * n}  # (the logits again, and two products)
        return backward if case["op"] == "loss_backward" else {k: forward[k] + backward[k] for k in forward}
    n, m = sorted((case["rows"], case["cols"]))
    # the Gram matrix and its square are symmetric: half of their cells
    flops = case["steps"] * (n * (n + 1.0) * m + n * (n + 1.0) * n + 2.0 * n * n * m)
    if case["op"] == "orthogonalize":
        return {"bytes": n * m * (e + SIZE[case["out"]]), "flops": flops}
    return {"bytes": n * m * (SIZE[case["grad"]] + 8 + 2 * e), "flops": flops}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, rows, pad = case["op"], case["rows"], case["pad"]
    dtype = TYPES[case["dtype"]]

    def inside(t, kind):  # rows inside wider rows where the case says so
        if not pad:
            return t.to(kind)
        wide = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=kind, device="cuda")
        wide[:, : t.shape[1]] = t
        return wide[:, : t.shape[1]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    s = {"case": case}
    if op.startswith("loss"):
        k, n = case["in"], case["out"]
        w = normal(n, k) * k**-0.5
        label = torch.randint(0, n, (rows,), device="cuda", generator=gen)
        known = torch.rand(rows, device="cuda", generator=gen)
        a = 2.0 * normal(rows, k) + torch.where(known < 0.5, 8.0, 0.0)[:, None] * w[label]  # logits of a model that has learnt half of its rows
        none = torch.rand(rows, device="cuda", generator=gen) >= case["labelled"]
        none[0] = False  # (a batch without any label would not be trained on)
        s["a"], s["w"], s["labels"] = inside(a, dtype), inside(w, dtype), torch.where(none, -1, label)
        s["bias"] = normal(n) * 0.1 if case["bias"] else None
        s["weight"] = torch.rand(rows, device="cuda", generator=gen) + 0.5 if case["weight"] else None
        s["rows"] = torch.tensor([case["count"]], dtype=torch.int32, device="cuda") if case["count"] else None
        live = case["count"] > 0  # buffers that hold more rows than there are: zeros where nobody writes
        s["lse"] = torch.zeros(rows, device="cuda") if live else None
        s["da"] = torch.zeros(rows, k, dtype=dtype, device="cuda") if live else None
        if op == "loss_backward":  # what the forward pass left
            z = s["a"].float() @ s["w"].float().t()
            s["lse"] = torch.logsumexp(z + s["bias"] if case["bias"] else z, 1)
            s["total"] = _weights(s).sum().reshape(1)
        return s
    cols, rank = case["cols"], min(rows, case["cols"], 32)
    # a momentum buffer: a few strong directions of falling strength, and noise in all
    strong = (normal(rows, rank) * torch.linspace(1.0, 0.1, rank, device="cuda")) @ normal(rank, cols)
    g = (strong * rank**-0.5 + 0.2 * normal(rows, cols)) * 1e-3
    if op == "orthogonalize":
        s["g"] = inside(g, dtype)
        return s
    s["g"] = inside(g, TYPES[case["grad"]])
    s["m"] = inside(6.0 * g + 1e-3 * normal(rows, cols), torch.float32)
    s["w"] = inside(normal(rows, cols) * cols**-0.5, dtype)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------------------

def _weights(s):
    """What each row counts: its weight, 0 where it has no label or is beyond the device's count."""
    here = s["labels"] >= 0
    if s["rows"] is not None:
        here = here & (torch.arange(here.numel(), device="cuda") < s["rows"])
    return torch.where(here, s["weight"] if s["weight"] is not None else 1.0, 0.0)


def _live(v, s):
    """Zeros in the rows that the device's count leaves out."""
    if s["rows"] is None:
        return v
    here = torch.arange(v.shape[0], device="cuda") < s["rows"]
    return torch.where(here if v.dim() == 1 else here[:, None], v, 0.0)


def _logits(s):
    z = torch.matmul(s["a"].float(), s["w"].float().t())
    return z + s["bias"] if s["bias"] is not None else z


def _plain_loss(s, z):
    top = z.max(1, keepdim=True).values
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    weight, total = _weights(s), _weights(s).sum()
    each = torch.where(weight != 0, lse - z.gather(1, s["labels"].clamp_min(0)[:, None])[:, 0], 0.0)
    return {"loss": (weight * each).sum() / torch.where(total != 0, total, 1.0), "lse": _live(lse, s)}, total


def _plain_gradients(s, z, lse, total):
    weight = (_weights(s) / torch.where(total != 0, total, 1.0))[:, None]
    dz = torch.exp(z - lse[:, None])
    dz.scatter_add_(1, s["labels"].clamp_min(0)[:, None], torch.full_like(weight, -1.0))
    dz = torch.where(weight != 0, dz * weight, 0.0)
    out = {"da": torch.matmul(dz, s["w"].float()).to(s["a"].dtype), "dw": torch.matmul(dz.t(), s["a"].float()).to(s["a"].dtype)}
    return {**out, "dbias": dz.sum(0)} if s["bias"] is not None else out


def _newton_schulz(g, steps, kind):
    """Products and what lies between them in `kind`."""
    x = g.to(kind)
    x = x / (torch.sqrt((g.double() ** 2).sum()) + EPS).to(kind)
    x = x.t() if g.shape[0] > g.shape[1] else x
    a, b, c = STEP
    for _ in range(steps):
        gram = torch.matmul(x, x.t())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return x.t() if g.shape[0] > g.shape[1] else x


def _scale(case):
    return max(1.0, case["rows"] / case["cols"]) ** 0.5


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "loss":
        return _plain_loss(s, _logits(s))[0]
    if op == "loss_backward":
        return _plain_gradients(s, _logits(s), s["lse"], s["total"])
    if op == "loss_step":
        z = _logits(s)
        out, total = _plain_loss(s, z)
        return {**out, **_plain_gradients(s, z, out["lse"], total)}
    if op == "orthogonalize":
        kind = TYPES[case["out"]]
        return {"o": _newton_schulz(s["g"], case["steps"], torch.float64 if kind == torch.float32 else torch.float32).to(kind).contiguous()}
    m = 0.95 * s["m"] + s["g"].float()
    u = 0.95 * m + s["g"].float() if case["nesterov"] else m
    o = _newton_schulz(u, case["steps"], torch.float32)
    s["m"].copy_(m)
    s["w"].copy_((1 - RATE * case["decay"]) * s["w"].float() - RATE * _scale(case) * o)
    return {"w": s["w"], "m": s["m"]}


# ---- the library's operators ----------------------------------------------------------------------------------------------------

def _kernels(s):
    from paper_2605_29346_amd import layers
    case, op = s["case"], s["case"]["op"]
    if op == "orthogonalize":
        return {"o": layers.orthogonalize(s["g"], steps=case["steps"], coefficients=STEP, eps=EPS, out_dtype=TYPES[case["out"]])}
    if op == "muon":
        layers.muon_step(s["w"], s["m"], s["g"], lr=RATE, momentum=0.95, nesterov=case["nesterov"], decay=case["decay"], scale=_scale(case), steps=case["steps"],
                         coefficients=STEP, eps=EPS)
        return {"w": s["w"], "m": s["m"]}
    given = {"bias": s["bias"], "weight": s["weight"], "rows": s["rows"]}
    out = {}
    lse, total = s["lse"], s.get("total")
    if op != "loss_backward":
        r = layers.linear_cross_entropy(s["a"], s["w"], s["labels"], lse=s["lse"], **given)
        out = {"loss": r.loss[0], "lse": r.lse}
        lse, total = r.lse, r.total
    if op != "loss":
        da, dw, dbias = layers.linear_cross_entropy_backward(s["a"], s["w"], s["labels"], lse, total=total, da=s["da"], need=(True, True, s["bias"] is not None), **given)
        out |= {"da": da, "dw": dw}
        if s["bias"] is not None:
            out["dbias"] = dbias
    return out


def run(state):
    return _kernels(state) if own else _plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op, rows = case["op"], case["rows"]
    if op.startswith("loss"):
        n = case["count"] or rows
        a, w = s["a"][:n].double(), s["w"].double()
        z = torch.addmm(s["bias"].double(), a, w.t()) if case["bias"] else a @ w.t()
        lse = torch.logsumexp(z, 1)
        label, who = s["labels"][:n], torch.arange(n, device="cuda")
        counts = torch.zeros(n, dtype=torch.float64, device="cuda")
        counts[label >= 0] = 1.0 if s["weight"] is None else s["weight"][:n][label >= 0].double()
        total = counts.sum().clamp_min(1e-300)
        whole = torch.zeros(rows, dtype=torch.float64, device="cuda")
        whole[:n] = lse
        out = {} if op == "loss_backward" else {"loss": counts @ (lse - z[who, label.clamp_min(0)]) / total, "lse": whole}
        if op == "loss":
            return out
        z.sub_(lse[:, None]).exp_()  # probabilities
        z[who, label.clamp_min(0)] -= 1.0
        z.mul_((counts / total)[:, None])
        da = torch.zeros(rows, case["in"], dtype=torch.float64, device="cuda")
        da[:n] = z @ w
        out |= {"da": da, "dw": z.t() @ a}
        return {**out, "dbias": z.sum(0)} if case["bias"] else out
    m = s["m"].double() * 0.95 + s["g"].double() if op == "muon" else None
    x = s["g"].double() if m is None else m * 0.95 + s["g"].double() if case["nesterov"] else m
    x = x / (x.pow(2).sum().sqrt() + EPS)
    eye = torch.eye(min(x.shape), dtype=torch.float64, device="cuda")
    for _ in range(case["steps"]):  # (a + b S + c S^2) on the shorter side, as a + S (b + c S)
        s2 = x @ x.t() if x.shape[0] <= x.shape[1] else x.t() @ x
        p = STEP[0] * eye + s2 @ (STEP[1] * eye + STEP[2] * s2)
        x = p @ x if x.shape[0] <= x.shape[1] else x @ p
    if op == "orthogonalize":
        return {"o": x}
    return {"w": s["w"].double() * (1 - RATE * case["decay"]) - RATE * _scale(case) * x, "m": m}
