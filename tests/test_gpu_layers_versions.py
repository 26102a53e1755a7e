"""What the operators write into tensors that the caller gave counts as a change in place: a backward pass that saved such a tensor before it is refused by torch, as behind torch's own changes."""
import pytest
import torch

from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def _m(rows, cols, kind=torch.float32):
    return torch.randn(rows, cols, device="cuda").to(kind)


@pytest.mark.parametrize("kind", [torch.float32, BF16], ids=str)
def test_an_update_behind_a_saved_weight(kind):
    w = _m(48, 64, kind).requires_grad_()
    x = _m(10, 64, kind).requires_grad_()
    y = (x @ w.t()).sum()  # (saves w for x's gradient)
    with torch.no_grad():
        layers.muon_step(w, torch.zeros(48, 64, device="cuda"), _m(48, 64), lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    momentum = _m(48, 64).requires_grad_()
    z = (momentum * momentum).sum()
    with torch.no_grad():
        layers.muon_step(w, momentum, _m(48, 64), lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    (x @ w.t()).sum().backward()  # (a pass that begins behind it runs)
    assert torch.equal(x.grad, torch.ones(10, 48, dtype=kind, device="cuda") @ w.detach())


V = lambda n: torch.zeros(n, device="cuda")
Y = lambda: torch.zeros(9, dtype=torch.int64, device="cuda")
GIVEN = {  # each call with every output that it takes, on 9 x 16 operands and 16 x 16 weights
    "linear": lambda: (lambda out, preact: layers.linear(_m(9, 16), _m(16, 16), out=out, preact=preact), [_m(9, 16), _m(9, 16)]),
    "linear_backward": lambda: (lambda da, dw, db: layers.linear_backward(_m(9, 16), _m(9, 16), _m(16, 16), da=da, dw=dw, dbias=db), [_m(9, 16), _m(16, 16), V(16)]),
    "dropout": lambda: (lambda out: layers.dropout(_m(9, 16), layers.Dropout(0.5, 1), out=out), [_m(9, 16)]),
    "rms_norm": lambda: (lambda y, h, r: layers.rms_norm(_m(9, 16), residual=_m(9, 16), y=y, h=h, rstd=r), [_m(9, 16), _m(9, 16), V(9)]),
    "rms_norm_backward": lambda: (lambda dx, dr, dg: layers.rms_norm_backward(_m(9, 16), _m(9, 16), V(9) + 1, gain=V(16) + 1, dx=dx, dr=dr, dgain=dg), [_m(9, 16), _m(9, 16), V(16)]),
    "linear_cross_entropy": lambda: (lambda *o: layers.linear_cross_entropy(_m(9, 16), _m(16, 16), Y(), loss=o[0], total=o[1], lse=o[2], row_loss=o[3]), [V(1), V(1), V(9), V(9)]),
    "linear_cross_entropy_backward": lambda: (lambda *o: layers.linear_cross_entropy_backward(_m(9, 16), _m(16, 16), Y(), V(9), da=o[0], dw=o[1], dbias=o[2]), [_m(9, 16), _m(16, 16), V(16)]),
    "orthogonalize": lambda: (lambda out: layers.orthogonalize(_m(9, 16), out=out), [_m(9, 16)]),
}


@pytest.mark.parametrize("name", GIVEN)
def test_outputs_that_were_given(name):
    call, outs = GIVEN[name]()
    before = [t._version for t in outs]
    call(*outs)
    assert all(t._version > v for t, v in zip(outs, before))
    with torch.inference_mode():  # (tensors without versions)
        call, outs = GIVEN[name]()
        call(*outs)


def test_a_refused_call_changes_nothing():
    w, m = _m(48, 64), _m(48, 64)
    before = w._version, m._version
    for bad in (dict(lr=float("nan")), dict(lr=0.1, steps=0), dict(lr=0.1, coefficients=(100.0, 0.0, 0.0))):
        with pytest.raises((ValueError, zg.ZgError)):
            layers.muon_step(w, m, _m(48, 64), **bad)
    assert (w._version, m._version) == before
