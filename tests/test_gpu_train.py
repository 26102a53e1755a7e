"""The training loop on device-resident mini-batches: its first step's loss and gradients against the same model differentiated by torch in 64 bits on
the host, and its losses over a run."""
import pytest
import torch

import layers_util as R
from paper_2605_29346_amd import train, zg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


def test_a_steps_loss_and_gradients():
    """bfloat16 between the layers: eight significant bits a rounding, a handful of roundings one behind the other, of random sign over
    hundreds of rows: 3 % of a gradient's length."""
    plan, model, labels, rows, fused, pool = train.make()
    ids = plan.view_S()[: plan.out.x_row_cap]
    plan.step(pool.batch_for(3).cuda(), 77)
    y = labels[ids.clamp(0, labels.numel() - 1).long()]
    loss, grads = model.step(fused, y, ids, rows, 77)
    n = int(rows.item())
    assert 64 < n < fused.shape[0]
    P = {k: v.double().cpu().requires_grad_() for k, v in model.params.items()}
    who = ids[:n].cpu().numpy()

    def norm(v, gain):
        return v * (v.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt() * gain

    a = R.d64(fused)[:n]
    x = R.drop(torch.relu(a @ P["W1"].t() + P["b1"]), (model.p, 77, 1), who)
    t = torch.nn.functional.silu(norm(x, P["g1"]) @ P["W2"].t() + P["b2"])
    h = R.drop(t, (model.p, 77, 2), who) + x
    logits = norm(h, P["g2"]) @ P["W3"].t() + P["b3"]
    want = torch.nn.functional.cross_entropy(logits, y[:n].cpu())
    want.backward()
    want = float(want.detach())
    assert abs(float(loss) - want) < 0.01 * want
    for name, p in P.items():
        err = (R.d64(grads[name]) - p.grad).norm() / p.grad.norm()
        assert err < 0.03, (name, float(err))


def test_the_loss_falls():
    losses = train.train(60)
    assert all(x == x for x in losses) and sum(losses[-5:]) < 0.8 * sum(losses[:5]), losses
