"""The order in which parts of a sum are added: up to 32 of them one after the other, more than that every 32nd and then those, whatever the result's size.  Each part holds one value (exact), so a
result is a chain of fp32 additions, bit by bit."""
import pytest
import torch

from paper_2605_29346_amd import layers, zg

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    zg.lib()


@pytest.mark.parametrize("kind", [F32, F16, BF16], ids=str)
# weights' rows and columns, parts of 256 rows of the batch each: few and many cells, parts of every number that changes the way they are joined
@pytest.mark.parametrize("out,in_,parts", [(64, 64, 2), (64, 64, 5), (256, 128, 16), (264, 136, 32), (64, 64, 33), (64, 72, 48), (1000, 520, 21), (1024, 512, 16), (1024, 1024, 16), (1024, 1024, 3), (1048, 2056, 6)], ids=str)
def test_parts_are_added_in_order(kind, out, in_, parts):
    g = torch.Generator(device="cuda").manual_seed(parts)
    rows = 256 * parts
    values = (torch.randn(parts, out, device="cuda", generator=g) * 2.0 ** torch.randint(-6, 7, (parts, out), device="cuda", generator=g)).to(kind)
    dy, a = torch.zeros(rows, out, dtype=kind, device="cuda"), torch.zeros(rows, in_, dtype=kind, device="cuda")
    dy[5::256], a[5::256] = values, 1.0
    dw = layers.linear_backward(dy, a, torch.zeros(out, in_, dtype=kind, device="cuda"), need=(False, True, False))[1]
    lanes = [torch.zeros(out, device="cuda") for _ in range(min(parts, 32))]
    for s in range(parts):
        lanes[s % 32] = lanes[s % 32] + values[s].float()
    want = torch.zeros(out, device="cuda")
    for v in lanes:
        want = want + v
    assert torch.equal(dw, want.to(kind)[:, None].expand(out, in_))
