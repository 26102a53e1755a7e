"""What the loss' gradients ask for as a workspace, over rows, widths, classes and types: the logits are not kept, and neither is anything like them.  Asked of the library on the host."""
import ctypes as C

import pytest

from paper_2605_29346_amd import zg

SIZE = {zg.F32: 4, zg.F16: 2, zg.BF16: 2}
GB = 2**30
SHARE = 7 * 2**28  # what may always be asked for
MORE = 2**28       # of parts of sums beside one whole dZ


def _bytes(rows, k, n, t, weight=False, **need):
    out = C.c_size_t()
    b = zg.LossGradArgs(rows=rows, in_=k, out=n, dtype=t, label_dtype=zg.I64, d_A=1 << 56, ld_A=k, d_W=2 << 56, ld_W=k, d_labels=3 << 56, d_weight=(4 << 56) if weight else None, d_lse=5 << 56, d_dA=6 << 56, ld_dA=k,
                        d_dW=7 << 56, ld_dW=k, d_dbias=8 << 56)
    for name, v in need.items():
        setattr(b, name, v)
    assert zg.lib().zg_linear_cross_entropy_backward_workspace(C.byref(b), C.byref(out)) == zg.OK
    return out.value


# what was asked for here: 17.5, 43.6, 9.1, 23.6 and 9.7 GB, the logits being 17.2, 41.9, 2.1, 17.2 and 2.1
@pytest.mark.parametrize("rows,k,n,t,most", [(1 << 20, 256, 4096, zg.F32, 2 * GB), (1 << 22, 256, 5000, zg.BF16, 2 * GB), (65536, 8192, 16384, zg.BF16, 2 * GB), (262144, 4096, 32768, zg.BF16, 3 * GB),
                                             (131072, 8192, 8192, zg.BF16, 2 * GB)], ids=str)
def test_many_rows_and_wide_ones(rows, k, n, t, most):
    assert _bytes(rows, k, n, t) <= most


@pytest.mark.parametrize("t", SIZE)
@pytest.mark.parametrize("weight", [False, True])
def test_never_more_than_the_logits(t, weight):
    """A share that does not grow, or one dZ of the operands' type (rows rounded up to eight classes), sums of it for dbias (an eighth) and parts of sums; far below that where the logits are large and `in` is
    not."""
    for rows in (1, 17, 300, 4099, 33000, 70000, 131073, 300000, 1 << 20, 3 << 20, (1 << 31) - 1):
        for k in (8, 256, 1024, 4096, 32768):
            for n in (2, 47, 1000, 4096, 5003, 20000, 131072, 1 << 20, zg.MAX_CLASSES):
                got, logits = _bytes(rows, k, n, t, weight), rows * ((n + 7) // 8 * 8) * SIZE[t]
                assert got <= max(SHARE, logits * 9 // 8 + MORE), (rows, k, n, got / GB, logits / GB)
                # Running sums at 32 bits: two of rows by `in` where the classes are more, and then dZ may be 4096 classes of all rows (with dbias' sums, an eighth); of classes by `in` where the rows are more, and
                # then dZ is of a piece of them.
                piece = 4608 * rows * SIZE[t] if rows <= n else 0
                assert got <= 2 * SHARE + 8 * min(rows, n) * k + piece + rows // 1024, (rows, k, n, got / GB, logits / GB)


@pytest.mark.parametrize("t", SIZE)
def test_copies_of_operands_are_of_a_piece_of_the_rows(t):
    """Rows that lie anyhow are copied as they are needed."""
    even, odd = _bytes(1 << 20, 304, 4096, t), _bytes(1 << 20, 301, 4096, t)
    assert odd <= even + (1 << 28)
