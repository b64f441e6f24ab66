"""Layer norm written over its inputs, on rows that begin off 16 bytes and have gaps between them."""
import numpy as np
import pytest

from tests.test_gpu_train_norm import TYPES, make, run_backward, run_forward, vector

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,H,pad,offset", [(700, 1367, 9, 1), (300, 2050, 2, 2), (900, 97, 3, 1), (1500, 130, 1, 0), (40, 10007, 5, 3), (9, 33001, 7, 1), (64, 515, 1, 5)])
def test_in_place_on_rows_with_gaps(rows, H, pad, offset, dtype, wdtype):
    """Results written over inputs whose rows begin off 16 bytes with other numbers between them: the same bits as into a tensor of its own, and
    the numbers between stay."""
    import torch
    rng = np.random.default_rng([rows, H])
    x, _ = make(rng, rows, H, dtype, pad, offset)
    dy, _ = make(rng, rows, H, dtype, pad, offset)
    gamma, _ = vector(rng, H, wdtype, 1.0, offset)
    beta, _ = vector(rng, H, wdtype, 0.0, offset)

    def copy_of(t):
        c, _ = make(np.random.default_rng(0), rows, H, dtype, pad, offset)
        c.copy_(t)
        return c

    def gaps(t):
        return t.as_strided((rows - 1, pad), (H + pad, 1), offset + H)

    out, _ = make(rng, rows, H, dtype, pad, offset)
    y, mean, rstd = run_forward(x, gamma, beta, 1e-5, wdtype, y=out)
    same = copy_of(x)
    assert torch.equal(run_forward(same, gamma, beta, 1e-5, wdtype, y=same)[0], y) and (gaps(same) == 77.0).all()
    dx, _ = make(rng, rows, H, dtype, pad, offset)
    want = run_backward(dy, x, gamma, mean, rstd, 3, 16, None, wdtype, dx=dx)
    for which in (0, 1):
        a = [copy_of(dy), copy_of(x)]
        got = run_backward(a[0], a[1], gamma, mean, rstd, 3, 16, None, wdtype, dx=a[which])
        assert all(torch.equal(p, q) for p, q in zip(got, want)) and (gaps(a[which]) == 77.0).all()
