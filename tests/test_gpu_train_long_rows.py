"""Layer norm on very wide rows."""
import numpy as np
import pytest

from tests import train_oracle as O
from tests.test_gpu_train_norm import host, run_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [40001, 1 << 20, 1 << 24])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_common_offset_of_a_wide_row(H, dtype):
    """Constant rows come out as zeros and rows with a common offset as their deviations, however wide: sums in float32 of at most 64 numbers
    one after the other, the rest in more bits, leave the mean within 70 half units of the offset."""
    import torch
    rng = np.random.default_rng(H)
    dt = getattr(torch, dtype)
    x = torch.full((2, H), 100.125 if dtype == "float32" else 100.5, device="cuda")
    x[1] += torch.from_numpy((rng.integers(0, 2, H) * 2 - 1).astype(np.float32)).cuda()
    x = x.to(dt)
    y, mean, rstd = run_forward(x, None, None, 1e-5, "float32")
    xd = host(x)
    off = 70 * O.U * np.abs(xd).mean(1)
    assert (np.abs(host(mean) - xd.mean(1)) <= off).all(), (host(mean), xd.mean(1))
    var = xd.var(1)
    room = (off ** 2 + 80 * O.U * var) / (var + 1e-5)                 # the mean's error squared; relative, half of it under the root
    assert (np.abs(host(rstd) * np.sqrt(var + 1e-5) - 1) <= room + 8 * O.U).all()
    want = (xd - xd.mean(1, keepdims=True)) / np.sqrt(var + 1e-5)[:, None]
    O.assert_within(host(y), want, (off / np.sqrt(var + 1e-5))[:, None] + np.abs(want) * (room[:, None] + 8 * O.U), dtype, "y")
