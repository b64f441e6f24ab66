"""Layer norm backward where the rows of one group lie behind a great many processes without rows."""
import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import train_oracle as O
from tests.test_gpu_train_norm import host, make, run_backward, run_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,k", [(8, 8), (300, 512), (8200, 8200)])
def test_gap_of_empty_processes(H, k):
    """Few hold rows: the first ones, some in the middle, the last ones."""
    rng = np.random.default_rng(H)
    rows, P = 700, 5000 if H < 8000 else 700
    x, xd = make(rng, rows, H, "bfloat16")
    dy, dyd = make(rng, rows, H, "bfloat16")
    _, mean, rstd = run_forward(x, None, None, 1e-5, "float32")
    for cut in (1, 33, 350, 699):
        splits = np.full(P + 1, cut)
        splits[:2] = (0, cut // 2)
        splits[P // 2:] += min(2, rows - cut)
        splits[-2:] = (rows - 1, rows)
        splits = np.sort(splits)
        got = run_backward(dy, x, None, mean, rstd, P, k, splits)
        want, off = O.norm_backward(dyd, xd, np.ones(H), host(mean), host(rstd), P, k, splits)
        O.assert_within(host(got[0]), want[0], off[0], "bfloat16", "dx")
        O.assert_within(host(got[1]), want[1], off[1], what="dgamma")
        O.assert_within(host(got[2]), want[2], off[2], what="dbeta")


@pytest.mark.parametrize("H,rows", [(8, 4096), (264, 4096), (8200, 2000)])
def test_empty_processes_cost_no_walk(H, rows):
    """The rows of a million processes (of some ten thousand, where rows are long) belong to the first and the last one, or to the first two:
    the same sums to be made and laid out, so about the same time. One by one, the processes between would take a hundred times as long."""
    import torch
    P, k = (1 << 20, 8) if H == 8 else (1 << 17, 264) if H == 264 else (1 << 13, 8200)
    gen = torch.Generator(device="cuda").manual_seed(H)
    x, dy = (torch.randn(rows, H, generator=gen, device="cuda").bfloat16() for _ in range(2))
    mean, rstd = x.float().mean(1), torch.ones(rows, device="cuda")
    desc = B.make_norm_desc(H, x.dtype, torch.float32, P=P, k=k)
    dx, S = torch.empty_like(x), -(-H // k)
    dg, db = torch.empty(S, P, k, device="cuda"), torch.empty(S, P, k, device="cuda")
    ws = torch.empty(B.ftc_layernorm_workspace_bytes(desc, rows), dtype=torch.uint8, device="cuda")
    far = torch.full((P + 1,), rows // 2 + 1, dtype=torch.int64, device="cuda")
    far[0], far[-1] = 0, rows
    near = torch.full((P + 1,), rows, dtype=torch.int64, device="cuda")
    near[0], near[1] = 0, rows // 2 + 1
    times = {}
    for turn in range(4):
        for name, splits in (("far", far), ("near", near)):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            B.ftc_layernorm_backward(desc, dy, x, None, mean, rstd, splits, dx, dg, db, ws)
            end.record()
            torch.cuda.synchronize()
            times[name] = min(times.get(name, 1e9), begin.elapsed_time(end)) if turn else 1e9
            last = P - 1 if name == "far" else 1
            assert torch.allclose(db[:, last].reshape(-1)[:H], dy[rows // 2 + 1:].float().sum(0), atol=1e-2)
    assert times["far"] < 2 * times["near"] + 0.1, times
