"""Layer norm forward and backward on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import train_oracle as O

pytestmark = pytest.mark.gpu

TYPES = [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16")]
SHAPES = [(1, 1), (1, 7), (3, 31), (2, 32), (5, 33), (4, 64), (17, 127), (9, 200), (300, 256), (33, 511), (6, 520), (7, 1000), (129, 1024), (3, 1367),
          (5, 2050), (11, 4096), (4, 5000), (2, 8192), (3, 10007), (2, 16384), (1, 16400), (2, 40000)]


def make(rng, rows, H, dtype, pad=0, offset=0, spread=1.0):
    """A [rows][H] device tensor of dtype (rows `pad` elements apart, `offset` elements into its storage) and its values."""
    import torch
    dt = getattr(torch, dtype)
    flat = torch.full((rows * (H + pad) + offset + 8,), 77.0, dtype=dt, device="cuda")
    t = flat[offset:offset + rows * (H + pad)].view(rows, H + pad)[:, :H]
    t.copy_(torch.from_numpy(rng.standard_normal((rows, H)) * spread + 0.25 * rng.standard_normal(H)))
    return t, t.double().cpu().numpy()


def vector(rng, H, dtype, mean, offset=0):
    import torch
    t = torch.zeros(H + offset, dtype=getattr(torch, dtype), device="cuda")[offset:]
    t.copy_(torch.from_numpy(mean + 0.3 * rng.standard_normal(H)))
    return t, t.double().cpu().numpy()


def run_forward(x, gamma, beta, eps, wdtype, y=None, stream=None):
    import torch
    rows, H = x.shape
    y = torch.full((rows, H), 55.0, dtype=x.dtype, device="cuda") if y is None else y
    mean, rstd = torch.full((rows,), 55.0, device="cuda"), torch.full((rows,), 55.0, device="cuda")
    desc = B.make_norm_desc(H, x.dtype, B._float_code(wdtype), eps=eps)
    B.ftc_layernorm_forward(desc, x, gamma, beta, y, mean, rstd, stream=stream)
    return y, mean, rstd


def run_backward(dy, x, gamma, mean, rstd, P, k, splits=None, wdtype="float32", dx=None, weights=True, stream=None):
    import torch
    rows, H = x.shape
    desc = B.make_norm_desc(H, x.dtype, B._float_code(wdtype), P=P, k=k)
    S = -(-H // k)
    dx = torch.full((rows, H), 55.0, dtype=x.dtype, device="cuda") if dx is None else dx
    dg, db = (torch.full((S, P, k), 55.0, device="cuda") for _ in range(2)) if weights else (None, None)
    ws = torch.full((max(16, B.ftc_layernorm_workspace_bytes(desc, rows)),), 0xFF, dtype=torch.uint8, device="cuda")     # NaN patterns
    d_splits = None if splits is None else torch.tensor(splits, dtype=torch.int64, device="cuda")
    B.ftc_layernorm_backward(desc, dy, x, gamma, mean, rstd, d_splits, dx, dg, db, ws, stream=stream)
    return dx, dg, db


def host(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,H", SHAPES)
def test_forward(rows, H, dtype, wdtype):
    rng = np.random.default_rng([rows, H, 1])
    for pad, offset in ((0, 0), (8, 8), (5, 3)):
        x, xd = make(rng, rows, H, dtype, pad, offset)
        gamma, gd = vector(rng, H, wdtype, 1.0, offset)
        beta, bd = vector(rng, H, wdtype, 0.0, offset)
        out, _ = make(rng, rows, H, dtype, 2 * pad, offset)
        got = run_forward(x, gamma, beta, 1e-5, wdtype, y=out)
        want, off = O.norm_forward(xd, gd, bd, 1e-5)
        O.assert_within(host(got[0]), want[0], off[0], dtype, f"y pad {pad}")
        O.assert_within(host(got[1]), want[1], off[1], what="mean")
        O.assert_within(host(got[2]), want[2], off[2], what="rstd")


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("H", [2, 24, 32, 40, 57, 64, 72, 97, 128, 130, 136, 193, 248, 256])
def test_forward_of_narrow_rows(H, dtype, wdtype):
    """Rows that share a warp: as many as end within its last round, and more than the GPU holds; nothing between the rows is written."""
    rng = np.random.default_rng([H, 9])
    for rows, pad, offset in ((1, 0, 0), (75, 8, 8), (75, 1, 1), (40003, 0, 0), (9001, 3, 2)):
        x, xd = make(rng, rows, H, dtype, pad, offset)
        gamma, gd = vector(rng, H, wdtype, 1.0, offset)
        beta, bd = vector(rng, H, wdtype, 0.0, offset)
        out, _ = make(rng, rows, H, dtype, pad, offset)
        got = run_forward(x, gamma, beta, 1e-5, wdtype, y=out)
        want, off = O.norm_forward(xd, gd, bd, 1e-5)
        O.assert_within(host(got[0]), want[0], off[0], dtype, f"y of {rows} rows")
        O.assert_within(host(got[1]), want[1], off[1], what="mean")
        O.assert_within(host(got[2]), want[2], off[2], what="rstd")
        if pad:
            assert (out.as_strided((rows - 1, pad), (H + pad, 1), offset + H) == 77.0).all() if rows > 1 else True


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,H", SHAPES)
def test_backward(rows, H, dtype, wdtype):
    rng = np.random.default_rng([rows, H, 2])
    for P, k, ragged, pad, offset in ((1, H, False, 0, 0), (3, 16, False, 8, 8), (5, 7, True, 5, 3)):
        x, xd = make(rng, rows, H, dtype, pad, offset)
        dy, dyd = make(rng, rows, H, dtype, 2 * pad, offset, 0.3)
        gamma, gd = vector(rng, H, wdtype, 1.0, offset)
        _, mean, rstd = run_forward(x, gamma, None, 1e-5, wdtype)
        splits = None
        if ragged:
            splits = np.concatenate([[0], np.sort(rng.integers(0, rows + 1, P - 1)), [rows]])
        dx, _ = make(rng, rows, H, dtype, pad, offset)
        got = run_backward(dy, x, gamma, mean, rstd, P, k, splits, wdtype, dx=dx)
        want, off = O.norm_backward(dyd, xd, gd, host(mean), host(rstd), P, k, splits)
        O.assert_within(host(got[0]), want[0], off[0], dtype, f"dx P {P}")
        O.assert_within(host(got[1]), want[1], off[1], what=f"dgamma P {P}")
        O.assert_within(host(got[2]), want[2], off[2], what=f"dbeta P {P}")


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("H", [2, 24, 32, 40, 57, 64, 72, 97, 128, 136, 201, 256])
def test_backward_of_narrow_rows(H, dtype, wdtype):
    """Rows that share a warp: processes that begin and end inside a round of rows, that have none, that write their messages themselves."""
    rng = np.random.default_rng([H, 11])
    for rows, P, k, ragged, pad, offset in ((1, 1, H, False, 0, 0), (333, 200, 7, True, 8, 8), (333, 111, 4, False, 1, 1), (20011, 5, 32, True, 0, 0), (9001, 3000, 8, True, 3, 2)):
        x, xd = make(rng, rows, H, dtype, pad, offset)
        dy, dyd = make(rng, rows, H, dtype, 2 * pad, offset, 0.3)
        gamma, gd = vector(rng, H, wdtype, 1.0, offset)
        _, mean, rstd = run_forward(x, gamma, None, 1e-5, wdtype)
        splits = np.sort(rng.integers(0, rows + 1, P + 1)) if ragged else None       # some rows are nobody's
        dx, _ = make(rng, rows, H, dtype, pad, offset)
        got = run_backward(dy, x, gamma, mean, rstd, P, k, splits, wdtype, dx=dx)
        want, off = O.norm_backward(dyd, xd, gd, host(mean), host(rstd), P, k, splits)
        O.assert_within(host(got[0]), want[0], off[0], dtype, f"dx of {rows} rows")
        O.assert_within(host(got[1]), want[1], off[1], what=f"dgamma of {rows} rows")
        O.assert_within(host(got[2]), want[2], off[2], what=f"dbeta of {rows} rows")
        if pad:
            assert (dx.as_strided((rows - 1, pad), (H + pad, 1), offset + H) == 77.0).all()
        alone = run_backward(dy, x, gamma, mean, rstd, P, k, splits, wdtype, weights=False)[0]
        assert (alone == got[0]).all()


@pytest.mark.parametrize("rows,H,P,k,splits", [
    (1000, 96, 64, 32, None), (700, 260, 1024, 4, None), (2000, 128, 3, 128, [0, 0, 2000, 2000]), (2000, 128, 4, 32, [100, 100, 900, 1500, 1900]),
    (900, 64, 3, 16, [0, 10, 5000, 6000]), (600, 1032, 600, 8, None), (5000, 40, 2, 64, [0, 1, 5000]), (64, 512, 8, 16, None), (1, 64, 2, 16, [0, 0, 1])])
def test_rows_of_processes(rows, H, P, k, splits):
    """Processes without rows, rows that nobody holds, splits behind the last row, more processes than rows."""
    rng = np.random.default_rng([rows, H, P])
    x, xd = make(rng, rows, H, "bfloat16")
    dy, dyd = make(rng, rows, H, "bfloat16")
    gamma, gd = vector(rng, H, "float32", 1.0)
    _, mean, rstd = run_forward(x, gamma, None, 1e-5, "float32")
    got = run_backward(dy, x, gamma, mean, rstd, P, k, splits)
    want, off = O.norm_backward(dyd, xd, gd, host(mean), host(rstd), P, k, splits)
    O.assert_within(host(got[0]), want[0], off[0], "bfloat16", "dx")
    O.assert_within(host(got[1]), want[1], off[1], what="dgamma")
    O.assert_within(host(got[2]), want[2], off[2], what="dbeta")
    again = run_backward(dy, x, gamma, mean, rstd, P, k, splits)
    for a, b in zip(got, again):
        assert (a == b).all()                                  # a fixed order of additions: the same bits


@pytest.mark.parametrize("H", [24, 513, 2048, 9000])
def test_differences(H):
    """The gradients against central differences of the forward pass's definition, along random directions."""
    import torch
    rng = np.random.default_rng(H)
    rows = 6
    x, xd = make(rng, rows, H, "float32")
    dy, dyd = make(rng, rows, H, "float32")
    gamma, gd = vector(rng, H, "float32", 1.0)
    beta, bd = vector(rng, H, "float32", 0.0)
    _, mean, rstd = run_forward(x, gamma, beta, 1e-5, "float32")
    dx, dg, db = (host(t) for t in run_backward(dy, x, gamma, mean, rstd, 1, H))

    def loss(x, g, b):
        return (dyd * O.norm_forward(x, g, b, 1e-5)[0][0]).sum()

    h = 1e-5                                    # error of a central difference: O(h^2) of the loss's size, rounding 2^-53 / h
    for grad, at in ((dx, 0), (dg.ravel()[:H], 1), (db.ravel()[:H], 2)):
        args = [xd, gd, bd]
        way = rng.standard_normal(args[at].shape)
        lo, hi = list(args), list(args)
        lo[at], hi[at] = args[at] - h * way, args[at] + h * way
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        room = 1e-5 * np.abs(grad * way).sum() + 1e-5
        assert abs(slope - (grad * way).sum()) <= room
    assert torch.isfinite(dy).all()


def test_rows_without_variance_and_large_values():
    """Constant rows (rstd = 1/sqrt(eps)), a large common offset, float16 values near its end, rows with NaN or infinity beside clean ones."""
    import torch
    H = 768 + 4
    x = torch.zeros(6, H, device="cuda")
    x[1] = 3.0
    x[2] = 1e4 + torch.arange(H, device="cuda") % 2
    x[3] = torch.linspace(-6e4, 6e4, H, device="cuda")
    x[4, 5] = float("nan")
    x[5, 6] = float("inf")
    y, mean, rstd = run_forward(x, None, None, 1e-5, "float32")
    xd = host(x)[:4]
    want, off = O.norm_forward(xd, np.ones(H), np.zeros(H), 1e-5)
    O.assert_within(host(y)[:4], want[0], off[0], what="y")
    O.assert_within(host(rstd)[:4], want[2], off[2], what="rstd")
    assert torch.isnan(y[4:]).all()
    y16 = run_forward(x[:4].half(), None, None, 1e-5, "float16")[0]
    want, off = O.norm_forward(host(x[:4].half()), np.ones(H), np.zeros(H), 1e-5)
    O.assert_within(host(y16), want[0], off[0], "float16", "y16")


@pytest.mark.parametrize("dtype,rows,H", [("bfloat16", 70, 1024), ("float32", 9, 333), ("float16", 5, 20000)])
def test_in_place_and_optional_outputs(dtype, rows, H):
    import torch
    rng = np.random.default_rng(H)
    x, _ = make(rng, rows, H, dtype)
    dy, _ = make(rng, rows, H, dtype)
    gamma, _ = vector(rng, H, "float32", 1.0)
    y, mean, rstd = run_forward(x, gamma, None, 1e-5, "float32")
    desc = B.make_norm_desc(H, x.dtype, torch.float32)
    same = x.clone()
    B.ftc_layernorm_forward(desc, same, gamma, None, same, None, None)            # y over x, no statistics
    assert (same == y).all()
    dx, dg, db = run_backward(dy, x, gamma, mean, rstd, 1, H)
    over = dy.clone()
    run_backward(over, x, gamma, mean, rstd, 1, H, dx=over)                       # dx over dy
    assert (over == dx).all()
    over = x.clone()
    got = run_backward(dy, over, gamma, mean, rstd, 1, H, dx=over)                # dx over x
    assert (over == dx).all() and (got[1] == dg).all() and (got[2] == db).all()
    alone = run_backward(dy, x, gamma, mean, rstd, 1, H, weights=False)[0]
    assert (alone == dx).all()
    ws = torch.empty(B.ftc_layernorm_workspace_bytes(desc, rows), dtype=torch.uint8, device="cuda")
    only = torch.full_like(dg, 9.0)
    B.ftc_layernorm_backward(desc, dy, x, gamma, mean, rstd, None, None, None, only, ws)   # dbeta alone
    assert (only == db).all()


def test_no_rows():
    import torch
    for H in (16, 1000):
        x = torch.empty(0, H, dtype=torch.bfloat16, device="cuda")
        stat = torch.empty(0, device="cuda")
        y, _, _ = run_forward(x, None, None, 1e-5, "float32")
        assert y.shape == (0, H)
        _, dg, db = run_backward(x, x, None, stat, stat, 3, 8)
        assert (dg == 0).all() and (db == 0).all()


def test_wide_strides_and_another_stream():
    """Rows far apart (offsets beyond 2^31 elements), on a stream that is not the current one."""
    import torch
    rows, H, far = 5, 520, (1 << 29) + 24
    side = torch.cuda.Stream()
    rng = np.random.default_rng(3)
    wide = torch.zeros(rows * far, dtype=torch.bfloat16, device="cuda")
    x = wide.as_strided((rows, H), (far, 1))
    src, xd = make(rng, rows, H, "bfloat16")
    x.copy_(src)
    gamma, gd = vector(rng, H, "float32", 1.0)
    torch.cuda.synchronize()
    y, mean, rstd = run_forward(x, gamma, None, 1e-5, "float32", y=x, stream=side)
    side.synchronize()
    want, off = O.norm_forward(xd, gd, np.zeros(H), 1e-5)
    O.assert_within(host(y), want[0], off[0], "bfloat16", "y")
    x.copy_(src)
    torch.cuda.synchronize()
    got = run_backward(x, x, gamma, mean, rstd, 2, 8, stream=side, dx=x)
    side.synchronize()
    want, off = O.norm_backward(xd, xd, gd, host(mean), host(rstd), 2, 8, None)
    O.assert_within(host(got[0]), want[0], off[0], "bfloat16", "dx")
    O.assert_within(host(got[1]), want[1], off[1], what="dgamma")


def test_workspace_is_wanted():
    import torch
    x = torch.zeros(4, 64, device="cuda")
    stat = torch.zeros(4, device="cuda")
    out = torch.zeros(64, device="cuda")
    desc = B.make_norm_desc(64, torch.float32)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    for ws in (None, small):
        assert B.ftc_layernorm_backward(desc, x, x, None, stat, stat, None, None, out, out, ws, check=False) == B.FTC_EWORKSPACE
    with pytest.raises(B.FtcError):
        B.ftc_layernorm_backward(desc, x, x, None, stat, stat, None, None, out, out, None)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,H,P,k", [(64, 512, 8, 16), (5, 96, 8, 32), (700, 260, 700, 4), (3000, 72, 2999, 7), (4096, 1024, 1024, 32), (2500, 33, 1300, 5), (8, 4099, 1, 4099),
                                        (600, 8192, 300, 128), (7, 1024, 1, 1000), (40, 24, 5, 24)])
def test_one_group_for_each_process(rows, H, P, k, dtype):
    """Many processes, or few rows each: every process's sums go straight to its messages, fill and empty processes included."""
    rng = np.random.default_rng([rows, H, P, 4])
    for pad, offset in ((0, 0), (3, 1)):
        x, xd = make(rng, rows, H, dtype, pad, offset)
        dy, dyd = make(rng, rows, H, dtype, pad, offset)
        gamma, gd = vector(rng, H, "float32", 1.0)
        _, mean, rstd = run_forward(x, gamma, None, 1e-5, "float32")
        got = run_backward(dy, x, gamma, mean, rstd, P, k)
        want, off = O.norm_backward(dyd, xd, gd, host(mean), host(rstd), P, k, None)
        O.assert_within(host(got[0]), want[0], off[0], dtype, "dx")
        O.assert_within(host(got[1]), want[1], off[1], what="dgamma")
        O.assert_within(host(got[2]), want[2], off[2], what="dbeta")
        splits = [p * rows // P for p in range(P + 1)]
        other = run_backward(dy, x, gamma, mean, rstd, P, k, splits)              # the same shares, given
        O.assert_within(host(other[1]), want[1], off[1], what="dgamma of splits")


@pytest.mark.parametrize("rows,H,P", [(2500, 1025, 3), (3000, 4424, 2), (1800, 6001, 1), (700, 8191, 5), (9000, 200, 16), (40, 12000, 3), (50, 12001, 40), (30, 33000, 2)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_rows(rows, H, P, dtype):
    """Rows enough for every block to walk several, two at a time; rows wider than a group holds."""
    rng = np.random.default_rng([rows, H, P, 5])
    x, xd = make(rng, rows, H, dtype)
    dy, dyd = make(rng, rows, H, dtype)
    gamma, gd = vector(rng, H, "float32", 1.0)
    beta, bd = vector(rng, H, "float32", 0.0)
    got = run_forward(x, gamma, beta, 1e-5, "float32")
    want, off = O.norm_forward(xd, gd, bd, 1e-5)
    O.assert_within(host(got[0]), want[0], off[0], dtype, "y")
    O.assert_within(host(got[1]), want[1], off[1], what="mean")
    O.assert_within(host(got[2]), want[2], off[2], what="rstd")
    _, mean, rstd = got
    got = run_backward(dy, x, gamma, mean, rstd, P, 32)
    want, off = O.norm_backward(dyd, xd, gd, host(mean), host(rstd), P, 32, None)
    O.assert_within(host(got[0]), want[0], off[0], dtype, "dx")
    O.assert_within(host(got[1]), want[1], off[1], what="dgamma")
    O.assert_within(host(got[2]), want[2], off[2], what="dbeta")
