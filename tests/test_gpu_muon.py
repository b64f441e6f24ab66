"""The orthogonalised update of many matrices against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_22445_b200 import binding as B
from tests import lm_oracle as O

pytestmark = pytest.mark.gpu
DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def make(rng, rows, cols, p="float32", g="float32", master=False, k=0, lost=0.0, lr_scale=1.0, decay=0.0):
    """One matrix: its tensors, and what the definition gets."""
    n = rows * cols
    grad = torch.from_numpy(rng.standard_normal((rows, cols)) * 0.1).to(DT[g]).cuda()
    weights = torch.from_numpy(rng.standard_normal((rows, cols)) * 0.5).float().cuda()
    param = weights.to(DT[p])
    m = rng.standard_normal((rows, cols)).astype(np.float32)
    status, mean, there = None, grad.double().cpu().numpy(), np.ones((rows, cols), bool)
    if k:
        messages = -(-n // k)
        st = np.zeros((messages, 4), np.int32)
        gone = rng.random(messages) < lost
        st[:, 0] = np.where(gone, 2 | 0xFF00 | 1 << 16, 1 << 16)
        st[:, 1] = np.where(gone, rng.integers(0, 2, messages) * 9, rng.integers(60, 65, messages))
        status = torch.from_numpy(st).cuda()
        each = np.repeat(st[:, 1], k)[:n].reshape(rows, cols)
        there = ~np.repeat(gone, k)[:n].reshape(rows, cols)
        mean = np.where(there, mean / np.maximum(each, 1), 0)
    entry = B.make_matrix(param, grad, master=weights if master else None, status=status, k=k, lr_scale=lr_scale, weight_decay=decay)
    start = (weights if master else param).double().cpu().numpy()
    return entry, dict(param=param, master=weights if master else None, m=m, start=start, mean=mean, there=there, lr_scale=lr_scale, decay=decay)


def momentum_of(plan, matrices):
    flat = torch.zeros(plan.blocks * B.FTC_STATE_BLOCK, device="cuda")
    at, views = 0, []
    for d in matrices:
        n = d["m"].size
        flat[at:at + n] = torch.from_numpy(d["m"].reshape(-1)).cuda()
        views.append(flat[at:at + n])
        at += -(-n // B.FTC_STATE_BLOCK) * B.FTC_STATE_BLOCK
    return flat, views


def step(entries, matrices, products, lr=0.1, scale=None, steps=5, nesterov=True, calls=1):
    plan = B.make_muon_plan(entries)
    flat, views = momentum_of(plan, matrices)
    hyper = B.make_muon(lr, 0.9, 1e-7, steps, nesterov, products)
    ws = torch.full((B.ftc_muon_workspace_bytes(plan, products),), 0x7F, dtype=torch.uint8, device="cuda")
    for _ in range(calls):
        B.ftc_muon_step(hyper, plan, flat, None if scale is None else torch.tensor([scale], device="cuda"), ws)
    assert int(ws[:4].view(torch.int32)) == 0
    return flat, views


def check(matrices, views, products, lr=0.1, scale=1.0, steps=5, nesterov=True):
    f = lambda v: float(np.float32(v))  # noqa: E731
    for d, view in zip(matrices, views):
        want, m1, x, off = O.muon(d["start"], d["m"].astype(np.float64), d["mean"] * f(scale), d["there"], f(lr), d["lr_scale"], f(d["decay"]), f(0.9),
                                  nesterov, f(1e-7), steps, products)
        got = view.double().cpu().numpy().reshape(want.shape)
        size = abs(d["m"]) + abs(d["mean"] * scale)
        assert (abs(got - m1) <= 4 * O.U32 * size).all()
        new = d["master"] if d["master"] is not None else d["param"]
        l = f(lr) * d["lr_scale"]
        name = str(new.dtype).replace("torch.", "")
        diff = np.linalg.norm(new.double().cpu().numpy() - want)
        room = l * off + (O.half_step(name) + 4 * O.U32) * np.linalg.norm(want) + 4 * O.U32 * np.linalg.norm(d["start"])
        assert diff <= room, (diff, room)
        if d["master"] is not None:
            assert torch.equal(d["param"], d["master"].to(d["param"].dtype))
        if off and np.linalg.norm(l * x) > 0:
            assert l * off < 0.5 * np.linalg.norm(l * x)          # the bound says something


SHAPES = [(1, 1), (1, 7), (9, 1), (8, 8), (16, 64), (64, 16), (63, 65), (100, 130), (128, 128), (129, 127), (130, 300), (256, 256), (300, 70), (257, 513), (640, 200),
          (100, 256), (128, 257), (512, 90), (70, 449), (128, 512), (128, 513), (513, 128)]


@pytest.mark.parametrize("products", [16, 32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_one_matrix(products, rows, cols):
    rng = np.random.default_rng(rows * 1000 + cols)
    entry, d = make(rng, rows, cols, decay=0.1)
    _, views = step([entry], [d], products)
    check([d], views, products)


@pytest.mark.parametrize("products", [16, 32])
@pytest.mark.parametrize("p,master", [("float32", False), ("bfloat16", True), ("float16", True), ("bfloat16", False), ("float16", False)])
@pytest.mark.parametrize("g,k,lost", [("bfloat16", 0, 0), ("float16", 0, 0), ("float32", 32, 0.05), ("float32", 7, 0.3), ("float32", 1, 0.1)])
def test_many(products, p, master, g, k, lost):
    rng = np.random.default_rng(k + 5)
    made = [make(rng, r, c, p, g, master, k, lost, lr_scale=s, decay=0.05) for r, c, s in ((70, 50, 1.0), (33, 200, 0.5), (128, 384, 2.0), (5, 3, 1.0), (200, 131, 1.0), (310, 90, 1.0))]
    entries, matrices = [m[0] for m in made], [m[1] for m in made]
    _, views = step(entries, matrices, products, scale=0.5)
    check(matrices, views, products, scale=0.5)


@pytest.mark.parametrize("steps", [1, 2, 8])
@pytest.mark.parametrize("nesterov", [True, False])
def test_steps(steps, nesterov):
    rng = np.random.default_rng(steps)
    entry, d = make(rng, 90, 150)
    _, views = step([entry], [d], 32, steps=steps, nesterov=nesterov)
    check([d], views, 32, steps=steps, nesterov=nesterov)


def test_nothing_delivered_stays():
    rng = np.random.default_rng(1)
    gone, a = make(rng, 40, 60, k=16, lost=1.1, decay=0.1)
    some, b = make(rng, 40, 60, k=16, lost=0.5, decay=0.1)
    before = a["param"].clone()
    _, views = step([gone, some], [a, b], 16)
    assert torch.equal(a["param"], before)
    assert torch.equal(views[0].cpu(), torch.from_numpy(a["m"].reshape(-1)))
    check([b], views[1:], 16)


@pytest.mark.parametrize("scale", [float("nan"), float("inf")])
def test_a_clip_factor_that_is_not_finite_changes_nothing(scale):
    rng = np.random.default_rng(2)
    entry, d = make(rng, 40, 60)
    before = d["param"].clone()
    _, views = step([entry], [d], 16, scale=scale)
    assert torch.equal(d["param"], before) and torch.equal(views[0].cpu(), torch.from_numpy(d["m"].reshape(-1)))


def test_nan_and_zeros():
    """A matrix that meets NaN has NaN in its weights, its neighbour none; one without momentum and gradient only decays."""
    rng = np.random.default_rng(4)
    made = [make(rng, 50, 70, decay=0.5) for _ in range(3)]
    made[0][0][1][1][3, 4] = float("nan")
    made[2][0][1][1].zero_()
    made[2][1]["m"][:] = 0
    _, views = step([m[0] for m in made], [m[1] for m in made], 16)
    assert made[0][1]["param"].isnan().any()
    check([made[1][1]], views[1:2], 16)
    want = made[2][1]["start"] * (1 - float(np.float32(0.1)) * 0.5)
    assert (abs(made[2][1]["param"].double().cpu().numpy() - want) <= 4 * O.U32 * abs(want)).all()


def test_momentum_behind_a_matrix_is_left():
    rng = np.random.default_rng(6)
    made = [make(rng, 9, 11), make(rng, 5, 60)]
    flat, _ = step([m[0] for m in made], [m[1] for m in made], 16)
    assert (flat[99:256] == 0).all() and (flat[556:] == 0).all()


def test_same_bits_again():
    rng = np.random.default_rng(7)
    out = []
    for _ in range(2):
        rng = np.random.default_rng(7)
        made = [make(rng, 300, 500, "bfloat16", "bfloat16", True), make(rng, 260, 140)]
        flat, _ = step([m[0] for m in made], [m[1] for m in made], 16, calls=2)
        out.append([flat] + [m[1]["param"] for m in made])
    assert all(torch.equal(a, b) for a, b in zip(*out))
