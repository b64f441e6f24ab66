"""Embedding lookup and its gradient against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_22445_b200 import binding as B
from tests import lm_oracle as O

pytestmark = pytest.mark.gpu
DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def tokens_of(rng, n, V, kind="some"):
    t = rng.integers(0, V, n)
    if kind == "one":                     # padding: most positions hold the same token
        t = np.where(rng.random(n) < 0.9, V // 2, t)
    if kind != "all" and n > 2:
        t[rng.random(n) < 0.1] = rng.choice([-1, -100, V, V + 7, 2 ** 31 - 1])
    return t


def wide(values, dtype, pad):
    """The rows as a slice of a wider tensor whose other elements must not matter."""
    t = torch.full((values.shape[0], values.shape[1] + pad), 7.0, dtype=dtype, device="cuda")
    t[:, :values.shape[1]] = torch.from_numpy(values).to(dtype)
    return t[:, :values.shape[1]]


@pytest.mark.parametrize("x,w", [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16")])
@pytest.mark.parametrize("n,V,H,pad,bits", [(1, 1, 1, 0, 64), (5, 7, 3, 1, 32), (64, 100, 256, 0, 64), (33, 64, 264, 8, 32), (130, 50, 301, 0, 64), (17, 9, 4096, 0, 32),
                                            (3, 300, 1025, 3, 64)])
def test_forward(x, w, n, V, H, pad, bits):
    rng = np.random.default_rng(n * H)
    table = wide(rng.standard_normal((V, H)), DT[w], pad)
    tokens = tokens_of(rng, n, V)
    scale = float(np.float32(1.7))
    y = wide(np.zeros((n, H)), DT[x], pad)
    t = torch.from_numpy(tokens).to(torch.int64 if bits == 64 else torch.int32).cuda()
    B.ftc_embedding_forward(B.make_embed_desc(V, H, DT[x], DT[w], scale=scale), t, table, y)
    want = O.embedding_forward(tokens, table.double().cpu().numpy(), scale)
    off = abs(want) * (O.half_step(x) + 2 * O.U32) + O.least(x) * O.half_step(x) * 2
    assert (abs(y.double().cpu().numpy() - want) <= off).all()
    if pad:
        assert (y._base[:, H:] == 7.0).all()


CASES = [  # n, V, H, P, k, kind
    (1, 1, 1, 1, 1, "all"), (1, 300, 8, 1, 8, "all"), (31, 5, 256, 1, 256, "some"), (32, 5, 256, 4, 32, "some"), (33, 5, 256, 4, 32, "some"),
    (700, 3, 40, 3, 8, "one"), (2500, 300, 24, 7, 4, "some"), (2500, 70000, 8, 1, 8, "some"), (900, 20, 301, 5, 7, "one"), (64, 1000, 33, 64, 5, "some"), (1025, 40, 72, 1, 8, "some"), (2048, 30, 40, 3, 8, "one"), (2049, 30, 40, 3, 8, "one"), (2047, 700, 37, 2, 5, "some"),
    (4096, 257, 16, 2, 16, "some"), (4097, 256, 16, 2, 16, "one"), (9001, 255, 520, 1, 520, "one"), (300, 65, 1032, 2, 12, "one"), (50, 17, 13, 3, 1000, "some"),
    (40000, 400, 8, 6, 4, "one"),
]


@pytest.mark.parametrize("x", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,V,H,P,k,kind", CASES)
@pytest.mark.parametrize("ragged", [False, True])
def test_backward(x, n, V, H, P, k, kind, ragged):
    rng = np.random.default_rng(n + H)
    tokens = tokens_of(rng, n, V, kind)
    dy = wide(rng.standard_normal((n, H)), DT[x], 8 if n % 2 else 0)
    splits = None
    if ragged:                            # some processes have none, some tokens have no process
        cuts = np.sort(rng.integers(0, n + 1, P + 1))
        cuts[-1] += rng.integers(0, 2)
        splits = torch.from_numpy(cuts.astype(np.int64)).cuda()
    scale = float(np.float32(2.5))
    desc = B.make_embed_desc(V, H, DT[x], P=P, k=k, scale=scale)
    out = torch.full((-(-V * H // k), P, k), float("nan"), device="cuda")
    ws = torch.full((max(16, B.ftc_embedding_workspace_bytes(desc, n)),), 0xA5, dtype=torch.uint8, device="cuda")
    t = torch.from_numpy(tokens).to(torch.int64 if n % 3 else torch.int32).cuda()
    B.ftc_embedding_backward(desc, t, dy, splits, out, ws)
    want, off = O.embedding_backward(tokens, dy.double().cpu().numpy(), V, scale, P, k, None if splits is None else splits.tolist())
    got = out.double().cpu().numpy()
    assert (abs(got - want) <= off).all()
    again = torch.full_like(out, 3.0)
    B.ftc_embedding_backward(desc, t, dy, splits, again, ws)
    assert torch.equal(out, again)        # the same bits, whatever the workspace held


def test_gradient_is_the_lookups():
    """Against differences of the forward pass: a change of one table element moves the loss by the gradient."""
    rng = np.random.default_rng(3)
    n, V, H, scale = 50, 11, 24, 1.5
    tokens = torch.from_numpy(rng.integers(-1, V, n)).cuda()
    table = torch.from_numpy(rng.integers(-8, 9, (V, H))).float().cuda()           # whole numbers: everything below is exact
    dy = torch.from_numpy(rng.integers(-8, 9, (n, H))).float().cuda()
    desc = B.make_embed_desc(V, H, torch.float32, scale=scale)
    grad = torch.empty(V, 1, H, device="cuda")
    ws = torch.empty(B.ftc_embedding_workspace_bytes(desc, n), dtype=torch.uint8, device="cuda")
    B.ftc_embedding_backward(desc, tokens, dy, None, grad, ws)
    y0, y1 = torch.empty(n, H, device="cuda"), torch.empty(n, H, device="cuda")
    B.ftc_embedding_forward(desc, tokens, table, y0)
    for v, h in ((0, 0), (10, 23), (4, 7)):
        table[v, h] += 2
        B.ftc_embedding_forward(desc, tokens, table, y1)
        assert float((dy * (y1 - y0)).sum()) == 2 * float(grad[v, 0, h])
        table[v, h] -= 2


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_gradient_off_16_bytes(offset):
    rng = np.random.default_rng(offset)
    n, V, H, P, k = 100, 10, 64, 2, 16
    tokens, dy = rng.integers(0, V, n), rng.standard_normal((n, H)).astype(np.float32)
    desc = B.make_embed_desc(V, H, torch.float32, P=P, k=k)
    room = torch.full((V * H * P + 8,), 5.0, device="cuda")
    out = room[offset:offset + V * H * P]
    ws = torch.empty(B.ftc_embedding_workspace_bytes(desc, n), dtype=torch.uint8, device="cuda")
    B.ftc_embedding_backward(desc, torch.from_numpy(tokens).cuda(), torch.from_numpy(dy).cuda(), None, out, ws)
    want, off = O.embedding_backward(tokens, dy.astype(np.float64), V, 1.0, P, k)
    assert (abs(out.double().cpu().numpy().reshape(want.shape) - want) <= off).all()
    assert (room[:offset] == 5).all() and (room[offset + V * H * P:] == 5).all()


def test_no_tokens():
    desc = B.make_embed_desc(9, 8, torch.bfloat16, P=3, k=5)
    out = torch.full((15, 3, 5), 4.0, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    B.ftc_embedding_backward(desc, none, torch.empty(0, 8, dtype=torch.bfloat16, device="cuda"), None, out, None)
    assert (out == 0).all()
    B.ftc_embedding_forward(desc, none, torch.zeros(9, 8, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 8, dtype=torch.bfloat16, device="cuda"))


def test_nan_stays_in_its_row():
    n, V, H = 70, 6, 32
    tokens = torch.arange(n, device="cuda") % V
    dy = torch.ones(n, H, device="cuda")
    dy[8] = float("nan")                  # token 2
    dy[9, 5] = float("inf")               # token 3
    desc = B.make_embed_desc(V, H, torch.float32)
    out = torch.empty(V, 1, H, device="cuda")
    ws = torch.empty(B.ftc_embedding_workspace_bytes(desc, n), dtype=torch.uint8, device="cuda")
    B.ftc_embedding_backward(desc, tokens, dy, None, out, ws)
    assert out[2].isnan().all() and out[3, 0, 5] == float("inf")
    rest = out.clone()
    rest[2] = 12
    rest[3, 0, 5] = 12
    assert ((rest == 11) | (rest == 12)).all()
