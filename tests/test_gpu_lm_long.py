"""Offsets beyond 2^32 elements, and large matrices, against plain arithmetic on the rows that lie there."""
import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import lm_oracle as O

pytestmark = pytest.mark.gpu


def test_embedding_beyond_32_bits():
    import torch
    V, H, n = 4300000, 1024, 3000                    # 4.4e9 elements
    table = torch.zeros(V, H, dtype=torch.bfloat16, device="cuda")
    table[-5:] = torch.arange(5, device="cuda").bfloat16()[:, None] + 1
    tokens = torch.arange(n, device="cuda") % 5 + V - 5
    y = torch.zeros(n, H, dtype=torch.bfloat16, device="cuda")
    desc = B.make_embed_desc(V, H, torch.bfloat16)
    B.ftc_embedding_forward(desc, tokens, table, y)
    assert torch.equal(y, ((torch.arange(n, device="cuda") % 5 + 1).bfloat16()[:, None]).expand(n, H))
    del table
    out = torch.full((V, 1, H), 7.0, device="cuda")
    ws = torch.empty(B.ftc_embedding_workspace_bytes(desc, n), dtype=torch.uint8, device="cuda")
    B.ftc_embedding_backward(desc, tokens, torch.ones(n, H, dtype=torch.bfloat16, device="cuda"), None, out, ws)
    assert (out[-5:] == n / 5).all()
    for part in out[:-5].split(1 << 19):
        assert not part.any()
    # few tokens, two processes
    few = 7
    desc = B.make_embed_desc(V // 2, H, torch.bfloat16, P=2, k=1)
    out = out.view(-1)[:V // 2 * H * 2].view(V // 2 * H, 2, 1)
    B.ftc_embedding_backward(desc, torch.full((few,), V // 2 - 1, device="cuda"), torch.ones(few, H, dtype=torch.bfloat16, device="cuda"), None, out, ws)
    assert (out[-H:, 0] == 3).all() and (out[-H:, 1] == 4).all() and not out[:-H].view(-1)[-(1 << 28):].any()


def test_logprobs_beyond_32_bits():
    import torch
    rows, V = 34000, 130000                          # 4.4e9 elements
    x = torch.zeros(rows, V, dtype=torch.float16, device="cuda")
    x[-3:] = torch.randn(3, V, device="cuda").half() * 3
    tokens = torch.full((rows,), V - 1, device="cuda")
    logprob, entropy, lse = (torch.zeros(rows, device="cuda") for _ in range(3))
    top, which = torch.zeros(rows, 2, device="cuda"), torch.zeros(rows, 2, dtype=torch.int32, device="cuda")
    desc = B.make_logprob_desc(V, torch.float16, top=2)
    B.ftc_token_logprobs(desc, x, tokens, logprob, entropy, lse, top, which)
    want = torch.log_softmax(x[-3:].double(), 1)
    assert (logprob[-3:] - want[:, -1]).abs().max() < 1e-5 and (top[-3:].double() - want.topk(2, 1).values).abs().max() < 1e-5
    assert (entropy[:-3] - entropy[0]).abs().max() == 0 and (which[0] == torch.tensor([0, 1], device="cuda")).all()
    ones = torch.ones(rows, device="cuda")
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, ones, None, x)          # in place
    want = -want.exp()
    want[:, -1] += 1
    assert (x[-3:].double() - want).abs().max() < 1e-3
    assert (x[1].float() - x[-4].float()).abs().max() == 0 and x[5, -1] > 0.99


@pytest.mark.parametrize("rows,cols,products", [(1200, 5000, 16), (7001, 1003, 16), (1536, 1536, 32)])
def test_large_matrices(rows, cols, products):
    """A matrix of many tiles against the definition and the bound that goes with it (sums of thousands of products are off by as many roundings as
    there are sixteens of them)."""
    import torch
    rng = np.random.default_rng(1)
    m = min(rows, cols)
    g = rng.standard_normal((rows, cols)) + 4 * rng.standard_normal((rows, 1)) * rng.standard_normal((1, cols)) / m ** 0.5
    if rows == cols:                                  # a square one has small singular values: lifted
        g += 2 * m ** 0.5 * np.eye(m)
    g = g.astype(np.float32)
    w, grad = torch.zeros(rows, cols, device="cuda"), torch.from_numpy(g).cuda()
    plan = B.make_muon_plan([B.make_matrix(w, grad)])
    momentum = torch.zeros(plan.blocks * 256, device="cuda")
    ws = torch.empty(B.ftc_muon_workspace_bytes(plan, products), dtype=torch.uint8, device="cuda")
    B.ftc_muon_step(B.make_muon(1.0, nesterov=False, products=products), plan, momentum, None, ws)
    _, m1, x, off = O.muon(np.zeros((rows, cols)), np.zeros((rows, cols)), g.astype(np.float64), np.ones((rows, cols), bool), 1.0, 1.0, 0.0, 0.95, False, 1e-7, 5, products)
    assert np.linalg.norm(w.double().cpu().numpy() + x) <= off + 4 * O.U32 * np.linalg.norm(x) and off < 0.2 * np.linalg.norm(x)
    assert torch.equal(momentum[:rows * cols].view(rows, cols), grad)
