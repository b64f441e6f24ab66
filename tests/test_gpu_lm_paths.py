"""The language model operators on the ways through their kernels that many rows, tall matrices and long lists of tokens take, against the
definitions in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_22445_b200 import binding as B
from tests import lm_oracle as O
from tests import test_gpu_embedding as E
from tests import test_gpu_logprobs as L
from tests import test_gpu_muon as M

pytestmark = pytest.mark.gpu


def per_sm(n):
    return n * torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,V,pad", [("six", 5003, 5), ("eight", 5003, 0), ("warps", 1000, 3), ("warps", 2048, 0)])
@pytest.mark.parametrize("top", [0, 5])
def test_many_rows(name, rows, V, pad, top):
    """Blocks of 128 threads a row from six rows an SM on, a warp for each from 32 on, of 65 to 512 vectors."""
    rows = {"six": per_sm(6) + 7, "eight": per_sm(8) + 13, "warps": per_sm(32) + 261}[rows]
    rng = np.random.default_rng(rows + V)
    x = L.logits_of(rng, rows, V, L.DT[name], pad, "masked")
    t, tokens = L.tokens_of(rng, rows, V, 64)
    desc, (given, entropy, lse), best, which = L.forward(x, tokens, 0.8, top)
    scale = float(np.float32(0.8))
    exact = x.double().cpu().numpy()
    w_lse, w_given, w_entropy, w_best, w_which, spread = O.logprobs(exact, t, scale, top)
    s_off = O.sum_off(spread, V)

    def close(got, want, off):
        got = got.double().cpu().numpy()
        same = (got == want) | (np.isnan(got) & np.isnan(want))
        with np.errstate(invalid="ignore"):
            assert (same | (abs(got - want) <= off)).all()

    with np.errstate(invalid="ignore"):
        close(lse, w_lse, s_off + 4 * O.U32 * (np.where(np.isfinite(w_lse), abs(w_lse), 0) + spread))
        close(given, w_given, s_off + 4 * O.U32 * np.where(np.isfinite(w_given), abs(w_given), 0) + 4 * O.U32)
        close(entropy, w_entropy, 4 * s_off * (1 + spread))
        if top:
            assert (which.cpu().numpy() == w_which).all()
            close(best, w_best, s_off[:, None] + 4 * O.U32 * (1 + np.where(np.isfinite(w_best), abs(w_best), 0)))
    if top:
        return
    keep = np.arange(rows) != 2           # the row at the type's lowest value: its p is not what lse in float32 says
    up, de = (torch.from_numpy(rng.standard_normal(rows)).float().cuda() for _ in range(2))
    d = torch.full((rows, V + pad), 7.0, dtype=L.DT[name], device="cuda")[:, :V]
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, up, de, d)
    want, off = O.logprobs_backward(exact[keep], t[keep], scale, lse.double().cpu().numpy()[keep], entropy.double().cpu().numpy()[keep], up.double().cpu().numpy()[keep],
                                    de.double().cpu().numpy()[keep])
    off = off + (abs(want) + off) * O.half_step(name) + O.least(name) * O.half_step(name) * 2
    assert (abs(d.double().cpu().numpy()[keep] - want) <= off).all()
    assert torch.isfinite(d[2]).all()
    if pad:
        assert (d._base[:, V:] == 7.0).all()


@pytest.mark.parametrize("products", [16, 32])
@pytest.mark.parametrize("p,master", [("float32", False), ("bfloat16", True), ("float16", False)])
@pytest.mark.parametrize("g,k,lost", [("bfloat16", 0, 0), ("float32", 32, 0.05), ("float32", 7, 0.3)])
def test_tall_matrices_of_whole_blocks(products, p, master, g, k, lost):
    rng = np.random.default_rng(k + 9)
    made = [M.make(rng, r, c, p, g, master, k, lost, lr_scale=s, decay=0.05) for r, c, s in ((384, 128, 1.0), (640, 256, 0.5), (256, 128, 1.0), (128, 640, 2.0))]
    entries, matrices = [m[0] for m in made], [m[1] for m in made]
    _, views = M.step(entries, matrices, products, scale=0.5)
    M.check(matrices, views, products, scale=0.5)


@pytest.mark.parametrize("n,V,H,P,k,ragged", [(5000, 300, 8, 1500, 4, True), (5000, 300, 8, 1500, 4, False), (40000, 200, 8, 3, 8, True), (40000, 70000, 8, 1, 8, False),
                                              (32768, 300, 8, 2, 8, True), (32769, 300, 8, 2, 8, True), (33000, 90000, 16, 1, 16, False), (70001, 255, 8, 1025, 4, True)])
def test_long_lists_of_tokens(n, V, H, P, k, ragged):
    """More processes than the sort keeps split points of, lists that leave shared memory, one to three passes."""
    rng = np.random.default_rng(n + V)
    tokens = E.tokens_of(rng, n, V, "one" if V < 300 else "some")
    dy = E.wide(rng.standard_normal((n, H)), torch.float32, 0)
    splits = None
    if ragged:
        cuts = np.sort(rng.integers(0, n + 1, P + 1))
        splits = torch.from_numpy(cuts.astype(np.int64)).cuda()
    desc = B.make_embed_desc(V, H, torch.float32, P=P, k=k, scale=2.5)
    out = torch.full((-(-V * H // k), P, k), float("nan"), device="cuda")
    ws = torch.full((B.ftc_embedding_workspace_bytes(desc, n),), 0xA5, dtype=torch.uint8, device="cuda")
    B.ftc_embedding_backward(desc, torch.from_numpy(tokens).cuda(), dy, splits, out, ws)
    want, off = O.embedding_backward(tokens, dy.double().cpu().numpy(), V, 2.5, P, k, None if splits is None else splits.tolist())
    assert (abs(out.double().cpu().numpy() - want) <= off).all()
