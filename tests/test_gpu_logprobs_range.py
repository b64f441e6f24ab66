"""Token log probabilities and their gradient where lse leaves float32, or says little of the probabilities in it, against the definition
in 64 bits from the logits alone."""
import numpy as np
import pytest
import torch

from paper_2602_22445_b200 import binding as B
from tests import lm_oracle as O

pytestmark = pytest.mark.gpu
DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
MOST = float(np.finfo(np.float32).max)


def forward(x, tokens, scale, top=0):
    rows, V = x.shape
    desc = B.make_logprob_desc(V, x.dtype, top=top, scale=scale)
    out = [torch.full((rows,), 77.0, device="cuda") for _ in range(3)]
    best = torch.full((rows, top), 77.0, device="cuda") if top else None
    which = torch.full((rows, top), 77, dtype=torch.int32, device="cuda") if top else None
    B.ftc_token_logprobs(desc, x, tokens, *out, best, which)
    return desc, out, best, which


def softmax_gradient(x, t, scale, up, de):
    """The definition from the logits alone, in 64 bits; entropy and its spread (the mean of |z - max|) too."""
    z = scale * x
    d = z - z.max(1, keepdims=True)
    s = np.exp(d).sum(1, keepdims=True)
    p = np.exp(d) / s
    logp = np.where(p > 0, d - np.log(s), 0)
    entropy = -(p * logp).sum(1, keepdims=True)
    g = -p * (up[:, None] + de[:, None] * (logp + entropy))
    g[np.arange(len(t)), t] += up
    return scale * g, p, logp, entropy, (p * -np.where(p > 0, d, 0)).sum(1, keepdims=True)


def edge_rows(rng, V, dtype, kind):
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = torch.from_numpy(rng.standard_normal((4, V))).to(dtype)
    if kind == "lowest":
        x[1] = low
        x[2] = low
        x[2, V // 3] = low / 2
    elif kind == "highest":
        x[1] = high
        x[2, V // 3] = high
        x[2, V - 1] = high
    else:                                 # either end in one row
        x[1, ::2] = low
        x[1, 1::2] = high
        x[2] = low
        x[2, 0] = high
    return x.cuda()


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [3, 90, 2048, 40001])
@pytest.mark.parametrize("kind", ["lowest", "highest", "both"])
@pytest.mark.parametrize("scale", [1.25, 1e4])
def test_rows_whose_lse_leaves_float32(name, V, kind, scale):
    """lse is held at float32's largest number there, never infinity, and log probabilities, entropy and gradient are those of the logits."""
    rng = np.random.default_rng(V)
    x = edge_rows(rng, V, DT[name], kind)
    t = np.array([0, V // 2, V // 3, V - 1])
    tokens = torch.from_numpy(t).cuda()
    desc, (given, entropy, lse), best, which = forward(x, tokens, scale, min(V, 3))
    scale = float(np.float32(scale))
    exact = x.double().cpu().numpy()
    w_lse, w_given, w_entropy, w_best, w_which, spread = O.logprobs(exact, t, scale, min(V, 3))
    s_off = O.sum_off(spread, V)
    got = lse.double().cpu().numpy()
    want = np.clip(w_lse, -MOST, MOST)
    assert np.isfinite(got).all() and (abs(got - want) <= s_off + 4 * O.U32 * (abs(want) + spread)).all()
    far = abs(w_given) > MOST             # a token that is further down than float32 reaches
    got = given.double().cpu().numpy()
    assert (abs(got - w_given)[~far] <= (s_off + 4 * O.U32 * (1 + abs(w_given)))[~far]).all() and np.isneginf(got[far]).all()
    assert (abs(entropy.double().cpu().numpy() - w_entropy) <= 4 * s_off * (1 + spread)).all()
    assert (which.cpu().numpy() == w_which).all()
    up, de = torch.tensor([1.0, -2.0, 0.5, 1.0], device="cuda"), torch.tensor([1.0, 3.0, -2.0, 0.0], device="cuda")
    d = torch.full((4, V), 7.0, dtype=DT[name], device="cuda")
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, up, de, d)
    want, p, logp, ent, spread = softmax_gradient(exact, t, scale, up.double().cpu().numpy(), de.double().cpu().numpy())
    # p by its exponent's roundings (of |log p| and of the largest of the row's lse that p is taken from, 2^7 in float32, 2^14 in 16 bits) and the
    # sum's; the entropy's by the forward pass
    held = np.minimum(abs(w_lse)[:, None], 2.0 ** 7 if name == "float32" else 2.0 ** 14)
    each = 4 * O.U32 * (1 + abs(logp) + held) + O.sum_off(spread, V)
    factor = abs(up.double().cpu().numpy())[:, None] + abs(de.double().cpu().numpy())[:, None] * (abs(logp) + ent + 1)
    off = scale * p * (factor * each + abs(de.double().cpu().numpy())[:, None] * 4 * O.sum_off(spread, V) * (1 + spread)) + scale * 4 * O.U32 * factor * p + scale * 2.0 ** -120
    rows = np.arange(4)
    off[rows, t] += scale * abs(up.double().cpu().numpy()) * 4 * O.U32
    off = off + (abs(want) + off) * O.half_step(name) + O.least(name) * O.half_step(name) * 2
    got = d.double().cpu().numpy()
    sure = abs(want) + off < torch.finfo(DT[name]).max
    assert np.isfinite(got[sure]).all() and (abs(got - want) <= off)[sure].all(), np.nanmax((abs(got - want) / off)[sure])
