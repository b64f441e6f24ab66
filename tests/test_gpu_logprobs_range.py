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


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [90, 3001, 40001])
@pytest.mark.parametrize("shift", [0, 100, 300, 3000, 15000, -3000])
def test_gradient_of_logits_far_from_zero(name, V, shift):
    """As near to the definition as the type allows, wherever the logits lie: p is good to 2^-17 in float32 and to a quarter of the type's half step in
    16 bits."""
    rng = np.random.default_rng(V + abs(shift))
    x = torch.from_numpy(rng.standard_normal((3, V)) * 3 + shift).to(DT[name]).cuda()
    t = np.array([0, V // 2, V - 1])
    tokens = torch.from_numpy(t).cuda()
    desc, (_, entropy, lse), _, _ = forward(x, tokens, 1.0)
    up, de = np.array([1.0, -2.0, 0.5]), np.array([0.0, 3.0, -2.0])
    d = torch.full((3, V), 7.0, dtype=DT[name], device="cuda")
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, torch.from_numpy(up).float().cuda(), torch.from_numpy(de).float().cuda(), d)
    want, p, logp, ent, spread = softmax_gradient(x.double().cpu().numpy(), t, 1.0, up, de)
    # an error e of log p moves p (up + de (log p + entropy)) by e p (|up| + |de| (|log p| + entropy + 1)): e is half a step of lse (2^-18 below 2^7,
    # 2^-14 below 2^11, 2^-11 below 2^14, where it is found from the logits), the forward pass's own, and three roundings of |log p|
    e = {"float32": 2.0 ** -18, "float16": 2.0 ** -14, "bfloat16": 2.0 ** -11}[name]
    e = e + 4 * O.U32 * (1 + abs(logp)) + O.sum_off(spread, V)
    off = p * (abs(up)[:, None] + abs(de)[:, None] * (abs(logp) + ent + 1)) * e + p * abs(de)[:, None] * 4 * O.sum_off(spread, V) * (1 + spread)
    off[np.arange(3), t] += abs(up) * 4 * O.U32
    off = off + (abs(want) + off) * O.half_step(name) + O.least(name) * O.half_step(name) * 2
    got = d.double().cpu().numpy()
    assert (abs(got - want) <= off).all(), (abs(got - want) / off).max()


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [4, 90, 40001])
@pytest.mark.parametrize("scale", [0.4, 1e-3, 1e-6])
def test_tokens_further_below_the_largest_than_float32_reaches(name, V, scale):
    """x[token] - max leaves float32 where the type's lowest value meets the largest one; times a small scale it does not."""
    rng = np.random.default_rng(V)
    x = edge_rows(rng, V, DT[name], "both")
    x[3] = torch.finfo(DT[name]).min
    x[3, 1] = torch.finfo(DT[name]).max / 2
    t = np.array([0, 0, V - 1, V // 2])
    _, (given, entropy, lse), best, which = forward(x, torch.from_numpy(t).cuda(), scale, 4)
    w_lse, w_given, w_entropy, w_best, w_which, spread = O.logprobs(x.double().cpu().numpy(), t, float(np.float32(scale)), 4)
    s_off = O.sum_off(spread, V)
    for got, want, off in ((given, w_given, s_off), (best, w_best, s_off[:, None]), (lse, w_lse, s_off)):
        assert (abs(got.double().cpu().numpy() - want) <= off + 4 * O.U32 * (1 + abs(want))).all()
    assert (which.cpu().numpy() == w_which).all() and (abs(entropy.double().cpu().numpy() - w_entropy) <= 4 * s_off * (1 + spread)).all()
