"""Token log probabilities, entropy, top alternatives and the logits' gradient against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_22445_b200 import binding as B
from tests import lm_oracle as O

pytestmark = pytest.mark.gpu
DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
INF = float("inf")


def logits_of(rng, rows, V, dtype, pad, kind):
    x = torch.from_numpy(rng.standard_normal((rows, V)) * 4).to(dtype)
    if kind == "masked":                  # parts, all but one, all of a row
        x[rng.random((rows, V)) < 0.5] = -INF
        x[0] = -INF
        if rows > 1:
            x[1] = -INF
            x[1, V // 2] = 3.0
        if rows > 2:
            x[2] = torch.finfo(dtype).min
        if rows > 3:
            x[3] = torch.finfo(dtype).min
            x[3, -1] = 1.0
    if kind == "same":
        x[:] = 2.5
    if kind == "far":
        x += 900 if dtype == torch.float16 else 3000
    if kind == "rising":                  # every element beats those before it
        x = torch.linspace(-9, 9, V, dtype=torch.float64).to(dtype).expand(rows, V).clone()
    room = torch.full((rows, V + pad), INF, dtype=dtype, device="cuda")
    room[:, :V] = x.cuda()
    return room[:, :V]


def forward(x, tokens, scale, top):
    rows, V = x.shape
    desc = B.make_logprob_desc(V, x.dtype, top=top, scale=scale)
    out = [torch.full((rows,), 77.0, device="cuda") for _ in range(3)]
    best = torch.full((rows, top), 77.0, device="cuda") if top else None
    which = torch.full((rows, top), 77, dtype=torch.int32, device="cuda") if top else None
    B.ftc_token_logprobs(desc, x, tokens, *out, best, which)
    return desc, out, best, which


def tokens_of(rng, rows, V, bits):
    t = rng.integers(0, V, rows)
    t[rng.random(rows) < 0.2] = rng.choice([-1, -100, V, 2 ** 31 - 1])
    return t, torch.from_numpy(t).to(torch.int64 if bits == 64 else torch.int32).cuda()


SIZES = [(1, 1, 0, 64), (3, 2, 1, 32), (5, 31, 0, 64), (9, 64, 0, 64), (2, 1000, 3, 32), (40, 1024, 0, 64), (7, 1025, 0, 32), (4, 5003, 5, 64), (1, 16384, 0, 64),
         (6, 32768, 8, 64), (1, 131072, 0, 32), (300, 2048, 0, 64), (2, 70001, 2, 64)]


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,V,pad,bits", SIZES)
@pytest.mark.parametrize("kind", ["plain", "masked", "same", "far", "rising"])
def test_forward(name, rows, V, pad, bits, kind):
    rng = np.random.default_rng(rows + V)
    x = logits_of(rng, rows, V, DT[name], pad, kind)
    t, tokens = tokens_of(rng, rows, V, bits)
    top, scale = min(V, (0, 1, 5, 20, 32)[(rows + len(kind)) % 5]), (1.0, 0.8)[rows % 2]
    _, (given, entropy, lse), best, which = forward(x, tokens, scale, top)
    scale = float(np.float32(scale))
    w_lse, w_given, w_entropy, w_best, w_which, spread = O.logprobs(x.double().cpu().numpy(), t, scale, top)
    s_off = O.sum_off(spread, V)

    def close(got, want, off):
        got = got.double().cpu().numpy()
        same = (got == want) | (np.isnan(got) & np.isnan(want))
        with np.errstate(invalid="ignore"):
            assert (same | (abs(got - want) <= off)).all(), abs(got - want).max()

    with np.errstate(invalid="ignore"):
        size = np.where(np.isfinite(w_lse), abs(w_lse), 0)
        close(lse, w_lse, s_off + 4 * O.U32 * (size + spread))
        close(given, w_given, s_off + 4 * O.U32 * np.where(np.isfinite(w_given), abs(w_given), 0) + 4 * O.U32)
        close(entropy, w_entropy, 4 * s_off * (1 + spread))
        if top:
            assert (which.cpu().numpy() == w_which).all()
            close(best, w_best, s_off[:, None] + 4 * O.U32 * (1 + np.where(np.isfinite(w_best), abs(w_best), 0)))


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,V,pad,bits", SIZES)
@pytest.mark.parametrize("kind", ["plain", "masked", "same", "rising"])
@pytest.mark.parametrize("what", ["both", "logprob", "entropy", "in place"])
def test_backward(name, rows, V, pad, bits, kind, what):
    rng = np.random.default_rng(rows * V)
    x = logits_of(rng, rows, V, DT[name], pad, kind)
    if kind == "masked" and rows > 2:
        x[2] = -INF                       # p of a row at the type's lowest value is beyond what lse can say in float32
    t, tokens = tokens_of(rng, rows, V, bits)
    desc, (given, entropy, lse), _, _ = forward(x, tokens, 0.8, 0)
    up = torch.from_numpy(rng.standard_normal(rows)).float().cuda() if what != "entropy" else None
    de = torch.from_numpy(rng.standard_normal(rows)).float().cuda() if what != "logprob" else None
    zero = np.zeros(rows)
    want, off = O.logprobs_backward(x.double().cpu().numpy(), t, float(np.float32(0.8)), lse.double().cpu().numpy(), entropy.double().cpu().numpy(),
                                    zero if up is None else up.double().cpu().numpy(), zero if de is None else de.double().cpu().numpy())
    if what == "in place":
        d = x
    else:
        d = torch.full((rows, V + pad), 7.0, dtype=DT[name], device="cuda")[:, :V]
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy if de is not None else None, up, de, d)
    got = d.double().cpu().numpy()
    off = off + (abs(want) + off) * O.half_step(name) + O.least(name) * O.half_step(name) * 2
    assert (abs(got - want) <= off).all(), (abs(got - want) / off).max()
    if pad:
        assert (d._base[:, V:] == (INF if what == "in place" else 7.0)).all()


@pytest.mark.parametrize("V", [100, 5000, 40000])
@pytest.mark.parametrize("bad", [float("nan"), INF])
def test_rows_with_nan_or_infinity(V, bad):
    x = torch.randn(4, V, device="cuda")
    x[1, V - 1] = bad
    x[2, 0] = bad
    tokens = torch.tensor([3, 3, -1, 5], device="cuda")
    desc, (given, entropy, lse), best, which = forward(x, tokens, 1.0, 4)
    for r in (1, 2):
        assert lse[r].isnan() and entropy[r].isnan() and best[r].isnan().all()
    assert given[1].isnan() and given[2] == 0
    assert all(torch.isfinite(v[r]).all() for v in (lse, entropy, best) for r in (0, 3))
    ones = torch.ones(4, device="cuda")
    d = torch.zeros_like(x)
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, ones, ones, d)
    assert d[1].isnan().all() and d[2].isnan().all() and torch.isfinite(d[0]).all() and torch.isfinite(d[3]).all()


def test_some_outputs_only():
    x = torch.randn(5, 3000, device="cuda")
    tokens = torch.arange(5, device="cuda")
    desc, (given, entropy, lse), _, _ = forward(x, tokens, 1.0, 0)
    a, b = torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda")
    B.ftc_token_logprobs(desc, x, tokens, a)
    B.ftc_token_logprobs(desc, x, None, None, None, b)
    assert torch.equal(a, given) and torch.equal(b, lse)
    top = B.make_logprob_desc(3000, torch.float32, top=3)
    v, w = torch.zeros(5, 3, device="cuda"), torch.zeros(5, 3, dtype=torch.int32, device="cuda")
    B.ftc_token_logprobs(top, x, None, None, None, None, v, w)
    assert torch.equal(w.long(), x.topk(3, 1).indices)


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [90, 40000])
@pytest.mark.parametrize("scale", [1e-6, 1e4, 1e6])
def test_masked_logits_at_the_ends_of_the_scale(name, V, scale):
    """-infinity is p = 0 however large the factors of the entropy's gradient are."""
    rng = np.random.default_rng(V)
    x = torch.from_numpy(rng.standard_normal((3, V)) / scale).float().clamp(-60000, 60000).to(DT[name])
    x[rng.random((3, V)) < 0.5] = -INF
    x[:, 1] = 0
    x = x.cuda()
    t = np.array([1, -1, 1])
    tokens = torch.from_numpy(t).cuda()
    desc, (_, entropy, lse), _, _ = forward(x, tokens, scale, 0)
    up, de = torch.tensor([1.0, -2.0, 0.0], device="cuda"), torch.tensor([1e3, -1e3, 1e3], device="cuda")
    d = torch.full((3, V), 7.0, dtype=DT[name], device="cuda")
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, up, de, d)
    want, off = O.logprobs_backward(x.double().cpu().numpy(), t, float(np.float32(scale)), lse.double().cpu().numpy(), entropy.double().cpu().numpy(),
                                    up.double().cpu().numpy(), de.double().cpu().numpy())
    got = d.double().cpu().numpy()
    if name == "float16":                 # gradients of up to 1e3 * scale: beyond what the type holds
        most = torch.finfo(torch.float16).max
        assert np.isfinite(got[abs(want) + off < most]).all() and not np.isnan(got).any()
        sure = abs(want) + off < most
        got, want, off = got[sure], want[sure], off[sure]
    off = off + (abs(want) + off) * O.half_step(name) + O.least(name) * O.half_step(name) * 2
    assert (abs(got - want) <= off).all(), (abs(got - want) / off).max()


def softmax_gradient(x, t, scale, up, de):
    """The definition from the logits alone, in 64 bits."""
    z = scale * x
    m = z.max(1, keepdims=True)
    s = np.exp(z - m).sum(1, keepdims=True)
    p = np.exp(z - m) / s
    logp = np.where(p > 0, z - m - np.log(s), 0)
    entropy = -(p * logp).sum(1, keepdims=True)
    g = -p * (up[:, None] + de[:, None] * (logp + entropy))
    g[np.arange(len(t)), t] += up
    return scale * g


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [3, 90, 2048, 40001])
@pytest.mark.parametrize("kind", ["lowest", "far", "far up"])
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_whose_lse_says_nothing_of_their_p(name, V, kind, in_place):
    """All of a row masked with the type's lowest value, or logits so far from zero that lse in float32 is too coarse: p comes from the logits."""
    rng = np.random.default_rng(V)
    low = torch.finfo(DT[name]).min
    x = torch.from_numpy(rng.standard_normal((3, V)) * 2).to(DT[name])
    if kind == "lowest":
        x[1] = low
    else:
        x[1] = (x[1].double() * 64 + (60000 if kind == "far up" else -60000)).to(DT[name])
    room = torch.full((3, V + 3), 7.0, dtype=DT[name], device="cuda")
    room[:, :V] = x.cuda()
    x = room[:, :V]
    t = np.array([V - 1, V // 2, 0])
    tokens = torch.from_numpy(t).cuda()
    desc, (_, entropy, lse), _, _ = forward(x, tokens, 0.5, 0)
    up, de = torch.tensor([1.0, -2.0, 0.5], device="cuda"), torch.tensor([1.0, 3.0, -2.0], device="cuda")
    exact = x.double().cpu().numpy()
    want = softmax_gradient(exact, t, 0.5, up.double().cpu().numpy(), de.double().cpu().numpy())
    d = x if in_place else torch.full((3, V), 7.0, dtype=DT[name], device="cuda")
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, up, de, d)
    got = d.double().cpu().numpy()
    # a term's exponent carries three roundings of z - max (64 at most where p counts) and the power 2^-22, s and ln s V additions, the entropy that
    # is given its own 4 sum_off (1 + spread); |log p + entropy| stays below 64 + ln V where p counts
    spread = np.log(V) + 8
    off = 0.5 * (2 + 3 * (64 + spread)) * (64 * 4 * O.U32 + 2.0 ** -22 + O.sum_off(spread, V)) + 0.5 * 3 * 4 * O.sum_off(spread, V) * (1 + spread)
    off = off + (abs(want) + off) * O.half_step(name) + O.least(name) * O.half_step(name) * 2
    assert (abs(got - want) <= off).all(), (abs(got - want) / off).max()
    assert (room[:, V:] == 7.0).all()


@pytest.mark.parametrize("V", [70, 50000])
def test_empty_and_broken_rows_with_large_factors(V):
    x = torch.randn(3, V, device="cuda")
    x[0] = -INF
    x[1, V // 2] = float("nan")
    tokens = torch.tensor([0, 1, 2], device="cuda")
    desc, (_, entropy, lse), _, _ = forward(x, tokens, 1e6, 0)
    d = torch.full_like(x, 7.0)
    many = torch.full((3,), 1e3, device="cuda")
    B.ftc_token_logprobs_backward(desc, x, tokens, lse, entropy, many, many, d)
    assert (d[0] == 0).all() and d[1].isnan().all() and torch.isfinite(d[2]).all()
