"""AdamW in 8 bits with betas near 1: codes that keep the states' mean, and states that follow those in 32 bits where nearest codes would not."""
import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import plain_adamw as A

pytestmark = pytest.mark.gpu
F = np.float32


class Job:
    def __init__(self, n, bits, seed=0, offset=0):
        import torch
        self.param = torch.zeros(n + offset, device="cuda")[offset:]
        self.grad = torch.zeros(n + offset, device="cuda")[offset:]
        self.table = B.make_param_table([B.make_param(self.param, self.grad)])
        nb = self.table.blocks
        types = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
        self.state = [torch.zeros(nb * 256, dtype=t, device="cuda") for t in types]
        if bits == 8:
            self.state += [torch.zeros(nb, device="cuda"), torch.zeros(nb, device="cuda")]

    def step(self, step, beta1, beta2):
        B.ftc_adamw_step(B.make_adamw(1e-3, beta1, beta2, 1e-8, step), self.table, *self.state)

    def values(self):
        import torch
        if len(self.state) == 2:
            return self.state
        out = [torch.empty(self.table.blocks * 256, device="cuda") for _ in range(2)]
        B.ftc_adamw_states(self.table, *self.state, *out)
        return out


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.99, 0.95), (0.99, 0.999), (0.96875, 0.96875), (0.97, 0.9999)])
@pytest.mark.parametrize("blocks,offset", [(40, 0), (40, 3), (12000, 0)])
def test_codes(beta1, beta2, blocks, offset):
    """Three steps' codes by their definition. A root that is off by 2^-22 of itself may turn a code whose u lies there; few do."""
    rng = np.random.default_rng(blocks + offset)
    import torch
    n = blocks * 256
    job = Job(n, 8, offset=offset)
    want = [t.cpu().numpy() for t in job.state]
    for step in (1, 2, 900000007):
        g = (10.0 ** rng.uniform(-3, 0, n) * rng.choice([-1, 1], n)).astype(F)
        m, v = A.moments(g, *A.decode(*want), beta1, beta2, step)
        job.grad.copy_(torch.from_numpy(g))
        job.step(step, beta1, beta2)
        got = [t.cpu().numpy() for t in job.state]
        xm, xv, ms, vs = A.squares_of_codes(m, v)
        assert (got[2] == ms).all() and (got[3] == vs).all()
        u = A.dither(np.arange(n), step).reshape(-1, 256)
        near = A.encode(m, v)
        for code, x, most, power, beta, nearest in ((np.abs(got[0].astype(int)), xm, 127, 2, beta1, np.abs(near[0].astype(int))), (got[1], xv, 255, 4, beta2, near[1])):
            if beta <= 0.96875:
                assert (code == nearest).all()
                continue
            lo, hi = (A.dithered_root(x * (1 + d), u, most, power).ravel() for d in (-2.0 ** -20, 2.0 ** -20))
            if power == 4:
                lo, hi = np.maximum(lo, 1), np.maximum(hi, 1)
            assert ((lo <= code) & (code <= hi)).all() and (lo != hi).mean() < 1e-3
        assert (np.sign(got[0]) * np.sign(m) >= 0).all()
        want = got


def test_mean_of_a_state_is_kept():
    """One step from zero states at many step numbers: the mean of what each element's codes stand for is the element's state, to the
    even spread of 4096 values of u (a few 4096ths of the way between two codes)."""
    import torch
    rng = np.random.default_rng(3)
    n, steps, beta = 512, 4096, 0.999
    g = (10.0 ** rng.uniform(-3, 0, n) * rng.choice([-1, 1], n)).astype(F)
    g[::256] = 1
    job = Job(n, 8)
    job.grad.copy_(torch.from_numpy(g))
    total = [torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2)]
    for step in range(1, steps + 1):
        for t in job.state:
            t.zero_()
        job.step(step, beta, beta)
        for sum_, x in zip(total, job.values()):
            sum_ += x.double()
    m, v = A.moments(g, np.zeros(n, F), np.zeros(n, F), beta, beta, 1)
    xm, xv, ms, vs = A.squares_of_codes(m, v)
    for got, want, x, power, unit in ((total[0], m, xm, 2, ms[:, None] / 127 ** 2), (total[1], v, xv, 4, vs[:, None] ** 2 / 255.0 ** 4)):
        c = np.floor(np.sqrt(x.astype(np.float64)))
        gap = ((c + 1) ** power - c ** power) * unit
        off = np.abs(got.cpu().numpy() / steps - want)
        lifted = (c == 0).ravel() if power == 4 else np.zeros(n, bool)           # code 0 is not given to a second moment above zero
        assert (off <= 8 / steps * gap.ravel() + 1e-6 * np.abs(want))[~lifted].all()


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.99), (0.9, 0.999), (0.98, 0.99)])
@pytest.mark.parametrize("shrink,part", [(0.1, 255), (0.01, 100)])
def test_states_follow_those_in_32_bits(beta1, beta2, shrink, part):
    """Gradients of a part of a block become small: after some multiples of 1 / (1 - beta2) steps the second moment is that of the small ones.
    A code that is rounded up and down with the right mean spreads around it (one code near 25 is a sixth of the root); nearest codes left the median
    at 1.5 to 75 times the root."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(int(1000 * beta2))
    blocks = 16
    small, big = (Job(blocks * 256, b) for b in (8, 32))
    scale = torch.ones(blocks, 256, device="cuda")
    first, steps = (1000, 3000) if beta2 == 0.99 else (2000, 10000)
    for step in range(1, first + steps + 1):
        if step == first:
            scale[:, :part] = shrink
        g = (torch.randn(blocks, 256, generator=gen, device="cuda") * scale).view(-1)
        for job in (small, big):
            job.grad.copy_(g)
            job.step(step, beta1, beta2)
    ratio = (small.values()[1].double() / big.values()[1].double()).sqrt().view(blocks, 256)[:, :part]
    assert 0.85 <= float(ratio.median()) <= 1.1
    assert 0.9 <= float((ratio ** 2).mean()) <= 1.15
    assert float(ratio.min()) > 0.2 and float(ratio.max()) < 3
    away = (small.values()[0] - big.values()[0]).view(blocks, 256)[:, :part]
    size = big.values()[0].view(blocks, 256)
    assert float(away.abs().mean()) < 0.02 * float(size.abs().amax(1).mean())   # first moments: within a code of the block's scale


def test_weights_follow_those_of_32_bits():
    """Elements whose gradients become small go on at the rate that 32-bit states give them, not at a part of it."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(2)
    small, big = (Job(256 * 8, b) for b in (8, 32))
    scale = torch.ones(8, 256, device="cuda")
    begin = None
    for step in range(1, 10001):
        if step == 2000:
            scale[:, :100] = 0.01
        if step == 8000:
            begin = [job.param.clone() for job in (small, big)]
        g = ((torch.randn(8, 256, generator=gen, device="cuda") + 0.5) * scale).view(-1)
        for job in (small, big):
            job.grad.copy_(g)
            job.step(step, 0.9, 0.999)
    moved = [(job.param - b).view(8, 256)[:, :100].mean() for job, b in zip((small, big), begin)]
    assert 0.8 < float(moved[0] / moved[1]) < 1.25


@pytest.mark.parametrize("beta2", [0.999, 0.99999, 1 - 2.0 ** -24])
def test_float32_states_over_steps(beta2):
    """States in 32 bits against the formula in 64: a step adds at most four half units (beta's rounding, two products, a sum) to what is off."""
    import torch
    rng = np.random.default_rng(5)
    n, beta1, steps = 2560, 0.95, 60
    job = Job(n, 32)
    m, v = np.zeros(n), np.zeros(n)
    for step in range(1, steps + 1):
        g = np.clip(rng.standard_normal(n), -6, 6).astype(F)
        job.grad.copy_(torch.from_numpy(g))
        job.step(step, beta1, beta2)
        m, v = m * beta1 + (1 - beta1) * g.astype(np.float64), v * beta2 + (1 - beta2) * g.astype(np.float64) ** 2
    got = [t.double().cpu().numpy() for t in job.state]
    assert (np.abs(got[1] - v) <= 2.0 ** -24 * 4 * (steps + 4) * v).all()
    assert (np.abs(got[0] - m) <= 2.0 ** -24 * 4 * (steps + 4) * 6).all()        # no gradient is larger than 6
