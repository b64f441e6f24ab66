"""AdamW's states have the bits of the formula in plain float32, and weights move by it: subnormal second moments, codes beside a tie."""
import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import plain_adamw as A

pytestmark = pytest.mark.gpu

LR, B1, B2 = 3e-3, 0.9, 0.95
F = np.float32


class Run:
    """One tensor (n a multiple of 256) from zero states, played on the GPU and in plain float32 side by side."""

    def __init__(self, p, bits, dtype="float32"):
        import torch
        n = len(p)
        self.bits, self.p = bits, p.astype(F)
        self.param = torch.from_numpy(self.p).cuda()
        self.grad = torch.zeros(n, device="cuda")
        self.table = B.make_param_table([B.make_param(self.param, self.grad)])
        if bits == 32:
            self.dev = [torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")]
            self.want = [np.zeros(n, F), np.zeros(n, F)]
        else:
            self.dev = [torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"),
                        torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")]
            self.want = [t.cpu().numpy() for t in self.dev]

    def step(self, g, step, eps):
        import torch
        g = g.astype(F)
        m, v = self.want if self.bits == 32 else A.decode(*self.want)
        m, v = A.moments(g, m, v, B1, B2, step)
        p, off = A.weights(self.p, m, v, LR, B1, B2, eps, step)
        self.want = [m, v] if self.bits == 32 else list(A.encode(m, v))
        self.grad.copy_(torch.from_numpy(g))
        B.ftc_adamw_step(B.make_adamw(LR, B1, B2, eps, step), self.table, *self.dev)
        for got, want, what in zip(self.dev, self.want, ("m", "v", "scales of m", "scales of v")):
            got = got.cpu().numpy()
            bad = np.flatnonzero(got != want)
            assert not len(bad), f"{what}, step {step}: {len(bad)} differ, first {got[bad[0]]} for {want[bad[0]]}"
        got = self.param.cpu().numpy()
        bad = np.flatnonzero(~(np.abs(got - p) <= off))
        assert not len(bad), f"weights, step {step}: {len(bad)} outside, moved {got[bad[0]] - self.p[bad[0]]} for {p[bad[0]] - self.p[bad[0]]}"
        self.p = got


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-30, 1e-20, 1e-17, 1e-8])
@pytest.mark.parametrize("size", [3e-18, 1e-19, 1e-20, 3e-22])
def test_second_moments_below_the_smallest_normal_number(size, eps, bits):
    """v = (1 - beta2) g^2 is a subnormal number: the root under the move and under the codes is that of v, not of zero. Few blocks, and more
    than the GPU holds at once."""
    rng = np.random.default_rng([bits, int(-np.log10(size))])
    for n in (256 * 3, 256 * 12000) if eps in (1e-30, 1e-8) else (256 * 3,):
        job = Run(0.01 * rng.standard_normal(n), bits)
        for step in (1, 2):
            job.step(size * rng.standard_normal(n), step, eps)


@pytest.mark.parametrize("bits", [32, 8])
def test_subnormal_and_normal_second_moments_in_one_block(bits):
    rng = np.random.default_rng(bits)
    n = 256 * 8
    job = Run(0.01 * rng.standard_normal(n), bits)
    for step in (1, 2, 3):
        job.step(10.0 ** rng.uniform(-23, -15, n) * rng.choice([-1, 1], n), step, 1e-28)


@pytest.mark.parametrize("blocks", [300, 24000])
def test_codes_beside_a_tie(blocks):
    """Gradients whose codes of v lie within some units in the last place of a half: the codes are those of plain float32."""
    rng = np.random.default_rng(blocks)
    top = 10.0 ** rng.uniform(-3, 1, (blocks, 1))
    half = rng.integers(60, 255, (blocks, 256)) + 0.5
    g = top * (half / 255) ** 2 * (1 + rng.uniform(-2e-6, 2e-6, (blocks, 256)))
    g[:, 0] = top[:, 0]
    job = Run(np.zeros(blocks * 256), 8)
    job.step(g.ravel(), 1, 1e-8)
