"""The training operators and the allreduce together: the example's steps, checked against plain arithmetic."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import oracle as orc
from tests import train_oracle as O

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_under_failures", os.path.join(ROOT, "examples", "train_under_failures.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_one_step_against_plain_arithmetic():
    import torch
    job = example().Trainer(P=12, f=2, rows=5, H=104, outputs=7, k=8, seed=3)
    gen_state = job.gen.get_state()
    w0 = job.weight.clone().normal_(0, 0.1, generator=job.gen)
    job.weight.copy_(w0)
    job.gen.set_state(gen_state)
    x = (torch.randn(job.rows, job.H, generator=job.gen, device="cuda") * 2 + 0.5).double()
    job.gen.set_state(gen_state)
    loss, (prefail, inop) = job.train_step()
    # the messages: each process's gradients by autograd in 64 bits
    gamma = torch.ones(job.H, dtype=torch.float64, device="cuda", requires_grad=True)
    beta = torch.zeros(job.H, dtype=torch.float64, device="cuda", requires_grad=True)
    w = w0.double().requires_grad_()
    z = x - x.mean(1, keepdim=True)
    target = z / z.square().mean(1, keepdim=True).sqrt() @ job.teacher.double()
    xh = z / (z.square().mean(1, keepdim=True) + 1e-5).sqrt()
    off = (xh * gamma + beta) @ w.view(job.H, -1) - target
    each = off.view(job.P, -1, job.outputs).square().sum(2).mean(1) * 0.5
    for p in (0, 5, 11):
        want = torch.autograd.grad(each[p], (gamma, beta, w), retain_graph=True)
        for g, q in zip(want, job.part):
            got = job.messages[q][:, p].reshape(-1)[:g.numel()].double()
            assert (got - g).norm() <= 1e-5 * g.norm() + 1e-9       # float32 through a forward and a backward pass
    assert abs(float(loss) - float(each.mean())) <= 1e-5 * float(each.mean())
    # what was delivered, bit for bit, and the sum over the processes included
    want_out, want_st = orc.batch(job.messages.cpu().numpy(), job.f, "sum", prefail, inop=inop, allreduce=True)
    assert np.array_equal(job.delivered.cpu().numpy(), want_out)
    assert np.array_equal(job.status.cpu().numpy().view(np.uint32), want_st)
    # the update
    shares = [O.shares(want_st[q], job.k, n) for q, n in zip(job.part, (job.H, job.H, job.weight.numel()))]
    grads = [want_out[q].ravel()[:len(s)] * s for q, s in zip(job.part, shares)]
    norm = np.sqrt(sum((g.astype(np.float64) ** 2).sum() for g in grads))
    assert abs(float(job.norm[0]) - norm) <= 1e-6 * norm
    clip = min(1.0, 1.0 / norm)
    for now, before, g, s, decay in zip((job.gamma, job.beta, job.weight), (np.ones(job.H), np.zeros(job.H), w0.double().cpu().numpy()), grads, shares, (0, 0, 0.01)):
        want, off = O.adamw(before, g, np.zeros(len(g)), np.zeros(len(g)), 1e-2, 0.9, 0.95, 1e-8, 1, decay, s * 0 + 1, clip)
        O.assert_within(now.double().cpu().numpy(), want[0], off[0] + 4 * O.U * 1e-2, what="weights")


def test_training_under_failures_learns():
    import torch
    job = example().Trainer(seed=1)
    first = float(job.train_step()[0])
    fewest = job.P
    for _ in range(149):
        loss, _ = job.train_step()
        fewest = min(fewest, int(job.status[:, 1].min()))
        assert (job.status[:, 0] & 0xFF == 0).all()
    assert fewest < job.P                                            # processes did fail
    assert float(loss) < 0.05 * first and torch.isfinite(job.weight).all()
