"""Embedding, norm, log probabilities, allreduce, gradient norm, orthogonalised update and AdamW together: the example's step against autograd in 64 bits,
the CPU oracle and the updates' definitions."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import oracle as orc
from tests import lm_oracle as L
from tests import train_oracle as O

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_language_model_under_failures", os.path.join(ROOT, "examples", "train_language_model_under_failures.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("P,f,rows,V,H,k", [(12, 2, 10, 37, 24, 8), (8, 1, 30, 301, 72, 7)])
def test_one_step(P, f, rows, V, H, k):
    import torch
    job = example().Trainer(P=P, f=f, rows=rows, V=V, H=H, k=k, seed=3)
    before = [p.clone() for p in job.params]
    state = job.gen.get_state()
    tokens, targets = job.batch()
    job.gen.set_state(state)
    loss, (prefail, inop) = job.train_step()
    # each process's gradients by autograd in 64 bits
    table, gamma, beta, hidden, head = leaves = [p.double().requires_grad_() for p in before]
    x = torch.where((tokens >= 0)[:, None], table[tokens.clamp(min=0)], 0)
    z = x - x.mean(1, keepdim=True)
    y = z / (z.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma + beta
    logp = torch.log_softmax(y @ hidden @ head, 1)
    entropy = -(logp.exp() * logp).sum(1)
    given = logp.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    each = (torch.where(targets >= 0, -given - job.bonus * entropy, 0).view(P, rows)).mean(1)
    for p in (0, 1, P - 1):
        for g, q in zip(torch.autograd.grad(each[p], leaves, retain_graph=True), job.part):
            got = job.messages[q][:, p].reshape(-1)
            assert (got[:g.numel()].double() - g.reshape(-1)).norm() <= 1e-5 * g.norm() + 1e-9       # float32 through two products and back
            assert (got[g.numel():] == 0).all()
    assert abs(float(loss) - float(each.mean().detach())) <= 1e-5 * abs(float(each.mean().detach()))
    # what was delivered, bit for bit
    want_out, want_st = orc.batch(job.messages.cpu().numpy(), f, "sum", prefail, inop=inop, allreduce=True)
    assert np.array_equal(job.delivered.cpu().numpy(), want_out)
    assert np.array_equal(job.status.cpu().numpy().view(np.uint32), want_st)
    # the updates
    shares = [O.shares(want_st[q], k, p.numel()) for q, p in zip(job.part, before)]
    grads = [want_out[q].ravel()[:len(s)].astype(np.float64) * s for q, s in zip(job.part, shares)]
    norm = np.sqrt(sum((g ** 2).sum() for g in grads))
    assert abs(float(job.norm[0]) - norm) <= 1e-6 * norm
    clip, lr = min(1.0, 1.0 / norm), 3e-2
    for i in (0, 1, 2, 4):
        zeros = np.zeros(len(grads[i]))
        want, off = O.adamw(before[i].double().cpu().numpy().ravel(), grads[i], zeros, zeros, lr, 0.9, 0.95, 1e-8, 1, 0.0, zeros + 1, clip)
        O.assert_within(job.params[i].double().cpu().numpy().ravel(), want[0], off[0] + 4 * O.U * lr, what=str(i))
    rate = 0.2 * H ** 0.5
    want, _, x, off = L.muon(before[3].double().cpu().numpy(), np.zeros((H, H)), (grads[3] * clip).reshape(H, H), np.ones((H, H), bool), lr, rate, 0.01, 0.95, True, 1e-7, 5, 32)
    moved = np.linalg.norm(job.hidden.double().cpu().numpy() - want)
    assert moved <= lr * rate * (off + 1e-6 * np.linalg.norm(x)) + 4 * L.U32 * np.linalg.norm(want), moved       # 1e-6: the clip factor's own


def test_it_runs_on():
    import torch
    job = example().Trainer(seed=1)
    for _ in range(5):
        loss, _ = job.train_step()
    assert torch.isfinite(loss) and all(torch.isfinite(p).all() for p in job.params)
