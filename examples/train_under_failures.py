"""Data-parallel training whose gradients go through the corrected allreduce while processes fail.

P simulated processes share a batch; each has its own gradient of a small model (layer norm, then a linear layer), sent as messages of k
elements. In every step some processes are dead before the allreduce and some die in it. The library computes the norm's passes with
the weight gradients of each process in the message layout, plays the allreduce of all messages, takes the norm of what was delivered and
makes the AdamW step with states in 8 bits -- the mean over the processes whose input is in each message, read from its status record.

    python examples/train_under_failures.py [steps]
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_22445_b200 import binding as B
from paper_2602_22445_b200 import scenarios as sc


class Trainer:
    """A norm and a linear layer on `P` processes with `rows` rows each, of which `f` may fail."""

    def __init__(self, P=32, f=3, rows=64, H=512, outputs=24, k=32, seed=0):
        self.P, self.f, self.rows, self.H, self.outputs, self.k = P, f, rows * P, H, outputs, k
        self.rng = np.random.Generator(np.random.PCG64(seed))
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.teacher = torch.randn(H, outputs, generator=self.gen, device="cuda") / H ** 0.5
        self.gamma, self.beta = torch.ones(H, device="cuda"), torch.zeros(H, device="cuda")
        self.weight = torch.zeros(H * outputs, device="cuda")
        self.norm_desc = B.make_norm_desc(H, torch.float32, P=P, k=k)
        # messages of gamma, beta and the linear layer, one after the other: [scenario][process][k]
        each = [-(-p.numel() // k) for p in (self.gamma, self.beta, self.weight)]
        cuts = np.cumsum([0] + each)
        self.S = int(cuts[-1])
        self.messages = torch.zeros(self.S, P, k, device="cuda")
        self.part = [slice(int(a), int(b)) for a, b in zip(cuts, cuts[1:])]
        self.delivered, self.status = torch.zeros(self.S, k, device="cuda"), torch.zeros(self.S, 4, dtype=torch.int32, device="cuda")
        self.sum_desc = B.make_desc(P, f, k, B.FTC_F32, "sum", root=0, max_inop=2)
        self.sum_ws = torch.empty(max(16, B.ftc_workspace_bytes(self.sum_desc, self.S, True)), dtype=torch.uint8, device="cuda")
        self.attempt = B.ftc_schedule_info(self.sum_desc)["rounds_attempt"]
        # the tensors with the delivered sums as gradients, their status records beside them
        self.table = B.make_param_table([
            B.make_param(p, self.delivered[q].view(-1)[:p.numel()], status=self.status[q], k=k, weight_decay=0.01 if p is self.weight else 0.0)
            for p, q in zip((self.gamma, self.beta, self.weight), self.part)])
        n = self.table.blocks
        self.m, self.v = torch.zeros(n * 256, dtype=torch.int8, device="cuda"), torch.zeros(n * 256, dtype=torch.uint8, device="cuda")
        self.m_scale, self.v_scale = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        self.norm = torch.zeros(2, device="cuda")
        self.norm_ws = torch.empty(B.ftc_grad_norm_workspace_bytes(self.table), dtype=torch.uint8, device="cuda")
        self.back_ws = torch.empty(B.ftc_layernorm_workspace_bytes(self.norm_desc, self.rows), dtype=torch.uint8, device="cuda")
        self.y, self.dx = torch.empty(self.rows, H, device="cuda"), torch.empty(self.rows, H, device="cuda")
        self.mean, self.rstd = torch.empty(self.rows, device="cuda"), torch.empty(self.rows, device="cuda")
        self.step = 0

    def failures(self):
        """The same pattern for every message of a step: up to f processes, some dead before the allreduce, up to two dying in it."""
        n = int(self.rng.integers(0, self.f + 1))
        victims = self.rng.choice(np.arange(self.f + 1, self.P), size=n, replace=False)
        dying = int(self.rng.integers(0, min(2, n) + 1))
        mask = sc.picks_to_masks(victims[None, dying:], self.P)
        inop = np.full((1, 2, 2), B.FTC_INOP_UNUSED, dtype=np.uint32)
        for i in range(dying):
            inop[0, i] = (victims[i], self.rng.integers(1, self.attempt))
        return np.repeat(mask, self.S, 0), np.repeat(inop, self.S, 0)

    def backward(self, x, target):
        """Loss, and every process's gradients as messages."""
        H, O, P = self.H, self.outputs, self.P
        B.ftc_layernorm_forward(self.norm_desc, x, self.gamma, self.beta, self.y, self.mean, self.rstd)
        w = self.weight.view(H, O)
        off = (self.y @ w - target) / (self.rows // P)              # each process's loss is the mean over its own rows
        B.ftc_layernorm_backward(self.norm_desc, off @ w.t(), x, self.gamma, self.mean, self.rstd, None, self.dx,
                                 self.messages[self.part[0]], self.messages[self.part[1]], self.back_ws)
        dw = torch.bmm(self.y.view(P, -1, H).transpose(1, 2), off.view(P, -1, O))
        flat = self.messages[self.part[2]].permute(1, 0, 2).reshape(P, -1).clone()
        flat[:, :H * O] = dw.view(P, -1)
        self.messages[self.part[2]] = flat.view(P, -1, self.k).permute(1, 0, 2)
        return 0.5 * (off * (self.rows // P)).square().sum(1).mean()

    def train_step(self, lr=1e-2):
        x = torch.randn(self.rows, self.H, generator=self.gen, device="cuda") * 2 + 0.5
        z = x - x.mean(1, keepdim=True)
        target = z / z.square().mean(1, keepdim=True).sqrt() @ self.teacher
        loss = self.backward(x, target)
        prefail, inop = self.failures()
        d_prefail, d_inop = (torch.from_numpy(np.ascontiguousarray(a).view(np.int32)).cuda() for a in (prefail, inop))
        B.ftc_allreduce_batch(self.sum_desc, self.S, self.messages, d_prefail, d_inop, None, self.delivered, self.status, self.sum_ws)
        self.step += 1
        B.ftc_grad_norm(self.table, 1.0, self.norm, None, self.norm_ws)
        B.ftc_adamw_step(B.make_adamw(lr, 0.9, 0.95, 1e-8, self.step), self.table, self.m, self.v, self.m_scale, self.v_scale, self.norm[1:])
        return loss, (prefail, inop)


def main(steps=200):
    job = Trainer()
    for i in range(steps):
        loss, _ = job.train_step()
        if i % 20 == 0 or i == steps - 1:
            included = job.status[:, 1]
            print(f"step {i:4d}  loss {float(loss):8.4f}  gradient norm {float(job.norm[0]):7.4f}  processes in the sum {int(included.min())}..{int(included.max())} of {job.P}")
    return float(loss)


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
