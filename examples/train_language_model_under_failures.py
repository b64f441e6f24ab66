"""Data-parallel training of a small language model whose gradients go through the corrected allreduce while processes fail.

P simulated processes share a batch of tokens; the model looks a token up, norms the row, multiplies it with a hidden matrix and takes logits for
the next token. The library computes the lookup, the norm, the log probabilities and all their gradients; the embedding's and the norm's come
out per process as messages, the two matrix products' are sent as messages too. It plays the allreduce of all messages, takes the norm of
what was delivered, moves the hidden matrix by an orthogonalised update and the other tensors by AdamW with states in 8 bits.

    python examples/train_language_model_under_failures.py [steps]
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
    """`P` processes with `rows` tokens each, of which `f` may fail; a vocabulary of V tokens, H channels, messages of k elements."""

    def __init__(self, P=16, f=2, rows=64, V=200, H=128, k=16, entropy_bonus=0.01, seed=0):
        self.P, self.f, self.n, self.V, self.H, self.k, self.bonus = P, f, rows * P, V, H, k, entropy_bonus
        self.rng = np.random.Generator(np.random.PCG64(seed))
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.follows = torch.randint(0, V, (V,), generator=gen, device="cuda")           # the text: a token is followed by one other, mostly
        self.table = torch.randn(V, H, generator=gen, device="cuda") * 0.5
        self.gamma, self.beta = torch.ones(H, device="cuda"), torch.zeros(H, device="cuda")
        self.hidden = torch.randn(H, H, generator=gen, device="cuda") / H ** 0.5
        self.head = torch.randn(H, V, generator=gen, device="cuda") / H ** 0.5
        self.params = (self.table, self.gamma, self.beta, self.hidden, self.head)
        # messages of all tensors, one after the other: [scenario][process][k]
        cuts = np.cumsum([0] + [-(-p.numel() // k) for p in self.params])
        self.S = int(cuts[-1])
        self.part = [slice(int(a), int(b)) for a, b in zip(cuts, cuts[1:])]
        self.messages = torch.zeros(self.S, P, k, device="cuda")
        self.delivered, self.status = torch.zeros(self.S, k, device="cuda"), torch.zeros(self.S, 4, dtype=torch.int32, device="cuda")
        self.sum_desc = B.make_desc(P, f, k, B.FTC_F32, "sum", root=0, max_inop=2)
        self.sum_ws = torch.empty(max(16, B.ftc_workspace_bytes(self.sum_desc, self.S, True)), dtype=torch.uint8, device="cuda")
        self.attempt = B.ftc_schedule_info(self.sum_desc)["rounds_attempt"]
        # the operators' descriptors and buffers
        self.embed_desc = B.make_embed_desc(V, H, torch.float32, P=P, k=k)
        self.norm_desc = B.make_norm_desc(H, torch.float32, P=P, k=k)
        self.prob_desc = B.make_logprob_desc(V, torch.float32)
        self.embed_ws = torch.empty(B.ftc_embedding_workspace_bytes(self.embed_desc, self.n), dtype=torch.uint8, device="cuda")
        self.norm_ws = torch.empty(B.ftc_layernorm_workspace_bytes(self.norm_desc, self.n), dtype=torch.uint8, device="cuda")
        self.x, self.y, self.dx = (torch.empty(self.n, H, device="cuda") for _ in range(3))
        self.mean, self.rstd, self.logprob, self.entropy, self.lse = (torch.empty(self.n, device="cuda") for _ in range(5))
        # what was delivered, as the updates take it
        grads = [self.delivered[q].view(-1)[:p.numel()] for p, q in zip(self.params, self.part)]
        status = [self.status[q] for q in self.part]
        self.all = B.make_param_table([B.make_param(p, g, status=s, k=k) for p, g, s in zip(self.params, grads, status)])
        self.rest = B.make_param_table([B.make_param(self.params[i], grads[i], status=status[i], k=k) for i in (0, 1, 2, 4)])
        self.plan = B.make_muon_plan([B.make_matrix(self.hidden, grads[3], status=status[3], k=k, lr_scale=0.2 * H ** 0.5, weight_decay=0.01)])
        self.norm, self.all_ws = torch.zeros(2, device="cuda"), torch.empty(B.ftc_grad_norm_workspace_bytes(self.all), dtype=torch.uint8, device="cuda")
        blocks = self.rest.blocks
        self.m, self.v = torch.zeros(blocks * 256, dtype=torch.int8, device="cuda"), torch.zeros(blocks * 256, dtype=torch.uint8, device="cuda")
        self.m_scale, self.v_scale = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda")
        self.momentum = torch.zeros(self.plan.blocks * 256, device="cuda")
        self.muon_ws = torch.empty(B.ftc_muon_workspace_bytes(self.plan), dtype=torch.uint8, device="cuda")
        self.step = 0

    def batch(self):
        """Tokens and the ones to predict; every tenth position of the batch is padding on either side."""
        tokens = torch.randint(0, self.V, (self.n,), generator=self.gen, device="cuda")
        other = torch.randint(0, self.V, (self.n,), generator=self.gen, device="cuda")
        targets = torch.where(torch.rand(self.n, generator=self.gen, device="cuda") < 0.9, self.follows[tokens], other)
        padding = torch.arange(self.n, device="cuda") % 10 == 9
        return torch.where(padding, -1, tokens), torch.where(padding, -1, targets)

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

    def send(self, which, each):
        """[P][elements] as a tensor's messages."""
        flat = torch.zeros(self.P, (self.part[which].stop - self.part[which].start) * self.k, device="cuda")
        flat[:, :each.shape[1]] = each
        self.messages[self.part[which]] = flat.view(self.P, -1, self.k).permute(1, 0, 2)

    def backward(self, tokens, targets):
        """Loss, and every process's gradients as messages. A process's loss: the mean over its positions of -logprob - bonus * entropy, padding 0."""
        P, H, V, rows = self.P, self.H, self.V, self.n // self.P
        B.ftc_embedding_forward(self.embed_desc, tokens, self.table, self.x)
        B.ftc_layernorm_forward(self.norm_desc, self.x, self.gamma, self.beta, self.y, self.mean, self.rstd)
        z = self.y @ self.hidden
        logits = z @ self.head
        B.ftc_token_logprobs(self.prob_desc, logits, targets, self.logprob, self.entropy, self.lse)
        scored = (targets >= 0).float()
        loss = -(self.logprob + self.bonus * self.entropy * scored).mean()
        up, de = -scored / rows, -self.bonus * scored / rows
        B.ftc_token_logprobs_backward(self.prob_desc, logits, targets, self.lse, self.entropy, up, de, logits)          # in place
        dz = logits @ self.head.t()
        self.send(4, torch.bmm(z.view(P, rows, H).transpose(1, 2), logits.view(P, rows, V)).view(P, -1))
        self.send(3, torch.bmm(self.y.view(P, rows, H).transpose(1, 2), dz.view(P, rows, H)).view(P, -1))
        B.ftc_layernorm_backward(self.norm_desc, dz @ self.hidden.t(), self.x, self.gamma, self.mean, self.rstd, None, self.dx,
                                 self.messages[self.part[1]], self.messages[self.part[2]], self.norm_ws)
        B.ftc_embedding_backward(self.embed_desc, tokens, self.dx, None, self.messages[self.part[0]], self.embed_ws)
        return loss

    def train_step(self, lr=3e-2):
        loss = self.backward(*self.batch())
        prefail, inop = self.failures()
        d_prefail, d_inop = (torch.from_numpy(np.ascontiguousarray(a).view(np.int32)).cuda() for a in (prefail, inop))
        B.ftc_allreduce_batch(self.sum_desc, self.S, self.messages, d_prefail, d_inop, None, self.delivered, self.status, self.sum_ws)
        self.step += 1
        B.ftc_grad_norm(self.all, 1.0, self.norm, None, self.all_ws)
        B.ftc_muon_step(B.make_muon(lr, products=32), self.plan, self.momentum, self.norm[1:], self.muon_ws)
        B.ftc_adamw_step(B.make_adamw(lr, 0.9, 0.95, 1e-8, self.step), self.rest, self.m, self.v, self.m_scale, self.v_scale, self.norm[1:])
        return loss, (prefail, inop)


def main(steps=200):
    job = Trainer()
    for i in range(steps):
        loss, _ = job.train_step()
        if i % 20 == 0 or i == steps - 1:
            B.check_muon(job.muon_ws)
            included = job.status[:, 1]
            print(f"step {i:4d}  loss {float(loss):8.4f}  gradient norm {float(job.norm[0]):7.4f}  processes in the sum {int(included.min())}..{int(included.max())} of {job.P}")
    return float(loss)


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
