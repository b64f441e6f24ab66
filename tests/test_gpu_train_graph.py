"""The training operators in a captured CUDA graph: the same bits as the calls, also where a call launches two kernels."""
import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_captured_step_equals_calls():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    rows, H, P, k = 900, 1032, 7, 24
    x, dy = (torch.randn(rows, H, generator=gen, device="cuda") for _ in range(2))
    gamma, beta = torch.ones(H, device="cuda"), torch.zeros(H, device="cuda")
    big = torch.randn(300000, generator=gen, device="cuda")
    desc = B.make_norm_desc(H, torch.float32, P=P, k=k)
    S = -(-H // k)

    def job():
        b = {n: torch.zeros(rows, H, device="cuda") for n in ("y", "dx")}
        b.update({n: torch.zeros(rows, device="cuda") for n in ("mean", "rstd")})
        b.update({n: torch.zeros(S, P, k, device="cuda") for n in ("dg", "db")})
        b["ws"] = torch.empty(B.ftc_layernorm_workspace_bytes(desc, rows), dtype=torch.uint8, device="cuda")
        b["p"] = [gamma.clone(), big.clone()]
        b["table"] = B.make_param_table([B.make_param(b["p"][0], beta + 0.5), B.make_param(b["p"][1], big * 0.1)])
        n = b["table"].blocks
        b["m"], b["v"] = torch.zeros(n * 256, dtype=torch.int8, device="cuda"), torch.zeros(n * 256, dtype=torch.uint8, device="cuda")
        b["ms"], b["vs"], b["norm"] = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(2, device="cuda")
        b["nws"] = torch.empty(B.ftc_grad_norm_workspace_bytes(b["table"]), dtype=torch.uint8, device="cuda")
        return b

    def step(b):
        B.ftc_layernorm_forward(desc, x, gamma, beta, b["y"], b["mean"], b["rstd"])
        B.ftc_layernorm_backward(desc, dy, x, gamma, b["mean"], b["rstd"], None, b["dx"], b["dg"], b["db"], b["ws"])
        B.ftc_grad_norm(b["table"], 1.0, b["norm"], None, b["nws"])
        B.ftc_adamw_step(B.make_adamw(1e-2, step=3), b["table"], b["m"], b["v"], b["ms"], b["vs"], b["norm"][1:])

    eager, held = job(), job()
    for _ in range(3):
        step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(held)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for name in ("y", "mean", "rstd", "dx", "dg", "db", "m", "v", "ms", "vs", "norm"):
        assert torch.equal(eager[name], held[name]), name
    assert all(torch.equal(a, b) for a, b in zip(eager["p"], held["p"]))
    assert np.isfinite(float(held["norm"][0])) and float(held["norm"][1]) < 1
