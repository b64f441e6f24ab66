"""The embedding, the log probabilities and the orthogonalised update in a captured CUDA graph and on a stream of their own: the same bits as the
calls, also where two graphs share a workspace and where an eager call comes between."""
import pytest

from paper_2602_22445_b200 import binding as B

pytestmark = pytest.mark.gpu


def make(n, V, H, P, k, shapes, products, seed=5):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b = {"embed": B.make_embed_desc(V, H, torch.bfloat16, torch.float32, P=P, k=k, scale=2.0), "prob": B.make_logprob_desc(V, torch.float16, top=3, scale=0.5)}
    b["tokens"] = torch.randint(-1, V, (n,), generator=gen, device="cuda")
    b["table"], b["y"] = torch.randn(V, H, generator=gen, device="cuda"), torch.zeros(n, H, dtype=torch.bfloat16, device="cuda")
    b["dy"], b["dtable"] = torch.randn(n, H, generator=gen, device="cuda").bfloat16(), torch.zeros(-(-V * H // k), P, k, device="cuda")
    b["ews"] = torch.empty(B.ftc_embedding_workspace_bytes(b["embed"], n), dtype=torch.uint8, device="cuda")
    b["x"], b["dx"] = torch.randn(n, V, generator=gen, device="cuda").half(), torch.zeros(n, V, dtype=torch.float16, device="cuda")
    for name in ("logprob", "entropy", "lse"):
        b[name] = torch.zeros(n, device="cuda")
    b["top"], b["which"] = torch.zeros(n, 3, device="cuda"), torch.zeros(n, 3, dtype=torch.int32, device="cuda")
    b["up"] = torch.randn(n, generator=gen, device="cuda")
    b["w"] = [torch.randn(s, generator=gen, device="cuda") for s in shapes]
    b["plan"] = B.make_muon_plan([B.make_matrix(w, torch.randn(w.shape, generator=gen, device="cuda")) for w in b["w"]])
    b["momentum"] = torch.zeros(b["plan"].blocks * 256, device="cuda")
    b["hyper"] = B.make_muon(1e-2, products=products)
    b["mws"] = torch.empty(B.ftc_muon_workspace_bytes(b["plan"], products), dtype=torch.uint8, device="cuda")
    return b


def step(b):
    B.ftc_embedding_forward(b["embed"], b["tokens"], b["table"], b["y"])
    B.ftc_embedding_backward(b["embed"], b["tokens"], b["dy"], None, b["dtable"], b["ews"])
    B.ftc_token_logprobs(b["prob"], b["x"], b["tokens"], b["logprob"], b["entropy"], b["lse"], b["top"], b["which"])
    B.ftc_token_logprobs_backward(b["prob"], b["x"], b["tokens"], b["lse"], b["entropy"], b["up"], b["up"], b["dx"])
    B.ftc_muon_step(b["hyper"], b["plan"], b["momentum"], None, b["mws"])


NAMES = ("y", "dtable", "logprob", "entropy", "lse", "top", "which", "dx", "momentum")
JOBS = [(300, 900, 64, 3, 16, [(40, 90), (300, 200)], 16), (5000, 2000, 40, 2, 7, [(64, 64)], 32), (3, 20000, 8, 1, 8, [(500, 130)], 32)]


def same(a, b):
    import torch
    torch.cuda.synchronize()
    for name in NAMES:
        assert torch.equal(a[name], b[name]), name
    assert all(torch.equal(x, y) for x, y in zip(a["w"], b["w"]))


@pytest.mark.parametrize("job", JOBS)
def test_captured_equals_calls(job):
    import torch
    eager, held = make(*job), make(*job)
    for _ in range(3):
        step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(held)
    for _ in range(3):
        graph.replay()
    same(eager, held)


@pytest.mark.parametrize("job", JOBS[:1])
def test_graphs_that_share_workspaces(job):
    import torch
    eager, held = [make(*job, seed=s) for s in (1, 2)], [make(*job, seed=s) for s in (1, 2)]
    for name in ("ews", "mws"):
        held[1][name] = held[0][name]
    graphs = []
    for b in held:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(b)
    for _ in range(2):
        for g in graphs:
            g.replay()
    for b in eager:
        step(b)
        step(b)
    for a, b in zip(eager, held):
        same(a, b)


@pytest.mark.parametrize("job", JOBS)
def test_on_another_stream(job):
    import torch
    a, b = make(*job), make(*job)
    step(a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(b)
    side.synchronize()
    same(a, b)
