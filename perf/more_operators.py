"""Workloads of the operators at the two ends of a language model and of its matrices' update, as a training step under failures has
them: embedding lookup and its gradient for each simulated process, log probabilities of given tokens with entropy and top
alternatives and their gradient, and the orthogonalised update of many matrices by Newton-Schulz products.

A case is a dict of plain values. `run` computes it in plain torch (32-bit arithmetic, rounded once at the end) or, with
`own` set, through this repository's library.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SZ = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                              # momentum is laid out in blocks of so many elements of one matrix
LR, MOMENTUM, DECAY, EPS = 3e-4, 0.95, 0.1, 1e-7
STEPS = 5
QUINTIC = (3.4445, -4.7750, 2.0315)      # a X + (b A + c A A) X with A = X X^T
IGNORED = -100                           # a token that stands for none (padding)


# ---- cases ----------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the tokens of one decoding step of 64 requests: a call's latency
        {"name": "embed fwd, 64 tokens", "op": "embed", "n": 64, "V": 32768, "H": 1024, "x": "bf16", "w": "bf16", "bits": 64, "scale": 32.0},
        # a training batch of 64k tokens of a model of 4096 channels
        {"name": "embed fwd, 64k tokens", "op": "embed", "n": 65536, "V": 65536, "H": 4096, "x": "bf16", "w": "f32", "bits": 64, "scale": 1.0},
        # 8 processes with 64 tokens each, a small vocabulary, messages of 16 elements: a call's latency
        {"name": "embed bwd, 8 processes", "op": "dembed", "n": 512, "V": 1000, "H": 256, "P": 8, "k": 16, "x": "f32", "w": "f32", "bits": 64, "scale": 16.0, "ragged": False},
        # packed sequences divided unevenly (some processes have none), sizes that no wide vector divides, messages across rows
        {"name": "embed bwd, ragged odd", "op": "dembed", "n": 8191, "V": 20011, "H": 301, "P": 16, "k": 7, "x": "f16", "w": "f32", "bits": 32, "scale": 1.0, "ragged": True},
        # a training batch of 32k tokens over 8 processes, messages of 32 elements
        {"name": "embed bwd, 32k tokens", "op": "dembed", "n": 32768, "V": 32768, "H": 1024, "P": 8, "k": 32, "x": "bf16", "w": "f32", "bits": 64, "scale": 32.0, "ragged": False},
        # one decoding step of 8 requests over a large vocabulary, with the alternatives that a server returns
        {"name": "logprobs, 8 rows", "op": "logp", "rows": 8, "V": 131072, "x": "bf16", "top": 20, "scale": 1.25, "pad": 0, "bits": 64},
        # scoring a prompt of odd length over an odd vocabulary, rows cut out of a padded matrix
        {"name": "logprobs, 1021 odd rows", "op": "logp", "rows": 1021, "V": 50021, "x": "f16", "top": 5, "scale": 1.0, "pad": 27, "bits": 64},
        # the loss of a training batch of 8k tokens, forward
        {"name": "logprobs, 8k tokens", "op": "logp", "rows": 8192, "V": 65536, "x": "bf16", "top": 0, "scale": 1.0, "pad": 0, "bits": 64},
        # and its gradient, with that of an entropy bonus
        {"name": "logprobs bwd, 8k tokens", "op": "dlogp", "rows": 8192, "V": 65536, "x": "bf16", "scale": 1.0, "pad": 0, "bits": 64},
        # a toy model's matrices: latency
        {"name": "muon, small", "op": "muon", "layers": 2, "H": 64, "F": 256, "p": "f32", "master": False, "g": "f32", "k": 0},
        # odd widths
        {"name": "muon, 4 odd layers", "op": "muon", "layers": 4, "H": 601, "F": 1803, "p": "f32", "master": False, "g": "bf16", "k": 0},
        # 12 layers in bf16 with a float32 copy, delivered messages of 32 elements as gradients
        {"name": "muon, 12 layers delivered", "op": "muon", "layers": 12, "H": 1024, "F": 4096, "p": "bf16", "master": True, "g": "f32", "k": 32},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "dembed", "dembed", "logp", "logp", "dlogp", "muon", "muon"])
    if op in ("embed", "dembed"):
        H = _spread(rng, 24, 4096)
        if rng.random() < 0.6:
            H = max(8, H // 8 * 8)
        c = {"op": op, "n": _spread(rng, 1, min(65536, 65536 * 4096 // H)), "V": _spread(rng, 64, 65536), "H": H, "x": rng.choice(["f32", "bf16", "bf16", "f16"]),
             "bits": rng.choice([64, 64, 32]), "scale": rng.choice([1.0, math.sqrt(H)])}
        c["w"] = rng.choice(["f32", c["x"]])
        if op == "dembed":
            c["n"] = min(c["n"], 32768 * 1024 // H)
            c["n"] = max(1, c["n"])
            c["P"] = min(_spread(rng, 1, 64), c["n"])
            c["V"] = max(64, min(c["V"], 32768 * 1024 * 8 // (c["P"] * H)))
            c["k"] = rng.choice([4, 8, 16, 32, 32, 7])
            c["ragged"] = rng.random() < 0.5
            if not c["ragged"]:
                c["n"] = c["n"] // c["P"] * c["P"]
        return c
    if op in ("logp", "dlogp"):
        V = _spread(rng, 64, 131072)
        if rng.random() < 0.5:
            V = max(64, V // 64 * 64)
        x = rng.choice(["bf16", "bf16", "f16", "f32"])
        c = {"op": op, "rows": _spread(rng, 1, min(16384, 8192 * 65536 * 2 // (V * SZ[x]))), "V": V, "x": x, "scale": rng.choice([1.0, 1.0, 1.25]),
             "pad": rng.choice([0, 0, 3, 64]), "bits": rng.choice([64, 64, 32])}
        if op == "logp":
            c["top"] = rng.choice([0, 0, 1, 5, 20])
        return c
    H = _spread(rng, 24, 1024)
    if rng.random() < 0.5:
        H = max(8, H // 8 * 8)
    c = {"op": op, "layers": rng.randint(1, 12), "H": H, "F": H * rng.randint(1, 4), "k": rng.choice([0, 0, 4, 32, 7]), "p": rng.choice(["f32", "bf16", "bf16", "f16"])}
    c["g"] = "f32" if c["k"] else rng.choice(["f32", "bf16", "f16"])
    c["master"] = c["p"] != "f32" and rng.random() < 0.6
    return c


def _shapes(case):
    """The kinds of matrices of a layer and how many of each the model has: four of the attention, two of the feed-forward block."""
    H, F, n = case["H"], case["F"], case["layers"]
    return [(4 * n, H, H), (n, H, F), (n, F, H)]


def work(case):
    if case["op"] in ("embed", "dembed"):
        n, H = case["n"], case["H"]
        if case["op"] == "embed":            # a table row that several tokens name is read once
            rows = case["V"] * (1 - (1 - 1 / case["V"]) ** n)
            return {"bytes": n * case["bits"] // 8 + rows * H * SZ[case["w"]] + n * H * SZ[case["x"]], "flops": n * H}
        out = -(-case["V"] * H // case["k"]) * case["k"] * case["P"]
        return {"bytes": n * case["bits"] // 8 + n * H * SZ[case["x"]] + 4 * out, "flops": 2 * n * H}
    if case["op"] in ("logp", "dlogp"):
        n = case["rows"] * case["V"]
        if case["op"] == "logp":
            return {"bytes": n * SZ[case["x"]] + case["rows"] * (case["bits"] // 8 + 12 + 8 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * n * SZ[case["x"]] + case["rows"] * (case["bits"] // 8 + 16), "flops": 8 * n}
    per = SZ[case["g"]] + (SZ[case["p"]] + 8 if case["master"] else 2 * SZ[case["p"]]) + 8 + (16 / case["k"] if case["k"] else 0)
    nbytes = flops = 0
    for count, rows, cols in _shapes(case):
        m, n = min(rows, cols), max(rows, cols)
        nbytes += count * m * n * per
        flops += count * STEPS * (3 * m * m * n + m ** 3)          # half of each of the two symmetric products
    return {"bytes": nbytes, "flops": flops}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"embed": _prepare_embed, "dembed": _prepare_embed, "logp": _prepare_logp, "dlogp": _prepare_logp, "muon": _prepare_muon}[case["op"]](case, gen)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda")


def _lib():
    from paper_2602_22445_b200 import binding
    return binding


def _prepare_embed(case, gen):
    n, V, H = case["n"], case["V"], case["H"]
    itype = torch.int64 if case["bits"] == 64 else torch.int32
    # text: few tokens are frequent, most are rare; which is which is spread over the vocabulary; one in fifty is padding
    rank = (torch.exp(_uniform(gen, n) * math.log(V)) - 1).long().clamp(0, V - 1)
    tokens = torch.randperm(V, generator=gen, device="cuda")[rank]
    s = {"case": case, "tokens": torch.where(_uniform(gen, n) < 0.02, torch.full_like(tokens, IGNORED), tokens).to(itype)}
    if case["op"] == "embed":
        s["table"] = (0.02 * _normal(gen, V, H)).to(DT[case["w"]])
        s["y"] = torch.zeros(n, H, dtype=DT[case["x"]], device="cuda")
    else:
        P, k = case["P"], case["k"]
        s["dy"] = (0.1 * _normal(gen, n, H)).to(DT[case["x"]])
        if case["ragged"]:          # cut points anywhere, so that some processes hold no tokens
            cuts = torch.randint(0, n + 1, (P - 1,), generator=gen, device="cuda").sort().values
            s["splits"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), n)])
        else:
            s["splits"] = None
        s["dtable"] = torch.zeros(-(-V * H // k), P, k, device="cuda")
    if own:
        s["lib"] = B = _lib()
        s["desc"] = B.make_embed_desc(V, H, DT[case["x"]], DT[case["w"]], P=case.get("P", 1), k=case.get("k"), scale=case["scale"])
        if case["op"] == "dembed":
            s["workspace"] = torch.empty(max(16, B.ftc_embedding_workspace_bytes(s["desc"], n)), dtype=torch.uint8, device="cuda")
    return s


def _prepare_logp(case, gen):
    rows, V, pad = case["rows"], case["V"], case["pad"]
    wide = torch.zeros(rows, V + pad, dtype=DT[case["x"]], device="cuda")
    x = wide[:, :V]
    # rows from flat to peaked; in some a part of the vocabulary is masked, in a few all but a handful of tokens
    spread = 1 + 3 * _uniform(gen, rows, 1)
    kept = torch.where(_uniform(gen, rows, 1) < 0.1, torch.where(_uniform(gen, rows, 1) < 0.2, 4 / V, 0.5), 1.1)
    for at in range(0, rows, 1024):
        part = slice(at, min(rows, at + 1024))
        z = _normal(gen, part.stop - at, V) * spread[part]
        z[_uniform(gen, part.stop - at, V) > kept[part]] = -math.inf
        z[:, 0] = 0.5               # something is left in every row
        x[part] = z
    tokens = torch.randint(0, V, (rows,), generator=gen, device="cuda")
    tokens = torch.where(x.gather(1, tokens[:, None])[:, 0].isinf(), 0, tokens)
    tokens = torch.where(_uniform(gen, rows) < 0.03, IGNORED, tokens)      # a part of each sequence is not scored
    s = {"case": case, "logits": x, "tokens": tokens.to(torch.int64 if case["bits"] == 64 else torch.int32)}
    if case["op"] == "logp":
        s["logprob"], s["entropy"], s["lse"] = (torch.zeros(rows, device="cuda") for _ in range(3))
        s["top_logprob"] = torch.zeros(rows, case["top"], device="cuda") if case["top"] else None
        s["top_token"] = torch.zeros(rows, case["top"], dtype=torch.int32, device="cuda") if case["top"] else None
    else:
        z = torch.cat([x[i:i + 1024].float() for i in range(0, rows, 1024)]) * case["scale"]
        s["lse"] = torch.logsumexp(z, 1)
        z -= s["lse"][:, None]
        s["entropy"] = -(z.exp() * z.clamp(min=-1e4)).sum(1)
        s["dlogprob"] = -1 / rows * (1 + 0.5 * _normal(gen, rows))
        s["dentropy"] = -0.01 / rows * (1 + 0.5 * _normal(gen, rows))
        s["dlogits"] = torch.zeros(rows, V, dtype=DT[case["x"]], device="cuda")
    if own:
        s["lib"] = _lib()
        s["desc"] = s["lib"].make_logprob_desc(V, DT[case["x"]], top=case.get("top", 0), scale=case["scale"])
    return s


def _prepare_muon(case, gen):
    s = {"case": case, "kinds": []}
    for count, rows, cols in _shapes(case):
        # gradients of a batch: channels of different sizes on both sides; the momentum after some hundred steps
        size = torch.exp(_normal(gen, count, 1, cols)) * torch.exp(0.5 * _normal(gen, count, rows, 1))
        n, padded = rows * cols, -(-rows * cols // BLOCK) * BLOCK
        kind = {"count": count, "rows": rows, "cols": cols}
        m = torch.zeros(count, padded, device="cuda")
        m[:, :n] = (1e-2 * size * _normal(gen, count, rows, cols)).view(count, n)
        kind["momentum"] = m
        grad = 1e-3 * size * _normal(gen, count, rows, cols)
        if case["k"]:           # sums of 64 processes, of which up to 4 have failed; few messages meet no failure-free subtree
            messages = -(-n // case["k"])
            st = torch.zeros(count, messages, 4, dtype=torch.int32, device="cuda")
            lost = _uniform(gen, count, messages) < 0.002
            st[:, :, 0] = torch.where(lost, 2 | 0xFF00 | 1 << 16, 1 << 16)
            st[:, :, 1] = torch.where(lost, 0, 64 - torch.randint(0, 5, (count, messages), generator=gen, device="cuda"))
            kind["status"] = st
            grad = 62 * grad
        else:
            kind["status"] = None
        kind["grad"] = grad.to(DT[case["g"]])
        weights = 0.02 * _normal(gen, count, rows, cols)
        kind["param"] = weights.to(DT[case["p"]])
        kind["master"] = weights if case["master"] else None
        s["kinds"].append(kind)
    s["scale"] = torch.tensor([0.75], device="cuda")         # the clip factor, where the norm left it
    if own:
        s["lib"] = B = _lib()
        s["momentum"] = torch.cat([d["momentum"].view(-1) for d in s["kinds"]])
        at = 0
        for d in s["kinds"]:
            size = d["momentum"].numel()
            d["momentum"] = s["momentum"][at:at + size].view(d["count"], -1)
            at += size
        s["plan"] = B.make_muon_plan([
            B.make_matrix(d["param"][i], d["grad"][i], master=d["master"][i] if case["master"] else None,
                          status=d["status"][i] if case["k"] else None, k=case["k"], lr_scale=_rate(d), weight_decay=DECAY)
            for d in s["kinds"] for i in range(d["count"])])
        # weights that are kept in 32 bits alone are updated with products of that precision
        s["hyper"] = B.make_muon(lr=LR, momentum=MOMENTUM, eps=EPS, steps=STEPS, nesterov=True, products=32 if case["p"] == "f32" else 16)
        s["workspace"] = torch.empty(B.ftc_muon_workspace_bytes(s["plan"]), dtype=torch.uint8, device="cuda")
    return s


def _rate(kind):
    """What a matrix's learning rate is multiplied by, so that its elements move about as far as AdamW's."""
    return 0.2 * math.sqrt(max(kind["rows"], kind["cols"]))


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"embed": _own_embed, "dembed": _own_dembed, "logp": _own_logp, "dlogp": _own_dlogp, "muon": _own_muon}[op](s)
    return {"embed": _plain_embed, "dembed": _plain_dembed, "logp": _plain_logp, "dlogp": _plain_dlogp, "muon": _plain_muon}[op](s)


def _own_embed(s):
    s["lib"].ftc_embedding_forward(s["desc"], s["tokens"], s["table"], s["y"])
    return s["y"]


def _own_dembed(s):
    s["lib"].ftc_embedding_backward(s["desc"], s["tokens"], s["dy"], s["splits"], s["dtable"], s["workspace"])
    return s["dtable"]


def _own_logp(s):
    s["lib"].ftc_token_logprobs(s["desc"], s["logits"], s["tokens"], s["logprob"], s["entropy"], s["lse"], s["top_logprob"], s["top_token"])
    return s["logprob"], s["entropy"], s["lse"], s["top_logprob"], s["top_token"]


def _own_dlogp(s):
    s["lib"].ftc_token_logprobs_backward(s["desc"], s["logits"], s["tokens"], s["lse"], s["entropy"], s["dlogprob"], s["dentropy"], s["dlogits"])
    return s["dlogits"]


def _own_muon(s):
    s["lib"].ftc_muon_step(s["hyper"], s["plan"], s["momentum"], s["scale"], s["workspace"])
    return [[d["param"], d["master"], d["momentum"]] for d in s["kinds"]]


def _plain_embed(s):
    case, t = s["case"], s["tokens"].long()
    there = (t >= 0) & (t < case["V"])
    rows = s["table"][t.clamp(0, case["V"] - 1)].float() * case["scale"]
    return torch.where(there[:, None], rows, torch.zeros_like(rows)).to(DT[case["x"]])


def _plain_dembed(s):
    case, t = s["case"], s["tokens"].long()
    n, V, H, P, k = (case[w] for w in ("n", "V", "H", "P", "k"))
    if s["splits"] is None:
        holder = torch.arange(n, device="cuda") // (n // P)
    else:
        holder = torch.repeat_interleave(torch.arange(P, device="cuda"), s["splits"][1:] - s["splits"][:-1], output_size=n)
    there = (t >= 0) & (t < V)
    rows = s["dy"].float() * (case["scale"] * there[:, None])
    sums = torch.zeros(P * V, H, device="cuda").index_add_(0, holder * V + t.clamp(0, V - 1), rows).view(P, V * H)
    S = -(-V * H // k)
    return torch.nn.functional.pad(sums, (0, S * k - V * H)).view(P, S, k).permute(1, 0, 2).contiguous()


def _plain_logp(s):
    case, t = s["case"], s["tokens"].long()
    V = case["V"]
    x = s["logits"].float()
    z = x * case["scale"]
    most = z.amax(1, keepdim=True)
    e = torch.exp(z - most)
    sums = e.sum(1, keepdim=True)
    lse = most + torch.log(sums)
    logp = z - lse
    entropy = -torch.where(e > 0, e / sums * logp, torch.zeros_like(e)).sum(1)
    given = torch.where((t >= 0) & (t < V), logp.gather(1, t.clamp(0, V - 1)[:, None])[:, 0], 0)
    if not case["top"]:
        return given, entropy, lse[:, 0], None, None
    # whole numbers in the logits' order, the lower index first where two are the same
    word = (x + 0.0).view(torch.int32).long()
    word = torch.where(word < 0, -(word & 0x7FFFFFFF), word)
    index = torch.topk(word * (1 << 32) + (V - 1 - torch.arange(V, device="cuda")), case["top"], dim=1).indices
    return given, entropy, lse[:, 0], logp.gather(1, index), index.int()


def _plain_dlogp(s):
    case, t = s["case"], s["tokens"].long()
    V = case["V"]
    logp = s["logits"].float() * case["scale"] - s["lse"][:, None]
    p = torch.exp(logp)
    there = (t >= 0) & (t < V)
    up = torch.where(there, s["dlogprob"], 0)[:, None]
    d = torch.where(p > 0, p * (-up - s["dentropy"][:, None] * (logp + s["entropy"][:, None])), torch.zeros_like(p))
    d.scatter_add_(1, t.clamp(0, V - 1)[:, None], up)
    return (d * case["scale"]).to(DT[case["x"]])


def _plain_muon(s):
    return [_plain_kind(s, d) for d in s["kinds"]]


def _plain_kind(s, d):
    """The matrices of one kind together, in place."""
    case, n = s["case"], d["rows"] * d["cols"]
    g = d["grad"].float().view(d["count"], n)
    m = d["momentum"][:, :n]
    if case["k"]:
        delivered = ((d["status"][:, :, 0] & 0xFF) == 0) & (d["status"][:, :, 1] > 0)
        share = torch.where(delivered, 1 / d["status"][:, :, 1].clamp(min=1).float(), 0).repeat_interleave(case["k"], 1)[:, :n]
        there = delivered.repeat_interleave(case["k"], 1)[:, :n]
        g = g * share * s["scale"]
        m1 = torch.where(there, m * MOMENTUM + g, m)
        u = torch.where(there, g + m1 * MOMENTUM, m)
    else:
        g = g * s["scale"]
        m1 = m * MOMENTUM + g
        u = g + m1 * MOMENTUM
    m.copy_(m1)
    x = (u / (u.square().sum(1, keepdim=True).sqrt() + EPS)).view(d["count"], d["rows"], d["cols"])
    if d["rows"] > d["cols"]:
        x = x.transpose(1, 2)
    a, b, c = QUINTIC
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    if d["rows"] > d["cols"]:
        x = x.transpose(1, 2)
    rate = LR * _rate(d)
    weight = d["master"] if case["master"] else d["param"]
    p = weight.float() * (1 - rate * DECAY) - rate * x
    weight.copy_(p)
    if case["master"]:
        d["param"].copy_(p)
    return [d["param"], d["master"], d["momentum"]]


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "dembed": _exact_dembed, "logp": _exact_logp, "dlogp": _exact_dlogp, "muon": _exact_muon}[case["op"]](case, s)


def _exact_embed(case, s):
    y = torch.zeros(case["n"], case["H"], dtype=torch.float64, device="cuda")
    at = ((s["tokens"] >= 0) & (s["tokens"] < case["V"])).nonzero()[:, 0]
    y[at] = s["table"][s["tokens"][at].long()].double().mul_(case["scale"])
    return y


def _exact_dembed(case, s):
    V, H, P, k, n = (case[w] for w in ("V", "H", "P", "k", "n"))
    cuts = s["splits"].tolist() if s["splits"] is not None else [p * (n // P) for p in range(P + 1)]
    out = torch.zeros(-(-V * H // k), P, k, dtype=torch.float64, device="cuda")
    for p in range(P):              # one process after the other, by a product with the tokens' indicator (sparse)
        t = s["tokens"][cuts[p]:cuts[p + 1]].long()
        at = ((t >= 0) & (t < V)).nonzero()[:, 0]
        if at.numel():
            which = torch.sparse_coo_tensor(torch.stack([t[at], at]), torch.full((at.numel(),), case["scale"], dtype=torch.float64, device="cuda"), (V, t.numel()))
            sums = torch.sparse.mm(which, s["dy"][cuts[p]:cuts[p + 1]].double()).reshape(-1)
            whole = V * H // k * k
            out[:whole // k, p] = sums[:whole].view(-1, k)
            if whole < V * H:
                out[-1, p, :V * H - whole] = sums[whole:]
    return out


def _exact_logp(case, s):
    V, top = case["V"], case["top"]
    found = []
    for x, t in zip(s["logits"].split(512), s["tokens"].long().split(512)):
        z = x.double() * case["scale"]
        lse = torch.logsumexp(z, 1)
        p = torch.softmax(z, 1)
        given = torch.stack([lse.new_zeros(()) if not 0 <= j < V else z[i, j] - lse[i] for i, j in enumerate(t.tolist())])
        row = [given, torch.special.entr(p).sum(1), lse]
        if top:
            order = torch.sort(z, dim=1, descending=True, stable=True)
            row += [order.values[:, :top] - lse[:, None], order.indices[:, :top].int()]
        found.append(row)
    return [torch.cat(part) for part in zip(*found)] + [None] * (0 if top else 2)


def _exact_dlogp(case, s):
    d = torch.empty(case["rows"], case["V"], dtype=torch.float64, device="cuda")
    for at in range(0, case["rows"], 512):
        part = slice(at, min(case["rows"], at + 512))
        z = s["logits"][part].double() * case["scale"]
        p = torch.exp(z - s["lse"][part, None].double())
        surprise = torch.where(p > 0, s["lse"][part, None].double() - z, 0)
        down = s["dentropy"][part, None].double() * p * (surprise - s["entropy"][part, None].double())
        scored = (s["tokens"][part] >= 0) & (s["tokens"][part] < case["V"])
        one = torch.zeros_like(p)
        rows = scored.nonzero()[:, 0]
        one[rows, s["tokens"][part][rows].long()] = 1
        d[part] = case["scale"] * (down + (s["dlogprob"][part].double() * scored)[:, None] * (one - p))
    return d


def _exact_muon(case, s):
    out = []
    for d in s["kinds"]:
        n = d["rows"] * d["cols"]
        param, momentum = (d["master"] if case["master"] else d["param"]).double(), d["momentum"].double()
        for i in range(d["count"]):
            g, m = d["grad"][i].double().reshape(-1) * s["scale"].double(), momentum[i, :n]
            u = g + MOMENTUM * (g + MOMENTUM * m)
            new = g + MOMENTUM * m
            if case["k"]:
                st = d["status"][i].long()[torch.arange(n, device="cuda") // case["k"]]
                there = ((st[:, 0] & 255) == 0) & (st[:, 1] > 0)
                g = g / st[:, 1].clamp(min=1)
                new = torch.where(there, g + MOMENTUM * m, m)
                u = torch.where(there, g + MOMENTUM * new, m)
            momentum[i, :n] = new
            x = u.view(d["rows"], d["cols"])
            x = x / (torch.linalg.matrix_norm(x) + EPS)
            for _ in range(STEPS):          # the same polynomial, by the smaller side's products
                if d["rows"] <= d["cols"]:
                    q = x @ x.mT
                    x = torch.addmm(x, torch.addmm(q, q, q, beta=QUINTIC[1], alpha=QUINTIC[2]), x, beta=QUINTIC[0])
                else:
                    q = x.mT @ x
                    x = torch.addmm(x, x, torch.addmm(q, q, q, beta=QUINTIC[1], alpha=QUINTIC[2]), beta=QUINTIC[0])
            param[i] -= LR * _rate(d) * (DECAY * param[i] + x)
        out.append([param, param if case["master"] else None, momentum])
    return out
