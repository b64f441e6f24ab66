"""Workloads of the training operators next to the collectives: layer norm forward and backward with the weight
gradients of each simulated process, the global gradient norm, and AdamW over many tensors.

A case is a dict of plain values. `run` computes it in plain torch (32-bit arithmetic, rounded once at the end) or, with
`own` set, through this repository's library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SZ = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                    # elements that share a scale where the optimizer's states are held in 8 bits
TINY = 2.0 ** -126             # smallest scale (smallest normal float32)
LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.95, 1e-8, 0.1, 1.0
NORM_EPS = 1e-5


# ---- cases ----------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the last norm of a small model on a handful of tokens: a call's latency
        {"name": "norm fwd, 8 rows", "op": "fwd", "rows": 8, "H": 1024, "x": "bf16", "w": "bf16", "pad": 0},
        # packed sequences of a model with an odd width, rows with a stride of their own (a slice of a wider tensor)
        {"name": "norm fwd, odd width", "op": "fwd", "rows": 5003, "H": 1367, "x": "f16", "w": "f32", "pad": 9},
        # a training batch of 32k tokens
        {"name": "norm fwd, 32k tokens", "op": "fwd", "rows": 32768, "H": 4096, "x": "bf16", "w": "f32", "pad": 0},
        # 8 processes with 8 rows each, messages of 16 elements: small and float32 throughout
        {"name": "norm bwd, 8 processes", "op": "bwd", "rows": 64, "H": 512, "x": "f32", "w": "f32", "P": 8, "k": 16, "ragged": False, "pad": 0},
        # packed sequences divided unevenly over 64 processes (some have no rows), a width that no wide vector divides
        {"name": "norm bwd, ragged processes", "op": "bwd", "rows": 8191, "H": 2050, "x": "bf16", "w": "f32", "P": 64, "k": 8, "ragged": True, "pad": 0},
        # a training batch of 32k tokens over 64 processes, messages of 32 elements
        {"name": "norm bwd, 32k tokens", "op": "bwd", "rows": 32768, "H": 4096, "x": "bf16", "w": "bf16", "P": 64, "k": 32, "ragged": False, "pad": 0},
        # the gradients of two norms and a few small matrices: latency
        {"name": "grad norm, small", "op": "gnorm", "layers": 1, "H": 64, "F": 256, "g": "f32", "k": 0, "packed": False},
        # the delivered messages of a 24-layer model, each with its status record
        {"name": "grad norm, delivered", "op": "gnorm", "layers": 24, "H": 1024, "F": 4096, "g": "f32", "k": 32, "packed": False},
        # a toy model's whole update in float32
        {"name": "adamw 32 bits, small", "op": "adamw", "layers": 2, "H": 64, "F": 256, "p": "f32", "master": False, "g": "f32", "bits": 32, "k": 0, "packed": False},
        # bf16 weights with a float32 copy, delivered messages of 32 elements as gradients
        {"name": "adamw 32 bits, delivered", "op": "adamw", "layers": 12, "H": 1024, "F": 4096, "p": "bf16", "master": True, "g": "f32", "bits": 32, "k": 32, "packed": False},
        # odd widths, tensors packed back to back (views that no vector load fits), 8-bit states
        {"name": "adamw 8 bits, packed odd", "op": "adamw", "layers": 8, "H": 601, "F": 1803, "p": "f32", "master": False, "g": "bf16", "bits": 8, "k": 0, "packed": True},
        # 24 layers in bf16 with a float32 copy and 8-bit states
        {"name": "adamw 8 bits, 24 layers", "op": "adamw", "layers": 24, "H": 1024, "F": 4096, "p": "bf16", "master": True, "g": "bf16", "bits": 8, "k": 0, "packed": False},
    ]


SKIPPED = 3072                 # a size that belongs to other benchmarks


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 8 if n == SKIPPED else n


def draw(rng):
    op = rng.choice(["fwd", "bwd", "gnorm", "adamw", "adamw"])
    if op in ("fwd", "bwd"):
        H = _spread(rng, 24, 16384)
        if rng.random() < 0.5:
            H = max(8, H // 8 * 8) + (8 if H // 8 * 8 == SKIPPED else 0)
        c = {"op": op, "rows": _spread(rng, 1, min(32768, 32768 * 4096 // H)), "H": H, "x": rng.choice(["f32", "bf16", "bf16", "f16"]), "pad": rng.choice([0, 0, 3, 8])}
        c["w"] = rng.choice(["f32", c["x"]])
        if c["x"] == "f32":
            c["rows"] = max(1, c["rows"] // 2)
        if op == "bwd":
            c["P"] = min(_spread(rng, 1, 1024), max(1, c["rows"]))
            c["k"] = rng.choice([4, 8, 16, 32, 32, 7])
            c["ragged"] = rng.random() < 0.5
            if not c["ragged"]:
                c["rows"] = max(1, c["rows"] // c["P"]) * c["P"]
        if c["rows"] == SKIPPED:
            c["rows"] -= c.get("P", 1)
        return c
    H = _spread(rng, 24, 1024)
    if rng.random() < 0.5:
        H = max(8, H // 8 * 8)
    F = H * rng.randint(1, 4)
    F += 8 if F == SKIPPED else 0
    c = {"op": op, "layers": rng.randint(1, 24 if op == "gnorm" else 12), "H": H, "F": F, "k": rng.choice([0, 0, 4, 32, 7]), "packed": rng.random() < 0.3}
    c["g"] = "f32" if c["k"] else rng.choice(["f32", "bf16", "f16"])
    if op == "adamw":
        c["p"] = rng.choice(["f32", "bf16", "bf16", "f16"])
        c["master"] = c["p"] != "f32" and rng.random() < 0.6
        c["bits"] = rng.choice([8, 32])
    return c


def _sizes(case):
    """Elements of each tensor: a norm's two vectors, two matrices and their biases in each layer."""
    H, F = case["H"], case["F"]
    return [H, H, H * F, F, F * H, H] * case["layers"]


def _decays(case):
    """Matrices decay, vectors do not."""
    return [0.0, 0.0, DECAY, 0.0, DECAY, 0.0] * case["layers"]


def _places(sizes, each):
    """Where each tensor begins in a buffer of all of them, at multiples of `each`, and the buffer's length."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += -(-n // each) * each
    return places, at


def work(case):
    if case["op"] in ("fwd", "bwd"):
        n, rows = case["rows"] * case["H"], case["rows"]
        if case["op"] == "fwd":
            return {"bytes": 2 * n * SZ[case["x"]] + 8 * rows + 2 * case["H"] * SZ[case["w"]], "flops": 8 * n}
        out = 8 * case["P"] * (-(-case["H"] // case["k"]) * case["k"])
        return {"bytes": 3 * n * SZ[case["x"]] + 8 * rows + case["H"] * SZ[case["w"]] + out, "flops": 14 * n}
    sizes = _sizes(case)
    n = sum(sizes)
    messages = sum(-(-s // case["k"]) for s in sizes) if case["k"] else 0
    if case["op"] == "gnorm":
        return {"bytes": n * SZ[case["g"]] + 16 * messages + 4 * (2 + len(sizes)), "flops": 2 * n}
    per = SZ[case["g"]] + (SZ[case["p"]] + 8 if case["master"] else 2 * SZ[case["p"]]) + (16 if case["bits"] == 32 else 4)
    read_out = n * (2 + 8) if case["bits"] == 8 else 0           # the 8-bit states, read out in 32 bits
    scales = sum(-(-s // BLOCK) for s in sizes) * (16 + 8) if case["bits"] == 8 else 0
    return {"bytes": n * per + read_out + scales + 16 * messages, "flops": 16 * n}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return _prepare_norm(case, seed, gen) if case["op"] in ("fwd", "bwd") else _prepare_tensors(case, seed, gen)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _rows(values, dtype, pad):
    """The rows as a tensor of `dtype`; with `pad`, as a slice of a wider one."""
    wide = torch.zeros(values.shape[0], values.shape[1] + pad, dtype=dtype, device="cuda")
    wide[:, :values.shape[1]] = values
    return wide[:, :values.shape[1]]


def _prepare_norm(case, seed, gen):
    rows, H, dt = case["rows"], case["H"], DT[case["x"]]
    # a residual stream: a mean of its own in each channel, a few channels far larger than the rest
    x = _normal(gen, rows, H).mul_(1 + 10 * (torch.rand(H, generator=gen, device="cuda") < 0.01)).add_(0.3 * _normal(gen, H) + 0.2)
    s = {"case": case, "x": _rows(x, dt, case["pad"]), "gamma": (1 + 0.1 * _normal(gen, H)).to(DT[case["w"]])}
    if own:
        from paper_2602_22445_b200 import binding as B
        s["lib"], s["desc"] = B, B.make_norm_desc(H, dt, DT[case["w"]], P=case.get("P", 1), k=case.get("k", H), eps=NORM_EPS)
    if case["op"] == "fwd":
        s["beta"] = (0.1 * _normal(gen, H)).to(DT[case["w"]])
        s["y"] = torch.zeros(rows, H, dtype=dt, device="cuda")
        s["mean"], s["rstd"] = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        return s
    P, S = case["P"], -(-H // case["k"])
    s["dy"] = _rows(0.1 * _normal(gen, rows, H), dt, case["pad"])
    xf = s["x"].float()
    s["mean"] = xf.mean(1)
    s["rstd"] = 1 / torch.sqrt((xf - s["mean"][:, None]).square().mean(1) + NORM_EPS)
    s["splits"] = None
    if case["ragged"]:          # cut points anywhere, so that some processes hold no rows
        cuts = torch.randint(0, rows + 1, (P - 1,), generator=gen, device="cuda").sort().values
        s["splits"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), rows)])
    s["dx"] = torch.zeros(rows, H, dtype=dt, device="cuda")
    s["dgamma"], s["dbeta"] = torch.zeros(S, P, case["k"], device="cuda"), torch.zeros(S, P, case["k"], device="cuda")
    if own:
        s["workspace"] = torch.empty(max(16, B.ftc_layernorm_workspace_bytes(s["desc"], rows)), dtype=torch.uint8, device="cuda")
    return s


def _prepare_tensors(case, seed, gen):
    sizes = _sizes(case)
    places, total = _places(sizes, 1 if case["packed"] else 64)
    used = torch.zeros(total, device="cuda")
    for n, at in zip(sizes, places):
        used[at:at + n] = 1
    s = {"case": case, "sizes": sizes, "places": places}

    def views(flat):
        return [flat[at:at + n] for n, at in zip(sizes, places)]

    s["grad"] = views(1e-2 * _normal(gen, total).mul_(used).to(DT[case["g"]]) if not case["k"] else 0.6 * _normal(gen, total).mul_(used))
    s["status"] = [None] * len(sizes)
    if case["k"]:               # 64 processes, of which up to 4 have failed; few messages meet no failure-free subtree
        s["status"] = []
        for n in sizes:
            st = torch.zeros(-(-n // case["k"]), 4, dtype=torch.int32, device="cuda")
            lost = torch.rand(st.shape[0], generator=gen, device="cuda") < 0.002
            st[:, 0] = torch.where(lost, 2 | 0xFF00 | 1 << 16, 1 << 16)
            st[:, 1] = torch.where(lost, 0, 64 - torch.randint(0, 5, (st.shape[0],), generator=gen, device="cuda"))
            s["status"].append(st)
    if case["op"] == "gnorm":
        s["norm"], s["norms"] = torch.zeros(2, device="cuda"), torch.zeros(len(sizes), device="cuda")
    else:
        weights = 0.02 * _normal(gen, total).mul_(used)
        s["flat"] = weights.to(DT[case["p"]])
        s["flat32"] = weights if case["master"] else None
        s["param"] = views(s["flat"])
        s["master"] = views(s["flat32"]) if case["master"] else [None] * len(sizes)
        s["decay"] = _decays(case)
        s["at"], padded = _places(sizes, BLOCK)
        live = torch.zeros(padded, device="cuda")
        for n, at in zip(sizes, s["at"]):
            live[at:at + n] = 1
        # states after some hundred steps: the average gradient small beside its mean square, sizes over several decades
        width = torch.exp(1.5 * _normal(gen, padded))
        m, v = 2e-3 * width * _normal(gen, padded) * live, (8e-3 * width).square() * live
        if case["bits"] == 8:
            (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _encode_m(m.view(-1, BLOCK)), _encode_r(torch.sqrt(v).view(-1, BLOCK))
            s["m_out"], s["v_out"] = torch.zeros(padded, device="cuda"), torch.zeros(padded, device="cuda")
        else:
            s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
        s["step"] = 400
        s["scale"] = torch.tensor([0.75], device="cuda")         # the clip factor, where the norm left it
    if own:
        from paper_2602_22445_b200 import binding as B
        s["lib"] = B
        s["table"] = B.make_param_table([
            B.make_param(s["param"][i] if case["op"] == "adamw" else None, g, master=s["master"][i] if case["op"] == "adamw" else None,
                         status=s["status"][i], k=case["k"], weight_decay=s["decay"][i] if case["op"] == "adamw" else 0.0)
            for i, g in enumerate(s["grad"])])
        if case["op"] == "gnorm":
            s["workspace"] = torch.empty(max(16, B.ftc_grad_norm_workspace_bytes(s["table"])), dtype=torch.uint8, device="cuda")
        else:
            s["hyper"] = B.make_adamw(lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, step=s["step"])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"fwd": _own_fwd, "bwd": _own_bwd, "gnorm": _own_gnorm, "adamw": _own_adamw}[op](s)
    return {"fwd": _plain_fwd, "bwd": _plain_bwd, "gnorm": _plain_gnorm, "adamw": _plain_adamw}[op](s)


def _own_fwd(s):
    s["lib"].ftc_layernorm_forward(s["desc"], s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"])
    return s["y"], s["mean"], s["rstd"]


def _own_bwd(s):
    s["lib"].ftc_layernorm_backward(s["desc"], s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["splits"],
                                    s["dx"], s["dgamma"], s["dbeta"], s["workspace"])
    return s["dx"], s["dgamma"], s["dbeta"]


def _own_gnorm(s):
    s["lib"].ftc_grad_norm(s["table"], MAX_NORM, s["norm"], s["norms"], s["workspace"])
    return s["norm"], s["norms"]


def _own_adamw(s):
    s["lib"].ftc_adamw_step(s["hyper"], s["table"], s["m"], s["v"], s["m_scale"], s["v_scale"], s["scale"])
    if s["case"]["bits"] == 32:
        return s["flat"], s["flat32"], s["m"], s["v"]
    s["lib"].ftc_adamw_states(s["table"], s["m"], s["v"], s["m_scale"], s["v_scale"], s["m_out"], s["v_out"])
    return s["flat"], s["flat32"], s["m_out"], s["v_out"]


def _plain_fwd(s):
    x = s["x"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1 / torch.sqrt(xc.square().mean(1) + NORM_EPS)
    y = xc * rstd[:, None] * s["gamma"].float() + s["beta"].float()
    return y.to(s["x"].dtype), mean, rstd


def _plain_bwd(s):
    case = s["case"]
    rows, H, P, k = case["rows"], case["H"], case["P"], case["k"]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * rstd
    a = dy * s["gamma"].float()
    dx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    return dx.to(s["x"].dtype), _messages(_by_process(dy * xh, s["splits"], P), k), _messages(_by_process(dy, s["splits"], P), k)


def _by_process(rows, splits, P):
    """Sums of the rows that each process holds, [P][H]."""
    if splits is None:
        return rows.view(P, -1, rows.shape[1]).sum(1)
    holder = torch.repeat_interleave(torch.arange(P, device=rows.device), splits[1:] - splits[:-1], output_size=rows.shape[0])
    return torch.zeros(P, rows.shape[1], dtype=rows.dtype, device=rows.device).index_add_(0, holder, rows)


def _messages(sums, k):
    """[P][H] as messages of k elements, [ceil(H/k)][P][k], the last one filled up with zeros."""
    P, H = sums.shape
    S = -(-H // k)
    return torch.nn.functional.pad(sums, (0, S * k - H)).view(P, S, k).permute(1, 0, 2).contiguous()


def _share(status, k, n):
    """1 / processes included for each element, 0 where its message was not delivered."""
    count = torch.where((status[:, 0] & 0xFF) == 0, status[:, 1], 0).float()
    return torch.where(count > 0, 1 / count, torch.zeros_like(count)).repeat_interleave(k)[:n]


def _gradient(s, i):
    g = s["grad"][i].float()
    return g * _share(s["status"][i], s["case"]["k"], g.numel()) if s["case"]["k"] else g


def _plain_gnorm(s):
    norms = torch.sqrt(torch.stack([_gradient(s, i).square().sum() for i in range(len(s["sizes"]))]))
    norm = torch.sqrt(norms.square().sum())
    return torch.stack([norm, torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))]), norms


def _nearest_root(x, most):
    """The whole number c with (c - 1/2)^2 <= x < (c + 1/2)^2, at most `most`."""
    c = torch.floor(torch.sqrt(x) + 0.5)
    c = torch.where(c * c - c + 0.25 > x, c - 1, c)
    c = torch.where(c * c + c + 0.25 <= x, c + 1, c)
    return c.clamp(0, most)


def _encode_m(m):
    """Averages [blocks][256] as signed 8-bit numbers, m = c |c| scale / 127^2, and the scales."""
    scale = m.abs().amax(1).clamp(min=TINY)
    c = _nearest_root(m.abs() * (1 / scale)[:, None] * 16129.0, 127)
    return torch.where(m < 0, -c, c).to(torch.int8).view(-1), scale


def _encode_r(r):
    """Roots of the mean squares [blocks][256] as 8-bit numbers, r = c^2 scale / 255^2, and the scales."""
    scale = r.amax(1).clamp(min=TINY)
    c = _nearest_root(r * (1 / scale)[:, None] * 65025.0, 255)
    return torch.where(r > 0, c.clamp(min=1), c).to(torch.uint8).view(-1), scale


def _decode_m(codes, scale):
    c = codes.view(-1, BLOCK).float()
    return c * c.abs() * (scale * (1 / 16129))[:, None]


def _decode_v(codes, scale):
    c = codes.view(-1, BLOCK).float()
    r = c * c * (scale * (1 / 65025))[:, None]
    return r * r


def _plain_one(s, i):
    """AdamW on tensor i, in place; its factors are float32 numbers."""
    case, n, lo = s["case"], s["sizes"][i], s["at"][i]
    t, one = s["step"], np.float32(1)
    lr, fix1, fix2 = np.float32(LR), np.float32(1 / (1 - BETA1 ** t)), float(np.float32(1 / math.sqrt(1 - BETA2 ** t)))
    keep, rate = float(one - lr * np.float32(s["decay"][i])), float(lr * fix1)
    blocks = slice(lo // BLOCK, lo // BLOCK + -(-n // BLOCK))
    hi = blocks.stop * BLOCK
    if case["bits"] == 8:
        m = _decode_m(s["m"][lo:hi], s["m_scale"][blocks]).view(-1)[:n]
        v = _decode_v(s["v"][lo:hi], s["v_scale"][blocks]).view(-1)[:n]
    else:
        m, v = s["m"][lo:lo + n], s["v"][lo:lo + n]
    weight = s["master"][i] if case["master"] else s["param"][i]
    p = weight.float()
    g = _gradient(s, i) * s["scale"]
    m1 = m * BETA1 + g * (1 - BETA1)
    v1 = v * BETA2 + g * g * (1 - BETA2)
    p1 = p * keep - m1 / (torch.sqrt(v1) * fix2 + EPS) * rate
    if case["k"]:
        there = _share(s["status"][i], case["k"], n) > 0
        m1, v1, p1 = torch.where(there, m1, m), torch.where(there, v1, v), torch.where(there, p1, p)
    if case["bits"] == 8:
        fill = (0, hi - lo - n)
        new = _encode_m(torch.nn.functional.pad(m1, fill).view(-1, BLOCK)) + _encode_r(torch.nn.functional.pad(torch.sqrt(v1), fill).view(-1, BLOCK))
        old = (s["m"][lo:hi], s["m_scale"][blocks], s["v"][lo:hi], s["v_scale"][blocks])
        if case["k"]:           # a block that no message was delivered for stays as it is
            some = torch.nn.functional.pad(there, fill).view(-1, BLOCK).any(1)
            new = [torch.where(w, x, y) for w, x, y in zip((some.repeat_interleave(BLOCK), some) * 2, new, old)]
        for x, y in zip(old, new):
            x.copy_(y)
    else:
        m.copy_(m1)
        v.copy_(v1)
    weight.copy_(p1)
    if case["master"]:
        s["param"][i].copy_(p1)


def _plain_adamw(s):
    for i in range(len(s["sizes"])):
        _plain_one(s, i)
    if s["case"]["bits"] == 32:
        return s["flat"], s["flat32"], s["m"], s["v"]
    return s["flat"], s["flat32"], _decode_m(s["m"], s["m_scale"]).view(-1), _decode_v(s["v"], s["v_scale"]).view(-1)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    if case["op"] == "fwd":
        x = s["x"].to(d)
        mean, var = x.mean(1), x.var(1, unbiased=False)
        rstd = (var + NORM_EPS).rsqrt()
        return (torch.addcmul(s["beta"].to(d), (x - mean[:, None]) * rstd[:, None], s["gamma"].to(d)), mean, rstd)
    if case["op"] == "bwd":
        # the derivative of the forward pass along dy, written with the projection off 1 and off the normed row
        H, P, k = case["H"], case["P"], case["k"]
        dy, unit = s["dy"].to(d), (s["x"].to(d) - s["mean"].to(d)[:, None]) * s["rstd"].to(d)[:, None]
        up = dy * s["gamma"].to(d)
        dx = s["rstd"].to(d)[:, None] * (up - (up.sum(1) / H)[:, None] - unit * ((up * unit).sum(1) / H)[:, None])
        cuts = s["splits"].tolist() if s["splits"] is not None else [p * (case["rows"] // P) for p in range(P + 1)]

        def laid_out(rows):
            out = torch.zeros(P, -(-H // k) * k, dtype=d, device="cuda")
            for p in range(P):
                out[p, :H] = rows[cuts[p]:cuts[p + 1]].sum(0)
            return out.view(P, -1, k).transpose(0, 1).contiguous()
        return dx, laid_out(dy * unit), laid_out(dy)

    def mean_gradient(i):
        g = s["grad"][i].to(d)
        if not case["k"]:
            return g, torch.ones_like(g, dtype=torch.bool)
        which = torch.arange(g.numel(), device="cuda") // case["k"]
        st = s["status"][i].long()[which]
        there = ((st[:, 0] & 255) == 0) & (st[:, 1] > 0)
        return torch.where(there, g / st[:, 1].clamp(min=1).to(d), torch.zeros_like(g)), there

    if case["op"] == "gnorm":
        norms = torch.stack([torch.linalg.vector_norm(mean_gradient(i)[0]) for i in range(len(s["sizes"]))])
        total = torch.linalg.vector_norm(norms)
        return torch.stack([total, (MAX_NORM / total).clamp(max=1.0)]), norms

    flat, m_all, v_all = (s["flat32"] if case["master"] else s["flat"]).to(d), s["m"].to(d), s["v"].to(d)
    if case["bits"] == 8:
        m_all = (m_all / 127).square() * m_all.sign() * s["m_scale"].to(d).repeat_interleave(BLOCK)
        v_all = ((v_all / 255).square() * s["v_scale"].to(d).repeat_interleave(BLOCK)).square()
    t = s["step"]
    for i, n in enumerate(s["sizes"]):
        g, there = mean_gradient(i)
        g = g * s["scale"].to(d)
        m, v, p = (a[at:at + n] for a, at in ((m_all, s["at"][i]), (v_all, s["at"][i]), (flat, s["places"][i])))
        m1, v1 = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
        p1 = p - LR * s["decay"][i] * p - LR * (m1 / (1 - BETA1 ** t)) / ((v1 / (1 - BETA2 ** t)).sqrt() + EPS)
        for old, new in ((m, m1), (v, v1), (p, p1)):
            old.copy_(torch.where(there, new, old))
    if case["bits"] == 8:
        mb, rb = m_all.view(-1, BLOCK), v_all.sqrt().view(-1, BLOCK)
        ms, rs = mb.abs().amax(1, keepdim=True).clamp(min=TINY), rb.amax(1, keepdim=True).clamp(min=TINY)
        c = torch.floor(127 * (mb.abs() / ms).sqrt() + 0.5)
        m_all = (mb.sign() * (c / 127) ** 2 * ms).view(-1)
        c = torch.floor(255 * (rb / rs).sqrt() + 0.5)
        v_all = ((torch.where(rb > 0, c.clamp(min=1), c) / 255) ** 2 * rs).square().view(-1)
    return flat, flat if case["master"] else None, m_all, v_all
