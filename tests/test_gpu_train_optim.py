"""Gradient norm and AdamW over many tensors on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import train_oracle as O

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 3e-3, 0.9, 0.95, 1e-8
SIZES = [1, 7, 255, 256, 257, 0, 1000, 4096, 12345, 64, 2048]


def tensor(rng, n, dtype, offset, spread):
    import torch
    t = torch.full((n + offset + 8,), 77.0, dtype=getattr(torch, dtype), device="cuda")[offset:offset + n]
    t.copy_(torch.from_numpy(spread * rng.standard_normal(n)))
    return t


def records(rng, n, k, lost=0.3):
    import torch
    S = -(-n // k)
    st = np.zeros((S, 4), dtype=np.uint32)
    st[:, 1] = rng.integers(1, 70, S)
    code = np.where(rng.random(S) < lost, rng.integers(1, 7, S), 0)
    st[:, 0] = code | (rng.integers(0, 4, S) << 8) | (1 << 16)
    st[code != 0, 1] = 0
    if S > 3:
        st[2, :2] = (1 << 16, 0)                # delivered, but nobody included: counts as not delivered
    return torch.from_numpy(st.view(np.int32)).cuda()


class Job:
    """Tensors of one table, their states and their copies in 64 bits."""

    def __init__(self, seed, sizes, p="float32", g="float32", master=False, k=0, bits=32, offset=0, fresh=False):
        import torch
        rng = np.random.default_rng(seed)
        self.sizes, self.p, self.bits, self.k = sizes, p, bits, k
        self.grad = [tensor(rng, n, g, offset, 0.3 * 10.0 ** rng.uniform(-4, 0)) for n in sizes]
        self.param = [tensor(rng, n, p, offset, 0.1) for n in sizes]
        self.master = [tensor(rng, n, "float32", offset, 0.1) if master else None for n in sizes]
        self.status = [records(rng, n, k) if k else None for n in sizes]
        self.decay = [0.1 if i % 2 else 0.0 for i in range(len(sizes))]
        self.lr_scale = [1.0 if i % 3 else 0.5 for i in range(len(sizes))]
        self.table = B.make_param_table([
            B.make_param(*t, status=s, k=k, lr_scale=r, weight_decay=d)
            for *t, s, r, d in zip(self.param, self.grad, self.master, self.status, self.lr_scale, self.decay)])
        self.at = np.cumsum([0] + [-(-n // 256) * 256 for n in sizes])
        n, nb = int(self.at[-1]), int(self.at[-1]) // 256
        assert self.table.blocks == nb
        live = np.zeros(n)
        for a, s in zip(self.at, sizes):
            live[a:a + s] = 0 if fresh else 1
        if bits == 32:
            self.m = torch.from_numpy((1e-2 * rng.standard_normal(n) * live).astype(np.float32)).cuda()
            self.v = torch.from_numpy(((2e-2 * rng.standard_normal(n)) ** 2 * live).astype(np.float32)).cuda()
            self.ms = self.vs = None
        else:
            self.m = torch.from_numpy((rng.integers(-127, 128, n) * live).astype(np.int8)).cuda()
            self.v = torch.from_numpy((rng.integers(0, 256, n) * live).astype(np.uint8)).cuda()
            some = live.reshape(-1, 256).any(1)
            self.ms = torch.from_numpy((1e-2 * np.exp(rng.standard_normal(nb)) * some).astype(np.float32)).cuda()
            self.vs = torch.from_numpy((2e-2 * np.exp(rng.standard_normal(nb)) * some).astype(np.float32)).cuda()

    def states(self):
        m, v = self.m.cpu().numpy(), self.v.cpu().numpy()
        if self.bits == 32:
            return m.astype(np.float64), v.astype(np.float64)
        return O.decode(m, v, self.ms.double().cpu().numpy(), self.vs.double().cpu().numpy())

    def weights(self):
        return [(w if w is not None else p).double().cpu().numpy() for w, p in zip(self.master, self.param)]

    def gradients(self):
        return [g.double().cpu().numpy() for g in self.grad]

    def shares(self):
        return [O.shares(None if s is None else s.cpu().numpy().view(np.uint32), self.k, n) for s, n in zip(self.status, self.sizes)]

    def step(self, step, scale=None, stream=None, lr=LR, eps=EPS):
        B.ftc_adamw_step(B.make_adamw(lr, B1, B2, eps, step), self.table, self.m, self.v, self.ms, self.vs, scale, stream=stream)

    def check(self, before, step, scale=1.0):
        """The state after one step from `before` = (weights, states)."""
        (w0, (m0, v0)), w1, (m1, v1) = before, self.weights(), self.states()
        codes = None if self.bits == 32 else (self.m.cpu().numpy().astype(np.float64), self.v.cpu().numpy().astype(np.float64))
        for i, (n, a) in enumerate(zip(self.sizes, self.at)):
            share, here = self.shares()[i], slice(a, a + n)
            want, off = O.adamw(w0[i], self.gradients()[i], m0[here], v0[here], LR * self.lr_scale[i], B1, B2, EPS, step, self.decay[i], share, scale)
            f32 = self.master[i] is not None or self.p == "float32"
            O.assert_within(w1[i], want[0], off[0], "float32" if f32 else self.p, f"weights of tensor {i}")
            if self.master[i] is not None:
                assert (self.param[i] == self.master[i].to(self.param[i].dtype))[share_mask(share)].all()
            if self.bits == 32:
                O.assert_within(m1[here], want[1], off[1], what=f"m of tensor {i}")
                O.assert_within(v1[here], want[2], off[2], what=f"v of tensor {i}")
            else:
                for b in range(a // 256, a // 256 + -(-n // 256)):
                    lo, hi = b * 256, min(b * 256 + 256, a + n)
                    q = slice(lo - a, hi - a)
                    if not (share[q] > 0).any():
                        assert (m1[lo:hi] == m0[lo:hi]).all() and (v1[lo:hi] == v0[lo:hi]).all()
                        continue
                    check_codes(codes[0][lo:hi], float(self.ms[b]), np.abs(want[1][q]), off[1][q], 127, 0)
                    assert (np.sign(codes[0][lo:hi]) * np.sign(want[1][q]) >= 0).all()
                    check_codes(codes[1][lo:hi], float(self.vs[b]), np.sqrt(want[2][q]), off[2][q] / np.maximum(2 * np.sqrt(want[2][q]), 1e-30), 255, 1)


def share_mask(share):
    import torch
    return torch.from_numpy(share > 0).cuda()


def check_codes(codes, scale, values, off, most, least):
    """codes of one block are the whole numbers nearest to most * sqrt(values / scale), as far as float32 can tell."""
    top = max(values.max(), O.TINY)
    assert abs(scale - top) <= off.max() + 4 * O.U * top
    # x = most^2 * value / scale carries the value's error, the scale's and three roundings; a code is off by half plus what that is
    # under the root
    x = values / scale
    room = 0.5 + most * (np.sqrt(x + off / scale + x * (off.max() / top + 8 * O.U)) - np.sqrt(x)) + 1e-6
    near = most * np.sqrt(x)
    if least:
        near = np.where(values > 0, np.maximum(near, least), near)
    assert (np.abs(np.abs(codes) - near) <= room).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g,master", [("float32", "float32", False), ("bfloat16", "float32", True), ("bfloat16", "bfloat16", False),
                                        ("float16", "float16", True), ("float32", "bfloat16", False), ("float16", "float32", False)])
@pytest.mark.parametrize("k,offset", [(0, 0), (0, 3), (32, 0), (7, 0), (4, 1), (1000, 16), (1, 0), (4, 4), (0, 12), (3, 2), (2, 5)])
def test_adamw(p, g, master, k, offset, bits):
    job = Job([bits, k, offset], SIZES, p, g, master, k, bits, offset)
    for step in (3, 4):
        before = job.weights(), job.states()
        job.step(step)
        job.check(before, step)


@pytest.mark.parametrize("p,g,master,k", [("bfloat16", "bfloat16", True, 0), ("float32", "float32", False, 32), ("float16", "float32", True, 7), ("float32", "float16", False, 1000)])
def test_long_tensors_in_8_bits(p, g, master, k):
    """More blocks than one for each warp that the GPU holds: warps walk, and fetch a block while they work on another."""
    job = Job([8, k, 77], [2_500_001, 300, 150_016, 5], p, g, master, k, 8)
    for step in (1, 5):
        before = job.weights(), job.states()
        job.step(step)
        job.check(before, step)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_zero_states_and_a_scale(bits):
    import torch
    job = Job([bits, 5], SIZES, "bfloat16", "float32", True, 16, bits, fresh=True)
    before = job.weights(), job.states()
    scale = torch.tensor([0.37], device="cuda")
    job.step(1, scale)
    job.check(before, 1, float(scale))
    m, v = job.states()
    for i, a in enumerate(job.at[:-1]):
        assert (m[a + SIZES[i]:job.at[i + 1]] == 0).all() and (v[a + SIZES[i]:job.at[i + 1]] == 0).all()      # fill stays zero


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [float("nan"), float("inf")])
def test_scale_that_is_not_finite_changes_nothing(bits, scale):
    import torch
    job = Job([bits, 6], [300, 5000], "float32", "float32", False, 0, bits)
    copies = [t.clone() for t in (*job.param, job.m, job.v)]
    job.step(2, torch.tensor([scale], device="cuda"))
    for a, b in zip(copies, (*job.param, job.m, job.v)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("k", [32, 7, 600])
def test_messages_not_delivered_keep_their_elements(k):
    """Weights and 32-bit states keep their bits; gradients of messages that were not delivered may hold anything."""
    import torch
    for bits in (32, 8):
        job = Job([k, bits], [5000, 100], "bfloat16", "float32", True, k, bits)
        gone = [torch.from_numpy(s == 0).cuda() for s in job.shares()]
        for g, w in zip(job.grad, gone):
            g[w] = float("nan")
        old = [t.clone() for t in (*job.param, *job.master)]
        states = job.m.clone(), job.v.clone()
        job.step(2)
        for a, b, w in zip(old, (*job.param, *job.master), gone * 2):
            assert torch.equal(a[w], b[w]) and not torch.equal(a, b) and torch.isfinite(b.float()).all()
        if bits == 32:
            for a, b in zip(states, (job.m, job.v)):
                for i, w in enumerate(gone):
                    x, y = a[job.at[i]:job.at[i] + len(w)], b[job.at[i]:job.at[i] + len(w)]
                    assert torch.equal(x[w], y[w])


def test_extreme_gradients():
    """Zero gradients from zero states, gradients whose squares underflow, a block with NaN or infinity beside clean ones."""
    import torch
    for bits in (32, 8):
        job = Job([bits], [256 * 5], "float32", "float32", False, 0, bits, fresh=True)
        job.grad[0].zero_()
        job.grad[0][256:512] = 1e-25
        job.grad[0][512:768] = 1e19
        job.grad[0][800] = float("nan")
        job.grad[0][1030] = float("inf")
        w0 = job.param[0].clone()
        job.step(1)
        w = job.param[0]
        keep = 1 - LR * job.lr_scale[0] * job.decay[0]
        assert torch.allclose(w[:256], w0[:256] * keep, rtol=1e-6, atol=0)          # 0 / (0 + eps)
        m, v = job.states()
        assert np.isfinite(m[:768]).all() and np.isfinite(v[:768]).all() and (m[:256] == 0).all()
        # each moves by lr where g*g is no zero in float32: m1/(1-b1) = g, sqrt(v1/(1-b2)) = |g|
        assert torch.allclose(w[512:768], w0[512:768] * keep - LR * job.lr_scale[0], rtol=1e-5, atol=1e-7)
        assert torch.isnan(w[800]) and torch.isnan(w[1030]) and torch.isnan(w[768:]).sum() == 2
        if bits == 8:
            assert np.isnan(m[768:1280]).all()                                     # the block says so as a whole
        else:
            assert np.isnan(m[800]) and np.isfinite(m[801:1030]).all()


def test_many_steps_in_8_bits_follow_32_bits():
    """A quadratic's minimum is reached with either kind of state."""
    import torch
    target = torch.linspace(-1, 1, 1024, device="cuda")
    for bits in (32, 8):
        job = Job([9], [1024], "float32", "float32", False, 0, bits, fresh=True)
        job.decay[0] = 0.0
        for step in range(1, 801):
            job.grad[0].copy_(job.param[0] - target)
            job.step(step, lr=2e-2 if step < 500 else 2e-3)
        assert (job.param[0] - target).abs().max() < 0.02


@pytest.mark.parametrize("sizes", [[1], [256], [3, 0, 5], SIZES, [70001] * 3, [13] * 500, [1 << 20, 1, 300]])
@pytest.mark.parametrize("g,k,offset", [("float32", 0, 0), ("bfloat16", 0, 1), ("float16", 0, 0), ("float32", 32, 0), ("float32", 7, 3), ("float32", 4, 4),
                                        ("float32", 0, 20), ("float32", 3, 2), ("float32", 1, 1)])
def test_grad_norm(sizes, g, k, offset):
    import torch
    job = Job([len(sizes), k], sizes, "float32", g, False, k, 32, offset)
    want = np.array([np.sqrt(((d * s) ** 2).sum()) for d, s in zip(job.gradients(), job.shares())])
    total = np.sqrt((want ** 2).sum())
    ws = torch.full((B.ftc_grad_norm_workspace_bytes(job.table),), 0xFF, dtype=torch.uint8, device="cuda")
    for top in (0.5 * total + 1e-30, 2 * total + 1e-30, float("inf")):
        norm, norms = torch.full((2,), 9.0, device="cuda"), torch.full((len(sizes),), 9.0, device="cuda")
        B.ftc_grad_norm(job.table, top, norm, norms, ws)
        # squares are added in 64 bits: the gradient times its share (2 roundings), the result (1)
        assert np.allclose(norms.double().cpu().numpy(), want, rtol=4 * O.U, atol=1e-40)
        assert abs(float(norm[0]) - total) <= 4 * O.U * total + 1e-40
        assert abs(float(norm[1]) - min(1.0, top / total if total else 1.0)) <= 8 * O.U
    alone = torch.full((2,), 9.0, device="cuda")
    B.ftc_grad_norm(job.table, 1.0, alone, None, ws)
    B.ftc_grad_norm(job.table, 1.0, norm, norms, ws)
    assert torch.equal(alone, norm)


@pytest.mark.parametrize("g", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("k,offset", [(0, 0), (0, 3), (32, 0), (32, 8), (32, 3), (8, 4), (7, 0), (9, 5), (5, 2), (6, 0), (4, 1), (4, 4), (3, 0), (300, 1), (1000, 0)])
def test_grad_norm_of_long_tensors(g, k, offset):
    """Warps that walk many blocks: few numbers among zeros, few delivered messages among such of NaN, so that one element too many or
    too few shows. Whole numbers and shares of powers of two: the sums are exact, and the root and its rounding are all that is off."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(100 * k + offset)
    params, want = [], []
    for n in (9_000_001, 513, 7_000_007, 2_000_000):
        grad = torch.empty(n + offset, dtype=getattr(torch, g), device="cuda")[offset:]
        values = torch.randint(-8, 9, (n,), generator=gen, device="cuda").double()
        few = 200 if n > 1000 else 2
        if k:
            messages = -(-n // k)
            status = torch.zeros(messages, 4, dtype=torch.int32, device="cuda")
            status[:, 1] = 1 << torch.randint(0, 3, (messages,), generator=gen, device="cuda")
            lost = torch.randint(0, few * 8 // k + 2, (messages,), generator=gen, device="cuda") > 0
            status[:, 0] = lost.int() * 2
            status[:, 1] *= 1 - (lost & (torch.arange(messages, device="cuda") % 2 == 0)).int()      # half of the lost ones with a count, half without
            each = lost.repeat_interleave(k)[:n]
            grad.copy_(torch.where(each, float("nan"), values))
            share = torch.where(lost, 0.0, 1.0 / status[:, 1].clamp(min=1).double()).repeat_interleave(k)[:n]
            want.append(((values * share) ** 2).sum())
        else:
            status, values = None, values * (torch.randint(0, few, (n,), generator=gen, device="cuda") == 0)
            grad.copy_(values)
            want.append((values ** 2).sum())
        params.append(B.make_param(None, grad, status=status, k=k))
    table = B.make_param_table(params)
    ws = torch.empty(B.ftc_grad_norm_workspace_bytes(table), dtype=torch.uint8, device="cuda")
    norm, norms = torch.empty(2, device="cuda"), torch.empty(4, device="cuda")
    B.ftc_grad_norm(table, 1e9, norm, norms, ws)
    want = torch.stack(want)
    assert torch.allclose(norms.double(), want.sqrt(), rtol=2 * O.U, atol=0)
    assert abs(float(norm[0]) - float(want.sum().sqrt())) <= 2 * O.U * float(want.sum().sqrt())


def test_grad_norm_extremes():
    import torch
    job = Job([1], [3000, 5], "float32", "float32", False, 0, 32)
    ws = torch.empty(B.ftc_grad_norm_workspace_bytes(job.table), dtype=torch.uint8, device="cuda")
    norm, norms = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    for value, want in ((1e30, 1e30), (1e-30, 1e-30), (0.0, 0.0)):
        for g in job.grad:
            g.zero_()
        job.grad[0][77] = value
        B.ftc_grad_norm(job.table, 1.0, norm, norms, ws)
        assert abs(float(norm[0]) - want) <= 2 * O.U * want and float(norms[1]) == 0
        assert abs(float(norm[1]) - (1 / want if want > 1 else 1.0)) <= 4 * O.U * float(norm[1])
    for value in (float("nan"), float("inf"), float("-inf")):
        job.grad[0][2999] = value
        B.ftc_grad_norm(job.table, 1.0, norm, norms, ws)
        assert not torch.isfinite(norm[0]) and torch.isnan(norm[1]) and float(norms[1]) == 0


def test_empty_tables():
    import torch
    empty = B.make_param(torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))
    for params in ([], [empty], [empty] * 40):
        table = B.make_param_table(params)
        assert table.blocks == 0
        ws = torch.empty(max(16, B.ftc_grad_norm_workspace_bytes(table)), dtype=torch.uint8, device="cuda")
        norm = torch.full((2,), 9.0, device="cuda")
        B.ftc_grad_norm(table, 1.0, norm, None, ws)
        assert norm.tolist() == [0.0, 1.0]
        none = torch.empty(0, device="cuda")
        B.ftc_adamw_step(B.make_adamw(1e-3), table, none, none)


def test_states_read_out():
    import torch
    job = Job([4], [5000, 300, 1], bits=8)
    n = job.table.blocks * 256
    m, v = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    B.ftc_adamw_states(job.table, job.m, job.v, job.ms, job.vs, m, v)
    want = job.states()
    assert np.allclose(m.double().cpu().numpy(), want[0], rtol=4 * O.U, atol=0)
    assert np.allclose(v.double().cpu().numpy(), want[1], rtol=8 * O.U, atol=0)


def test_another_stream():
    import torch
    side = torch.cuda.Stream()
    job, twin = (Job([8], SIZES, "bfloat16", "float32", True, 16, 8) for _ in range(2))
    torch.cuda.synchronize()
    job.step(1, stream=side)
    side.synchronize()
    twin.step(1)
    torch.cuda.synchronize()
    assert torch.equal(job.m, twin.m) and all(torch.equal(a, b) for a, b in zip(job.master, twin.master))


def test_refusals_on_the_device():
    import torch
    g = torch.zeros(300, device="cuda")
    table = B.make_param_table([B.make_param(None, g)])
    m = torch.zeros(512, device="cuda")
    assert B.ftc_adamw_step(B.make_adamw(1e-3), table, m, m, check=False) == B.FTC_EINVAL       # a table without weights
    assert B.ftc_grad_norm(table, 1.0, torch.zeros(2, device="cuda"), None, None, check=False) == B.FTC_EWORKSPACE
    with pytest.raises(ValueError):
        B.ftc_adamw_step(B.make_adamw(1e-3), table, m[:256], m[:256])
    with pytest.raises(ValueError):
        B.ftc_adamw_step(B.make_adamw(1e-3), table, m.to(torch.int8), m.to(torch.uint8))        # no scales
    with pytest.raises(ValueError):
        B.make_param(torch.zeros(299, device="cuda"), g)
    with pytest.raises(ValueError):
        B.make_param(g, g, status=torch.zeros(3, 4, dtype=torch.int32, device="cuda"), k=32)


def test_a_tensor_of_more_than_32_bits_of_elements():
    """2^32 + 1000 elements: offsets, blocks and messages beyond 32 bits (27 GB on the device)."""
    import torch
    n = (1 << 32) + 1000
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("40 GB of device memory are wanted")
    grad, param = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    spots = torch.tensor([0, 255, (1 << 31) + 7, (1 << 32) - 1, 1 << 32, (1 << 32) + 300, n - 1], device="cuda")
    grad[spots] = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 7.0], dtype=torch.bfloat16, device="cuda")
    table = B.make_param_table([B.make_param(param, grad)])
    norm = torch.empty(2, device="cuda")
    ws = torch.empty(B.ftc_grad_norm_workspace_bytes(table), dtype=torch.uint8, device="cuda")
    B.ftc_grad_norm(table, 1e9, norm, None, ws)
    assert abs(float(norm[0]) - 140 ** 0.5) <= 4 * O.U * 140 ** 0.5
    m, v = torch.zeros(table.blocks * 256, dtype=torch.int8, device="cuda"), torch.zeros(table.blocks * 256, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(table.blocks, device="cuda"), torch.zeros(table.blocks, device="cuda")
    B.ftc_adamw_step(B.make_adamw(0.5, B1, B2, EPS, 1), table, m, v, ms, vs)
    assert torch.equal(param[spots].float(), torch.full((7,), -0.5, device="cuda"))      # the first step moves by lr against the sign
    assert int(torch.count_nonzero(param[:1 << 30])) == 2 and int(torch.count_nonzero(param[-(1 << 30):])) == 4
    assert int(m[n - 1]) == 127 and int(v[n - 1]) == 255
    # the same gradients in float32 as messages of 256, some with records of their own beyond element 2^32
    del m, v, ms, vs, param, grad, table
    k = 256
    status = torch.zeros(-(-n // k), 4, dtype=torch.int32, device="cuda")
    status[:, 1] = 2
    status[(n - 1) // k, 0] = 2                                                        # the last message was not delivered
    status[(1 << 32) // k, 1] = 4                                                      # that of element 2^32: four processes
    grad = torch.zeros(n, device="cuda")
    grad[spots] = torch.arange(1.0, 8.0, device="cuda")
    table = B.make_param_table([B.make_param(None, grad, status=status, k=k)])
    ws = torch.empty(B.ftc_grad_norm_workspace_bytes(table), dtype=torch.uint8, device="cuda")
    B.ftc_grad_norm(table, 1e9, norm, None, ws)
    shares = {(n - 1) // k: 0.0, (1 << 32) // k: 0.25}
    want = sum(((i + 1) * shares.get(s // k, 0.5)) ** 2 for i, s in enumerate(spots.tolist())) ** 0.5
    assert abs(float(norm[0]) - want) <= 8 * O.U * want
