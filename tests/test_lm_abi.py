"""The host side of the embedding, the token log probabilities and the orthogonalised update, without a GPU: refusals before anything
touches a device, the plan of matrices, and the 64-bit definitions that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import lm_oracle as O

FAKE = 1 << 20                     # an aligned address that nothing reads: every call below is refused first
BIG = 1 << 50


def embed(V=50, H=64, P=1, k=64, dtype=B.FTC_BF16, wdtype=B.FTC_F32, bits=64, scale=1.0):
    return B.ftc_embed_t(V, H, P, k, dtype, wdtype, bits, scale)


def embed_forward(d, n=4, tokens=FAKE, table=FAKE, ts=64, y=FAKE, ys=64):
    return B.load().ftc_embedding_forward(C.byref(d) if d else None, n, tokens, table, ts, y, ys, None)


def embed_backward(d, n=4, tokens=FAKE, dy=FAKE, ds=64, splits=None, out=FAKE, ws=FAKE, wsb=BIG):
    return B.load().ftc_embedding_backward(C.byref(d) if d else None, n, tokens, dy, ds, splits, out, ws, wsb, None)


@pytest.mark.parametrize("bad", [dict(V=0), dict(V=(1 << 30) + 1), dict(H=0), dict(H=(1 << 24) + 1), dict(P=0), dict(P=(1 << 20) + 1), dict(k=0), dict(k=(1 << 24) + 1),
                                 dict(V=1 << 30, H=1 << 11), dict(V=1 << 20, H=1 << 10, P=1 << 11), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_embedding_descriptors_refused(bad):
    d = embed(**bad)
    assert embed_forward(d, ts=1 << 24, ys=1 << 24) == B.FTC_EINVAL and embed_backward(d, ds=1 << 24) == B.FTC_EINVAL
    assert B.ftc_embedding_workspace_bytes(d, 5) == 0


@pytest.mark.parametrize("bad", [dict(dtype=B.FTC_I32), dict(wdtype=B.FTC_F16), dict(dtype=B.FTC_F32, wdtype=B.FTC_BF16), dict(bits=16), dict(bits=0)])
def test_embedding_types_refused(bad):
    assert embed_forward(embed(**bad)) == B.FTC_EUNSUPPORTED and embed_backward(embed(**bad)) == B.FTC_EUNSUPPORTED


def test_embedding_arguments_refused():
    d = embed()
    assert embed_forward(None) == B.FTC_EINVAL and embed_backward(None) == B.FTC_EINVAL
    for bad in (dict(tokens=None), dict(table=None), dict(y=None), dict(ts=63), dict(ys=63), dict(tokens=FAKE + 4), dict(table=FAKE + 2), dict(y=FAKE + 1), dict(ts=1 << 41),
                dict(n=(1 << 31) + 1)):
        assert embed_forward(d, **bad) == B.FTC_EINVAL, bad
    for bad in (dict(tokens=None), dict(dy=None), dict(ds=63), dict(out=None), dict(out=FAKE + 2), dict(dy=FAKE + 1), dict(splits=FAKE + 4), dict(tokens=FAKE + 4)):
        assert embed_backward(d, **bad) == B.FTC_EINVAL, bad
    need = B.ftc_embedding_workspace_bytes(d, 4)
    for bad in (dict(ws=None), dict(wsb=need - 1), dict(ws=FAKE + 8)):
        assert embed_backward(d, **bad) == B.FTC_EWORKSPACE, bad
    assert embed_backward(embed(V=1, H=1 << 24, k=1), n=1 << 31, ds=1 << 24) == B.FTC_ETOOLARGE
    assert embed_forward(d, n=0, tokens=None, table=None, y=None) == B.FTC_OK
    assert B.ftc_embedding_workspace_bytes(d, 0) == 0 and need > 0


def logp(V=50, dtype=B.FTC_BF16, bits=64, top=0, scale=1.0):
    return B.ftc_logprob_t(V, dtype, bits, top, scale)


def logp_forward(d, rows=4, x=FAKE, xs=64, tokens=FAKE, out=FAKE, entropy=FAKE, lse=FAKE, tv=None, ti=None):
    return B.load().ftc_token_logprobs(C.byref(d) if d else None, rows, x, xs, tokens, out, entropy, lse, tv, ti, None)


def logp_backward(d, rows=4, x=FAKE, xs=64, tokens=FAKE, lse=FAKE, entropy=FAKE, up=FAKE, de=FAKE, dx=2 * FAKE, ds=64):
    return B.load().ftc_token_logprobs_backward(C.byref(d) if d else None, rows, x, xs, tokens, lse, entropy, up, de, dx, ds, None)


@pytest.mark.parametrize("bad", [dict(V=0), dict(V=(1 << 30) + 1), dict(top=33), dict(V=5, top=6), dict(scale=0.0), dict(scale=-1.0), dict(scale=1e7), dict(scale=1e-7), dict(scale=float("nan"))])
def test_logprob_descriptors_refused(bad):
    assert logp_forward(logp(**bad), xs=1 << 31) == B.FTC_EINVAL and logp_backward(logp(**bad), xs=1 << 31, ds=1 << 31) == B.FTC_EINVAL


def test_logprob_arguments_refused():
    for bad in (dict(dtype=B.FTC_I64), dict(bits=8)):
        assert logp_forward(logp(**bad)) == B.FTC_EUNSUPPORTED and logp_backward(logp(**bad)) == B.FTC_EUNSUPPORTED
    d = logp()
    assert logp_forward(None) == B.FTC_EINVAL and logp_backward(None) == B.FTC_EINVAL
    for bad in (dict(x=None), dict(xs=49), dict(xs=1 << 41), dict(tokens=None), dict(x=FAKE + 1), dict(tokens=FAKE + 4), dict(out=FAKE + 2), dict(entropy=FAKE + 1), dict(lse=FAKE + 2),
                dict(tv=FAKE), dict(ti=FAKE), dict(tv=FAKE, ti=FAKE), dict(rows=1 << 31)):
        assert logp_forward(d, **bad) == B.FTC_EINVAL, bad
    for bad in (dict(), dict(tv=FAKE), dict(ti=FAKE), dict(tv=FAKE, ti=FAKE + 2)):
        assert logp_forward(logp(top=3), **bad) == B.FTC_EINVAL, bad
    for bad in (dict(x=None), dict(dx=None), dict(lse=None), dict(xs=49), dict(ds=49), dict(tokens=None), dict(entropy=None), dict(dx=FAKE + 1), dict(up=FAKE + 2), dict(de=FAKE + 2),
                dict(lse=FAKE + 1)):
        assert logp_backward(d, **bad) == B.FTC_EINVAL, bad
    assert logp_backward(d, dx=FAKE, ds=65) == B.FTC_EINVAL                                  # in place, rows elsewhere
    assert logp_forward(d, rows=0, x=None) == B.FTC_OK and logp_backward(d, rows=0, x=None) == B.FTC_OK
    assert logp_forward(d, tokens=None, out=None, entropy=None, lse=None) == B.FTC_OK        # nothing asked for


def entry(rows=6, cols=50, n=None, param=FAKE, master=None, grad=FAKE, status=None, k=0, pd=B.FTC_F32, gd=B.FTC_F32, lr=1.0, wd=0.0, reserved=0):
    return B.ftc_matrix_t(B.ftc_param_t(param, master, grad, status, rows * cols if n is None else n, k, pd, gd, lr, wd, reserved), rows, cols)


def build(*entries, short=0):
    lib = B.load()
    arr = (B.ftc_matrix_t * max(1, len(entries)))(*entries)
    size = lib.ftc_muon_plan_bytes(arr, len(entries))
    buf = np.zeros(max(1, size // 8), dtype=np.uint64)
    return size, lib.ftc_muon_plan_build(arr, len(entries), buf.ctypes.data, max(0, size - short)), buf


def test_plan_layout():
    lib = B.load()
    size, rc, buf = build(entry(6, 50), entry(300, 1), entry(1, 256, gd=B.FTC_BF16, grad=FAKE + 2), entry(700, 1000, pd=B.FTC_F16, param=FAKE + 2))
    assert rc == B.FTC_OK and size % 8 == 0
    assert lib.ftc_muon_plan_blocks(buf.ctypes.data) == 2 + 2 + 1 + 2735
    low, high = (lib.ftc_muon_workspace_bytes(buf.ctypes.data, p) for p in (16, 32))
    assert 0 < low < high <= 2 * low and lib.ftc_muon_workspace_bytes(buf.ctypes.data, 8) == 0
    # blocks of 128 x 64 float16 of X, twice, of A and B
    x, a = 1 + 5 + 4 + 6 * 16, 2 + 2 + 2 + 6 * 12
    assert 2 * (x + a) * 16384 <= low <= 2 * (x + a) * 16384 + (1 << 17)
    size, rc, buf = build()
    assert rc == B.FTC_OK and lib.ftc_muon_plan_blocks(buf.ctypes.data) == 0


@pytest.mark.parametrize("bad", [dict(grad=None), dict(param=None), dict(grad=FAKE + 2), dict(param=FAKE + 1), dict(master=FAKE + 2), dict(status=FAKE, k=0), dict(status=FAKE + 4, k=4),
                                 dict(pd=B.FTC_I32), dict(gd=B.FTC_U64), dict(reserved=1), dict(lr=float("nan")), dict(wd=float("inf")), dict(n=299), dict(rows=0), dict(cols=0),
                                 dict(rows=16385, cols=16385), dict(rows=1, cols=(1 << 20) + 1), dict(rows=1 << 12, cols=1 << 20)])
def test_plan_entries_refused(bad):
    size, rc, _ = build(entry(), entry(**bad))
    assert size == 0 and rc == B.FTC_EINVAL


def test_muon_calls_refused():
    lib = B.load()
    _, rc, buf = build(entry())
    assert rc == B.FTC_OK and build(entry(), short=8)[1] == B.FTC_EINVAL
    no_plan = np.zeros(64, dtype=np.uint64)
    assert lib.ftc_muon_plan_blocks(None) == 0 and lib.ftc_muon_plan_blocks(no_plan.ctypes.data) == 0 and lib.ftc_muon_workspace_bytes(no_plan.ctypes.data, 16) == 0
    need = lib.ftc_muon_workspace_bytes(buf.ctypes.data, 16)

    def step(h=buf.ctypes.data, d=FAKE, m=FAKE, scale=None, ws=FAKE, wsb=BIG, **hyper):
        a = dict(lr=1e-3, momentum=0.9, eps=1e-7, steps=5, nesterov=1, products=16, reserved=0) | hyper
        return lib.ftc_muon_step(C.byref(B.ftc_muon_t(**a)), h, d, m, scale, ws, wsb, None)

    for bad in (dict(h=None), dict(h=no_plan.ctypes.data), dict(d=None), dict(d=FAKE + 8), dict(m=None), dict(m=FAKE + 16), dict(scale=FAKE + 2), dict(lr=-1.0), dict(lr=float("nan")),
                dict(lr=1e39), dict(momentum=1.0), dict(momentum=1 - 1e-9), dict(momentum=-0.1), dict(eps=0.0), dict(eps=float("inf")), dict(steps=0), dict(steps=17), dict(nesterov=2),
                dict(reserved=1)):
        assert step(**bad) == B.FTC_EINVAL, bad
    assert step(products=8) == B.FTC_EUNSUPPORTED
    for bad in (dict(ws=None), dict(ws=FAKE + 128), dict(wsb=need - 1), dict(products=32, wsb=need)):
        assert step(**bad) == B.FTC_EWORKSPACE, bad
    assert step(h=build()[2].ctypes.data, m=None, ws=None) == B.FTC_OK                       # nothing to do


def test_gradient_against_differences():
    """The 64-bit forms against each other: the gradient is that of logprob and entropy."""
    rng = np.random.default_rng(1)
    x, t = rng.standard_normal((3, 9)) * 2, np.array([4, -1, 8])
    x[1, 3] = -np.inf
    up, de = rng.standard_normal(3), rng.standard_normal(3)
    lse, given, entropy, *_ = O.logprobs(x, t, 0.7)
    g, _ = O.logprobs_backward(x, t, 0.7, lse, entropy, up, de)
    for r in range(3):
        for j in range(9):
            if not np.isfinite(x[r, j]):
                assert g[r, j] == 0
                continue
            parts = []
            for h in (1e-5, -1e-5):
                y = x.copy()
                y[r, j] += h
                _, given, entropy, *_ = O.logprobs(y, t, 0.7)
                parts.append((up * given + de * entropy).sum())
            assert abs((parts[0] - parts[1]) / 2e-5 - g[r, j]) < 1e-8


def test_embedding_definition():
    """The gradient against differences of the lookup, for each process, and the messages' layout."""
    rng = np.random.default_rng(2)
    n, V, H, P, k, scale = 23, 5, 3, 4, 4, 1.5
    tokens, dy, table = rng.integers(-1, V + 1, n), rng.standard_normal((n, H)), rng.standard_normal((V, H))
    splits = [2, 9, 9, 20, 22]
    out, off = O.embedding_backward(tokens, dy, V, scale, P, k, splits)
    flat = out.transpose(1, 0, 2).reshape(P, -1)
    assert out.shape == (4, 4, 4) and (flat[:, V * H:] == 0).all() and (off >= 0).all()
    for v in range(V):
        for h in range(H):
            e = np.zeros((V, H))
            e[v, h] = 0.5
            moved = dy * (O.embedding_forward(tokens, table + e, scale) - O.embedding_forward(tokens, table, scale)) / 0.5
            for p in range(P):
                assert abs(moved[splits[p]:splits[p + 1]].sum() - flat[p, v * H + h]) < 1e-12


def test_muon_definition():
    """The steps are the quintic on the singular values; their bound is one for a rounded computation of the same."""
    rng = np.random.default_rng(4)
    for rows, cols in ((6, 9), (9, 6), (8, 8)):
        g, m, p = (rng.standard_normal((rows, cols)) for _ in range(3))
        there = np.ones((rows, cols), bool)
        new, m1, x, off = O.muon(p, m, g, there, 0.1, 2.0, 0.3, 0.9, True, 1e-7, 5, 16)
        u = g + 0.9 * m1
        a, s, b = np.linalg.svd(u / (np.linalg.norm(u) + 1e-7), full_matrices=False)
        for _ in range(5):
            s = 3.4445 * s - 4.775 * s ** 3 + 2.0315 * s ** 5
        assert np.allclose(x, (a * s) @ b, atol=1e-12) and np.allclose(new, p * (1 - 0.06) - 0.2 * x)
        # float16 operands, sums in 64 bits
        def half(v):
            return (v * 16384).astype(np.float16).astype(np.float64) / 16384
        y = u / (np.linalg.norm(u) + 1e-7)
        y = half(y.T if rows > cols else y)
        eye = np.eye(len(y))
        for _ in range(5):
            q = y @ y.T
            q = half(q * (1 - eye)) + q * eye
            r = half(3.4445 * eye - 4.775 * q + 2.0315 * q @ q)
            y = half(r @ y)
        y = y.T if rows > cols else y
        assert 0 < np.linalg.norm(y - x) <= off


class Tensor:
    """As much of a CUDA tensor as the binding looks at."""
    is_cuda = True

    def __init__(self, shape, dtype, size):
        self.shape, self.dtype, self.size = tuple(shape), dtype, size

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self.size

    def is_contiguous(self):
        return True

    def is_floating_point(self):
        return "float" in self.dtype

    def stride(self):
        return self.shape[1], 1

    def data_ptr(self):
        return FAKE


def test_tokens_of_either_width_leave_the_descriptor(monkeypatch):
    class Library:
        seen = []

        def ftc_embedding_forward(self, desc, *rest):
            self.seen.append(desc.token_bits)
            return B.FTC_OK

        def ftc_token_logprobs(self, desc, *rest):
            self.seen.append(desc.token_bits)
            return B.FTC_OK

    monkeypatch.setattr(B, "_lib", Library())
    e, p = B.make_embed_desc(7, 4, "float32"), B.make_logprob_desc(7, "float32")
    before = bytes(e), bytes(p)
    for size in (8, 4, 8):
        t = Tensor((3,), "int%d" % (8 * size), size)
        B.ftc_embedding_forward(e, t, Tensor((7, 4), "float32", 4), Tensor((3, 4), "float32", 4), stream=1)
        B.ftc_token_logprobs(p, Tensor((3, 7), "float32", 4), t, Tensor((3,), "float32", 4), stream=1)
        assert (bytes(e), bytes(p)) == before
    assert Library.seen == [64, 64, 32, 32, 64, 64]
    for bad in (Tensor((3,), "int16", 2), Tensor((3,), "float32", 4)):
        with pytest.raises(ValueError):
            B.ftc_embedding_forward(e, bad, Tensor((7, 4), "float32", 4), Tensor((3, 4), "float32", 4), stream=1)
    with pytest.raises(ValueError):
        B.ftc_embedding_forward(e, t, Tensor((7, 4), "bfloat16", 2), Tensor((3, 4), "float32", 4), stream=1)
    with pytest.raises(ValueError):
        B.ftc_token_logprobs(p, Tensor((3, 7), "float32", 4), Tensor((4,), "int64", 8), Tensor((3,), "float32", 4), stream=1)
    with pytest.raises(ValueError):
        B.ftc_token_logprobs(B.make_logprob_desc(7, "float32", top=2), Tensor((3, 7), "float32", 4), None, None, d_top_logprob=Tensor((3, 2), "float32", 4),
                             d_top_token=Tensor((3, 2), "int64", 8), stream=1)
