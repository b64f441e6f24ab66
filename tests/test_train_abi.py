"""The training operators' host side, without a GPU: refusals before anything touches a device, the table of tensors, and the 64-bit
definitions that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_22445_b200 import binding as B
from tests import train_oracle as O

NONE = None
FAKE = 1 << 20                     # an aligned address that nothing reads: every call below is refused first


def norm(H=64, P=1, k=64, dtype=B.FTC_BF16, wdtype=B.FTC_F32, eps=1e-5):
    return B.ftc_norm_t(H, P, k, dtype, wdtype, eps)


def forward(d, rows=4, x=FAKE, xs=64, gamma=FAKE, y=FAKE, ys=64, mean=FAKE):
    return B.load().ftc_layernorm_forward(C.byref(d) if d else None, rows, x, xs, gamma, None, y, ys, mean, None, None)


def backward(d, rows=4, dy=FAKE, dys=64, x=FAKE, xs=64, mean=FAKE, rstd=FAKE, splits=None, dx=FAKE, dxs=64, dg=None, db=None, ws=None, wsb=0):
    return B.load().ftc_layernorm_backward(C.byref(d) if d else None, rows, dy, dys, x, xs, None, mean, rstd, splits, dx, dxs, dg, db, ws, wsb, None)


@pytest.mark.parametrize("bad", [dict(H=0), dict(H=(1 << 24) + 1), dict(P=0), dict(P=(1 << 20) + 1), dict(k=0), dict(eps=-1.0), dict(eps=float("nan"))])
def test_descriptor_refused(bad):
    assert forward(norm(**bad)) == B.FTC_EINVAL and backward(norm(**bad)) == B.FTC_EINVAL
    assert B.ftc_layernorm_workspace_bytes(norm(**bad), 5) == 0


@pytest.mark.parametrize("dtype,wdtype", [(B.FTC_I32, B.FTC_F32), (B.FTC_BF16, B.FTC_F16), (B.FTC_F32, B.FTC_BF16), (9, 9)])
def test_types_refused(dtype, wdtype):
    assert forward(norm(dtype=dtype, wdtype=wdtype)) == B.FTC_EUNSUPPORTED and backward(norm(dtype=dtype, wdtype=wdtype)) == B.FTC_EUNSUPPORTED


def test_arguments_refused():
    d = norm()
    assert forward(None) == B.FTC_EINVAL and backward(None) == B.FTC_EINVAL
    for bad in (dict(x=None), dict(y=None), dict(xs=63), dict(ys=63), dict(x=FAKE + 1), dict(y=FAKE + 1), dict(gamma=FAKE + 2), dict(mean=FAKE + 2), dict(xs=1 << 41)):
        assert forward(d, **bad) == B.FTC_EINVAL, bad
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dys=1), dict(xs=1), dict(dxs=1), dict(dy=FAKE + 1), dict(dg=FAKE + 2),
                dict(splits=FAKE + 4)):
        assert backward(d, **bad) == B.FTC_EINVAL, bad
    assert forward(d, rows=0, x=None, y=None) == B.FTC_OK                      # no rows: nothing to do
    assert backward(d, rows=0) == B.FTC_OK and backward(d, dx=None) == B.FTC_OK   # nothing asked for
    assert B.make_norm_desc(64, "bfloat16").wdtype == B.FTC_BF16
    with pytest.raises(ValueError):
        B.make_norm_desc(64, "int32")


def test_batch_calls_still_refuse_the_new_types():
    for dt in (B.FTC_BF16, B.FTC_F16):
        assert B.ftc_kernel_name(B.make_desc(8, 1, 4, dt, "sum")) == "invalid"


def entry(n=300, param=FAKE, master=None, grad=FAKE, status=None, k=0, pd=B.FTC_F32, gd=B.FTC_F32, lr=1.0, wd=0.0, reserved=0):
    return B.ftc_param_t(param, master, grad, status, n, k, pd, gd, lr, wd, reserved)


def build(*entries, short=0):
    lib = B.load()
    arr = (B.ftc_param_t * max(1, len(entries)))(*entries)
    size = lib.ftc_param_table_bytes(arr, len(entries))
    buf = np.zeros(max(1, size // 8), dtype=np.uint64)
    rc = lib.ftc_param_table_build(arr, len(entries), buf.ctypes.data, max(0, size - short))
    return size, rc, buf


def test_table_layout():
    size, rc, buf = build(entry(300), entry(0), entry(256), entry(1, grad=FAKE + 4), entry(2000, pd=B.FTC_F16, gd=B.FTC_BF16, grad=FAKE + 2))
    assert rc == B.FTC_OK and size % 8 == 0
    assert B.load().ftc_param_table_blocks(buf.ctypes.data) == 2 + 0 + 1 + 1 + 8
    assert B.load().ftc_grad_norm_workspace_bytes(buf.ctypes.data) > 0
    size, rc, buf = build()
    assert rc == B.FTC_OK and B.load().ftc_param_table_blocks(buf.ctypes.data) == 0


@pytest.mark.parametrize("bad", [dict(grad=None), dict(grad=FAKE + 2), dict(param=FAKE + 1), dict(master=FAKE + 2), dict(status=FAKE, k=0), dict(status=FAKE + 4, k=4),
                                 dict(status=FAKE, k=1 << 31), dict(pd=B.FTC_I32), dict(gd=B.FTC_U64), dict(n=1 << 41), dict(reserved=1), dict(lr=float("nan")),
                                 dict(wd=float("inf"))])
def test_table_entries_refused(bad):
    size, rc, _ = build(entry(), entry(**bad))
    assert size == 0 and rc == B.FTC_EINVAL


def test_calls_on_tables_refused():
    lib = B.load()
    _, rc, buf = build(entry())
    assert rc == B.FTC_OK and build(entry(), short=8)[1] == B.FTC_EINVAL
    h = buf.ctypes.data
    no_table = np.zeros(64, dtype=np.uint64)
    assert lib.ftc_param_table_blocks(no_table.ctypes.data) == 0 and lib.ftc_param_table_blocks(None) == 0
    assert lib.ftc_grad_norm_workspace_bytes(no_table.ctypes.data) == 0

    def norm_call(h=h, d=FAKE, top=1.0, out=FAKE):
        return lib.ftc_grad_norm(h, d, top, out, None, FAKE, 1 << 30, None)

    for bad in (dict(h=None), dict(h=no_table.ctypes.data), dict(d=None), dict(d=FAKE + 8), dict(top=0.0), dict(top=float("nan")), dict(out=None), dict(out=FAKE + 2)):
        assert norm_call(**bad) == B.FTC_EINVAL, bad

    def step(h=h, d=FAKE, m=FAKE, v=FAKE, ms=FAKE, vs=FAKE, scale=None, **hyper):
        a = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, state_bits=8, reserved=0) | hyper
        return lib.ftc_adamw_step(C.byref(B.ftc_adamw_t(**a)), h, d, m, v, ms, vs, scale, None)

    for bad in (dict(h=None), dict(d=None), dict(m=None), dict(v=None), dict(m=FAKE + 16), dict(ms=None), dict(vs=FAKE + 2), dict(scale=FAKE + 1), dict(lr=-1.0),
                dict(lr=float("inf")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=float("nan")), dict(step=0), dict(reserved=7)):
        assert step(**bad) == B.FTC_EINVAL, bad
    assert step(state_bits=16) == B.FTC_EUNSUPPORTED
    assert step(h=build(entry(param=None))[2].ctypes.data) == B.FTC_EINVAL      # a table without weights
    assert step(h=build(entry(n=0, param=None, grad=None))[2].ctypes.data) == B.FTC_OK     # nothing to do
    assert lib.ftc_adamw_states(0, None, None, None, None, None, None, None) == B.FTC_OK
    assert lib.ftc_adamw_states(1, FAKE, FAKE, FAKE, None, FAKE, FAKE, None) == B.FTC_EINVAL
    assert lib.ftc_adamw_states(1, FAKE, FAKE, FAKE, FAKE, FAKE + 4, FAKE, None) == B.FTC_EINVAL


@pytest.mark.parametrize("name", ["beta1", "beta2"])
@pytest.mark.parametrize("bits", [8, 32])
def test_betas_that_are_one_in_float32_refused(name, bits):
    """A state would grow without ever decaying."""
    _, rc, buf = build(entry())
    assert rc == B.FTC_OK
    for beta in (1 - 1e-8, 1 - 2.0 ** -26, np.nextafter(1, 0), 1.0, float("nan")):
        a = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, state_bits=bits, reserved=0) | {name: beta}
        assert B.load().ftc_adamw_step(C.byref(B.ftc_adamw_t(**a)), buf.ctypes.data, FAKE, FAKE, FAKE, FAKE, FAKE, None, None) == B.FTC_EINVAL, beta
    _, rc, buf = build(entry(n=0, param=None, grad=None))
    for beta in (1 - 2.0 ** -24, 0.99999, 0.0):
        a = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, state_bits=bits, reserved=0) | {name: beta}
        assert B.load().ftc_adamw_step(C.byref(B.ftc_adamw_t(**a)), buf.ctypes.data, FAKE, FAKE, FAKE, FAKE, FAKE, None, None) == B.FTC_OK, beta


def test_learning_rates_beyond_float32_refused():
    """An infinite rate times a weight decay of zero would make every weight NaN."""
    for n, lr, want in ((300, 1e39, B.FTC_EINVAL), (300, 3.5e38, B.FTC_EINVAL), (0, 3.4e38, B.FTC_OK)):
        buf = build(entry(n=n))[2]
        hyper = B.ftc_adamw_t(lr, 0.9, 0.99, 1e-8, 1, 32, 0)
        assert B.load().ftc_adamw_step(C.byref(hyper), buf.ctypes.data, FAKE, FAKE, FAKE, None, None, None, None) == want, lr


def test_definitions():
    """The 64-bit gradients against central differences, and the messages' layout."""
    rng = np.random.default_rng(0)
    rows, H, P, k = 5, 13, 3, 4
    x, dy = rng.standard_normal((rows, H)), rng.standard_normal((rows, H))
    gamma, beta = rng.standard_normal(H), rng.standard_normal(H)
    (_, mean, rstd), _ = O.norm_forward(x, gamma, beta, 1e-5)
    splits = [0, 2, 2, 5]
    (dx, dg, db), _ = O.norm_backward(dy, x, gamma, mean, rstd, P, k, splits)

    def loss(x, g, b, part=slice(None)):
        return (dy * O.norm_forward(x, g, b, 1e-5)[0][0])[part].sum()

    h = 1e-6
    for r, c in ((0, 0), (3, 12), (4, 5)):
        e = np.zeros((rows, H))
        e[r, c] = h
        assert abs((loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h) - dx[r, c]) < 1e-7
    for c in (0, 7, 12):
        e = np.zeros(H)
        e[c] = h
        for p, (lo, hi) in enumerate(zip(splits, splits[1:])):
            part = slice(lo, hi)
            assert abs((loss(x, gamma + e, beta, part) - loss(x, gamma - e, beta, part)) / (2 * h) - dg[c // k, p, c % k]) < 1e-7
            assert abs((loss(x, gamma, beta + e, part) - loss(x, gamma, beta - e, part)) / (2 * h) - db[c // k, p, c % k]) < 1e-7
    assert dg.shape == (4, 3, 4) and (dg[3, :, 1:] == 0).all() and (dg[:, 1] == 0).all()
