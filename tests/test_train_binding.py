"""The binding's part of the training calls, without a GPU: a library that only notes what it is given."""
import ctypes as C
import threading

import pytest

from paper_2602_22445_b200 import binding as B


class Tensor:
    """As much of a CUDA tensor as the binding looks at."""

    is_cuda = True

    def __init__(self, n, dtype, size):
        self.n, self.dtype, self.size = n, dtype, size

    def numel(self):
        return self.n

    def element_size(self):
        return self.size

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Table:
    blocks, h_ptr, d_ptr, n_params = 2, 4096, 4096, 1


class Library:
    def __init__(self, during=None):
        self.seen, self.during = [], during

    def ftc_adamw_step(self, hyper, *rest):
        if self.during:
            self.during()
        hyper = hyper._obj if hasattr(hyper, "_obj") else hyper
        self.seen.append((hyper.state_bits, hyper.step, hyper.lr))
        return B.FTC_OK


def states(bits):
    n = Table.blocks * B.FTC_STATE_BLOCK
    if bits == 32:
        return [Tensor(n, "float32", 4), Tensor(n, "float32", 4)]
    return [Tensor(n, "int8", 1), Tensor(n, "uint8", 1), Tensor(2, "float32", 4), Tensor(2, "float32", 4)]


def test_the_caller_keeps_its_hyper(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "_lib", lib)
    hyper = B.make_adamw(1e-3, step=7)
    before = bytes(hyper)
    for bits in (8, 32, 8):
        B.ftc_adamw_step(hyper, Table, *states(bits), stream=1)
        assert bytes(hyper) == before
    assert lib.seen == [(8, 7, 1e-3), (32, 7, 1e-3), (8, 7, 1e-3)]


def test_one_hyper_for_tables_of_different_states(monkeypatch):
    """A call that another thread's call meets halfway: each gets the bits of its own states."""
    hyper = B.make_adamw(1e-3)

    def other_thread():
        lib.during = None
        t = threading.Thread(target=lambda: B.ftc_adamw_step(hyper, Table, *states(32), stream=1))
        t.start()
        t.join()

    lib = Library(other_thread)
    monkeypatch.setattr(B, "_lib", lib)
    B.ftc_adamw_step(hyper, Table, *states(8), stream=1)
    assert [bits for bits, _, _ in lib.seen] == [32, 8]


def test_states_refused(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "_lib", lib)
    n = Table.blocks * B.FTC_STATE_BLOCK
    for bad in ([Tensor(n, "bfloat16", 2)] * 2, [Tensor(n, "int32", 4)] * 2, [Tensor(n - 1, "float32", 4)] * 2, states(8)[:2], [states(8)[0], states(32)[1]]):
        with pytest.raises(ValueError):
            B.ftc_adamw_step(B.make_adamw(1e-3), Table, *bad, stream=1)
    assert not lib.seen and C.sizeof(B.ftc_adamw_t) == 48
