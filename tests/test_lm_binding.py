"""The binding of the language model operators, without a GPU: what a call that leaves something out gets, and what is refused."""
import inspect

import pytest

from paper_2602_22445_b200 import binding as B
from tests.test_lm_abi import Tensor


def test_products_that_nobody_chose_are_the_exact_ones():
    assert B.make_muon(1e-3).products == 32
    assert inspect.signature(B.ftc_muon_workspace_bytes).parameters["products"].default == B.make_muon(1e-3).products
    assert B.make_muon(1e-3, products=16).products == 16


@pytest.mark.parametrize("dtype,size", [("complex64", 8), ("qint32", 4), ("float32", 4), ("float64", 8), ("int16", 2), ("bool", 1)])
def test_tokens_that_are_no_whole_numbers_are_refused(monkeypatch, dtype, size):
    class Library:
        def __getattr__(self, name):
            raise AssertionError("not refused")

    monkeypatch.setattr(B, "_lib", Library())
    embed, prob = B.make_embed_desc(7, 4, "float32", P=2), B.make_logprob_desc(7, "float32", top=2)
    bad, good, rows, table, top = Tensor((3,), dtype, size), Tensor((3,), "int64", 8), Tensor((3, 7), "float32", 4), Tensor((7, 4), "float32", 4), Tensor((3, 2), "float32", 4)
    x = Tensor((3, 4), "float32", 4)
    for call in (lambda: B.ftc_embedding_forward(embed, bad, table, x, stream=1),
                 lambda: B.ftc_embedding_backward(embed, bad, x, None, Tensor((56,), "float32", 4), None, stream=1),
                 lambda: B.ftc_embedding_backward(embed, good, x, Tensor((3,), dtype, size), Tensor((56,), "float32", 4), None, stream=1),
                 lambda: B.ftc_token_logprobs(prob, rows, bad, None, d_top_logprob=top, d_top_token=Tensor((3, 2), "int32", 4), stream=1),
                 lambda: B.ftc_token_logprobs(prob, rows, good, None, d_top_logprob=top, d_top_token=Tensor((3, 2), dtype, size), stream=1)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("size", [16, 4096])
def test_a_wait_that_gave_up_is_told(size):
    import torch
    for dtype in (torch.uint8, torch.int16, torch.float32, torch.int64):
        ws = torch.zeros(size, dtype=dtype)
        B.check_muon(ws)
        ws.view(torch.uint8)[4] = 9           # behind the word
        B.check_muon(ws)
        ws.view(torch.uint8)[0] = 1
        with pytest.raises(B.FtcError):
            B.check_muon(ws)
