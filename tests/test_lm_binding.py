"""The binding of the language model operators, without a GPU: what a call that leaves something out gets, and what is refused."""
import inspect

from paper_2602_22445_b200 import binding as B


def test_products_that_nobody_chose_are_the_exact_ones():
    assert B.make_muon(1e-3).products == 32
    assert inspect.signature(B.ftc_muon_workspace_bytes).parameters["products"].default == B.make_muon(1e-3).products
    assert B.make_muon(1e-3, products=16).products == 16
