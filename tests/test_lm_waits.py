"""The waits of the orthogonalised update's kernels, as far as their source shows them (nothing here runs on a GPU)."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_22445_b200", "csrc", "ftc_muon.cu")


def kernels():
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    parts = re.split(r"__global__", text)[1:]
    return {re.search(r"(\w+)\(MuonArgs a", part).group(1): part for part in parts}


def test_kernels_that_give_up_do_not_go_by_who_has():
    """A block that gives up sets the workspace's first word while others begin: threads that each read it could part before a barrier, which has no
    limit."""
    bodies = kernels()
    setting = {name for name, body in bodies.items() if re.search(r"\*a\.word = 1", body)}
    assert setting == {"muon_products_kernel", "muon_small_kernel"}
    for name in setting:
        assert len(re.findall(r"a\.word", bodies[name])) == 1, name


def test_what_can_be_refused_is_asked_before_the_momentum_moves():
    """The momentum moves in place in the first kernel, so an error after it would count the gradient twice where the call is made again."""
    text = open(SOURCE).read()
    host = text[text.index("muon_small_kernel<SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize"):]
    first = host.index("muon_momentum_kernel<<<")
    assert max(host.rindex(name) for name in ("cudaFuncSetAttribute", "cudaOccupancyMaxActiveClusters", "ready<SPLIT>(a")) < first
