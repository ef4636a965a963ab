"""Which form the update of the factors takes, counted in the launches of a captured call: one for short factors of small rank, up to the length where that is the faster way for their number,
else three; and that either gives the update of the definition, on both sides of every bound."""
import pytest
import torch

from test_gpu_update_factors import check, make

pytestmark = pytest.mark.gpu


def launches(members, r):
    import paper_2502_08141_b200 as lw
    from cuda.bindings import runtime

    lw.lowra_update_factors(members, 0.02, rank=r)          # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        lw.lowra_update_factors(members, 0.02, rank=r)
    status, _, nodes = runtime.cudaGraphGetNodes(runtime.cudaGraph_t(graph.raw_cuda_graph()))
    assert int(status) == 0
    return nodes


@pytest.mark.parametrize("r,count,longest", [(16, 1, 5632), (16, 2, 7680), (16, 3, 7680), (16, 4, 8192), (16, 14, 8192), (32, 1, 2048), (32, 14, 2048)])
def test_one_launch_where_it_is_faster(r, count, longest):
    shapes = lambda L: [(L, r) if i % 2 else (r, L) for i in range(count)]
    for L, expected in ((longest, 1), (longest + 8, 3)):
        members = make(shapes(L), r)
        check(members, r)
        assert launches(members, r) == expected, L
    if count > 1:                                            # the longest of them decides
        members = make([(64, r)] * (count - 1) + [(r, longest + 8)], r)
        check(members, r)
        assert launches(members, r) == 3


@pytest.mark.parametrize("r,count", [(16, 15), (32, 15), (48, 1), (64, 2)])
def test_more_factors_or_a_larger_rank_take_three(r, count):
    members = make([(64, r)] * count, r)
    check(members, r)
    assert launches(members, r) == 3
