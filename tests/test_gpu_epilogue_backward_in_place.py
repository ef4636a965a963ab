"""The gradient through what stands behind a product, in place: rows that end inside a sector of 32 bytes and begin in their neighbour's, every way through the kernels (flat, runs, narrow),
each output in every input's place, repeated, and captured in a graph."""
import pytest
import torch

from test_gpu_epilogue_backward import inputs

pytestmark = pytest.mark.gpu

SHAPES = [(3, 8), (37, 24), (128, 4104), (333, 4104), (1001, 520)]
PLACES = [("dY", "multiply"), ("pre", "dY"), ("multiply", "pre"), ("dY", None), (None, "pre")]         # of dZ and of dmultiply


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("bias", [False, True])
def test_every_place(M, N, bias):
    import paper_2502_08141_b200 as lw

    dY, pre, multiply = inputs(M, N, seed=M)
    want = lw.lowra_epilogue_backward(dY, pre, "gelu", multiply=multiply, want_bias=bias)
    for first, second in PLACES:
        for _ in range(3):
            a = dict(dY=dY.clone(), pre=pre.clone(), multiply=multiply.clone())
            got = lw.lowra_epilogue_backward(a["dY"], a["pre"], "gelu", multiply=a["multiply"], dZ=a.get(first), dmultiply=a.get(second), want_bias=bias)
            assert all(x is None and y is None or torch.equal(x, y) for x, y in zip(got, want)), (first, second)
            for name, t in (("dY", dY), ("pre", pre), ("multiply", multiply)):
                assert name in (first, second) or torch.equal(a[name], t), name


def test_captured():
    import paper_2502_08141_b200 as lw

    M, N = 333, 1032
    dY, pre, multiply = inputs(M, N, seed=9)
    want = lw.lowra_epilogue_backward(dY, pre, "silu", multiply=multiply, want_bias=True)
    place, other, dbias = dY.clone(), multiply.clone(), torch.empty(N, device="cuda")
    workspace = torch.empty(lw.lowra_epilogue_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lw.lowra_epilogue_backward(place, pre, "silu", multiply=other, dZ=place, dmultiply=other, dbias=dbias, workspace=workspace)
    for _ in range(3):
        place.copy_(dY)
        other.copy_(multiply)
        dbias.zero_()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip((place, other, dbias), want))


def test_side_by_side():
    """All arrays in one piece of memory, one directly behind the other, are in nobody's way."""
    import paper_2502_08141_b200 as lw

    M, N = 37, 264
    dY, pre, multiply = inputs(M, N, seed=2)
    want = lw.lowra_epilogue_backward(dY, pre, "silu", multiply=multiply, want_bias=True)
    block = torch.zeros(5 * M * N + 2 * N, dtype=torch.bfloat16, device="cuda")
    rows = [block[i * M * N:(i + 1) * M * N].view(M, N) for i in range(5)]
    dbias = block[5 * M * N:].view(torch.float32)
    for to, t in zip(rows[1::2] + rows[4:], (dY, pre, multiply)):
        to.copy_(t)
    got = lw.lowra_epilogue_backward(rows[1], rows[3], "silu", multiply=rows[4], dZ=rows[0], dmultiply=rows[2], dbias=dbias)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(rows[1], dY) and torch.equal(rows[3], pre) and torch.equal(rows[4], multiply)
