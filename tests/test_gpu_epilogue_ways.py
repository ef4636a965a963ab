"""What the products with an epilogue, its gradient and the update of the factors take does not depend on which of the binding's two ways a call goes: the native one, or the interpreted one
that calls with a stream take."""
import pytest
import torch

from epilogue_reference import Weight

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "interpreted"])
def way(request):
    return dict(stream=None if request.param == "native" else torch.cuda.current_stream())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_bias_is_a_vector(way, dtype):
    import paper_2502_08141_b200 as lw

    w = Weight(264, 384, {1: 0.5, 2: 0.5}, 16)
    X = w.draw(5, w.K).bfloat16()
    bias = w.draw(w.N).to(dtype)
    run = lambda b: lw.lowra_lora_forward_epilogue(*w.head(), X, w.A[0], w.B[0], 2.0, bias=b, **way)
    run(bias)
    for other in (bias.view(1, -1), bias.view(-1, 1), bias.view(2, -1), bias.new_zeros(w.N + 1), bias.new_zeros(0), bias[0]):
        with pytest.raises(ValueError, match="bias must be"):
            run(other)


def test_scratch_counts_in_bytes(way):
    import paper_2502_08141_b200 as lw

    M, N = 900, 264
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)
    dY, pre = draw(M, N).bfloat16(), draw(M, N).bfloat16()
    size = lw.lowra_epilogue_workspace_bytes(M, N)
    whole = lambda n, dtype: torch.empty(n // dtype.itemsize, dtype=dtype, device="cuda")
    run = lambda ws: lw.lowra_epilogue_backward(dY, pre, "silu", want_bias=True, workspace=ws, **way)
    want = run(None)
    for dtype in (torch.uint8, torch.float32, torch.float64):
        assert all(a is None or torch.equal(a, b) for a, b in zip(run(whole(size, dtype)), want))
        with pytest.raises(lw.LowraError) as e:
            run(whole(size - 8, dtype))
        assert e.value.code == lw.LOWRA_ERR_WORKSPACE
    shapes = [(2056, 48), (48, 1000)]
    grads = [draw(*s) for s in shapes]
    size = lw.lowra_update_workspace_bytes(shapes, 48)

    def update(ws):
        members = [dict(grad=g, update=torch.empty_like(g)) for g in grads]
        lw.lowra_update_factors(members, 0.02, workspace=ws, **way)
        return [m["update"] for m in members]

    want = update(None)
    for dtype in (torch.uint8, torch.float32, torch.float64):
        assert all(torch.equal(a, b) for a, b in zip(update(whole(size, dtype)), want))
        with pytest.raises(lw.LowraError) as e:
            update(whole(size - 8, dtype))
        assert e.value.code == lw.LOWRA_ERR_WORKSPACE
