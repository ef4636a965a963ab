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
