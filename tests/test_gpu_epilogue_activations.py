"""The activations behind a product are those of fp32 on every path: where a residual cancels them, so that no rounding to bf16 hides what they are off by, and at infinities.

The products are known exactly: every token picks out one input feature, and the low-rank factors are zero, so Z is a decoded weight plus the bias, rounded to fp32 once."""
import pytest
import torch

from epilogue_reference import HALF, Weight, activate

pytestmark = pytest.mark.gpu

U = torch.finfo(torch.float32).eps / 2                  # a rounding to fp32: 2^-24
PATHS = [(520, 384, 3), (520, 384, 300), (1800, 2304, 65), (1032, 4096, 600)]      # few tokens, whole tiles, shared tiles


def one_feature_each(N, K, M):
    w = Weight(N, K, {1: 0.3, 2: 0.5, 4: 0.2}, 16)
    picked = torch.arange(M, device="cuda") * 37 % K
    X = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    X[torch.arange(M, device="cuda"), picked] = 1.0
    zero = (torch.zeros_like(w.A[0]), torch.zeros_like(w.B[0]))
    return w, X, zero, w.W_hat[0].float()[:, picked].t().contiguous()


@pytest.mark.parametrize("N,K,M", PATHS)
@pytest.mark.parametrize("activation", ["relu", "gelu", "gelu_tanh", "silu"])
def test_a_residual_that_cancels_the_activation(N, K, M, activation):
    """How far the activation may be off, relative, in roundings: 2^x 4; 1/x 4 and what its argument is off by 4, which count up to threefold in the tail's polynomial; the polynomial
    16, its fit 2 and products 6: at most 52.  The exponent z^2 / 2, |z| or 2 t of the tanh form is off by four roundings of itself, and that is relative in 2^x."""
    import paper_2502_08141_b200 as lw

    w, X, (A, B), picked = one_feature_each(N, K, M)
    bias = w.draw(N).clamp(-2.5, 2.5) * 2
    z = (picked + bias).double()
    h = activate(z, activation)
    exponent = {"relu": 0.0 * z, "gelu": z * z / 2, "gelu_tanh": 2 * 0.8 * (z.abs() + 0.044715 * z.abs() ** 3), "silu": z.abs()}[activation]
    off = (52 + 4 * exponent) * U * h.abs()
    for factor in (None, w.draw(M, N).bfloat16()):
        behind = h if factor is None else h * factor.double()
        residual = (-behind).bfloat16()
        y = behind + residual.double()
        far = off * (1.0 if factor is None else factor.double().abs()) + 2 * U * (behind.abs() + y.abs())
        Y = lw.lowra_lora_forward_epilogue(*w.head(), X, A, B, 2.0, bias=bias, activation=activation, multiply=factor, residual=residual)
        excess = ((Y.double() - y).abs() / (far * (1 + HALF) + HALF * y.abs() + 1e-30)).max().item()
        assert excess <= 1.0, (factor is not None, excess)


@pytest.mark.parametrize("N,K,M", PATHS)
@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_infinities(N, K, M, activation):
    import paper_2502_08141_b200 as lw

    w, X, (A, B), _ = one_feature_each(N, K, M)
    bias, inf = torch.zeros(N, device="cuda"), float("inf")
    bias[::2] = torch.tensor([inf, -inf, 3e38, -3e38], device="cuda").repeat(N)[: bias[::2].numel()]
    Z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    Y = lw.lowra_lora_forward_epilogue(*w.head(), X, A, B, 2.0, bias=bias, activation=activation, pre=Z)
    assert bool((Z[:, 0::8] == inf).all()) and bool((Z[:, 2::8] == -inf).all())
    assert bool((Y[:, 0::8] == inf).all()) and bool((Y[:, 4::8] > 2.9e38).all()) and bool(Y[:, 1::2].isfinite().all())
    if activation == "none":
        assert bool((Y[:, 2::8] == -inf).all())
    else:
        assert bool((Y[:, 2::8] == 0).all() if activation == "relu" else Y[:, 2::8].isnan().all()) and bool((Y[:, 6::8] == 0).all())
