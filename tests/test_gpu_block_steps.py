"""A block's training step call by call: every output against the formula in 64 bits on the very inputs that the call had, element by element, within what fp32 sums and the roundings to bf16 that
lie inside of a call may be off by.  (tests/test_gpu_block_training.py holds the whole step against the whole of it, where the roundings between the calls add up.)"""
import pytest
import torch

from epilogue_reference import F32, HALF, Weight, forward, slope
from update_reference import momentum_of, update

pytestmark = pytest.mark.gpu

MIX = {1: 0.3, 2: 0.5, 4: 0.2}
S = 2.0


def agree(got, want, off, what):
    excess = ((got.double() - want).abs() / (off + 1e-30)).max().item()
    assert excess <= 1.0, (what, excess)


def input_gradient(W_hat, g, A, B):
    """dY deq(Wq) + s (dY B^T) A^T, whose first product is rounded to bf16, and so is the result."""
    W, g, a, b = (t.double() for t in (W_hat, g, A, B))
    u = S * g @ b.t()
    want = g @ W + u @ a.t()
    n, r = W.shape[0], A.shape[1]
    off = (n + r + 4) * F32 * (g.abs() @ W.abs() + S * (g.abs() @ b.abs().t()) @ a.abs().t()) + HALF * (u.abs() @ a.abs().t())
    return want, off * (1 + HALF) + HALF * want.abs()


def factor_gradients(X, g, A, B):
    """dA = X^T (s dY B^T), dB = (s X A)^T dY; the products in brackets are rounded to bf16, and so are the results."""
    x, g, a, b = (t.double() for t in (X, g, A, B))
    out = []
    for left, first, second in ((x, g, b.t()), (g, x, a)):
        inner, size = S * first @ second, S * first.abs() @ second.abs()
        want = left.t() @ inner
        off = left.abs().t() @ ((first.shape[1] + 4) * F32 * size + HALF * inner.abs()) + (x.shape[0] + 4) * F32 * (left.abs().t() @ inner.abs())
        out.append((want, off * (1 + HALF) + HALF * want.abs()))
    return out[0], tuple(t.t() for t in out[1])


@pytest.mark.parametrize("D,F,M,r", [(256, 1024, 40, 16), (512, 1408, 333, 64), (1024, 4096, 777, 128)])
def test_every_call_of_a_step(D, F, M, r):
    import paper_2502_08141_b200 as lw

    w1, w2 = Weight(F, D, MIX, r, seed=11), Weight(D, F, MIX, r, seed=12)
    b1, b2 = w1.draw(F).bfloat16() * 0.1, w2.draw(D) * 0.1
    stream, dY = w1.draw(M, D).bfloat16(), w1.draw(M, D).bfloat16() * 1e-3
    X = stream.clone()
    A1, B1, A2, B2 = w1.A[0], w1.B[0], w2.A[0], w2.B[0]

    Z = torch.empty(M, F, dtype=torch.bfloat16, device="cuda")
    H = lw.lowra_lora_forward_epilogue(*w1.head(), X, A1, B1, S, bias=b1, activation="gelu", pre=Z)
    y, z, y_off, z_off = forward(w1.W_hat[0], X, A1, B1, S, bias=b1, activation="gelu")
    agree(H, y, y_off, "H")
    agree(Z, z, z_off, "Z")
    Y = lw.lowra_lora_forward_epilogue(*w2.head(), H, A2, B2, S, bias=b2, residual=stream, Y=stream)        # added to the stream in place
    y, _, y_off, _ = forward(w2.W_hat[0], H, A2, B2, S, bias=b2, residual=X)
    assert Y is stream
    agree(Y, y, y_off, "Y")

    dH = lw.lowra_lora_backward_input(*w2.head(), dY, A2, B2, S)
    agree(dH, *input_gradient(w2.W_hat[0], dY, A2, B2), "dH")
    dZ, _, db1 = lw.lowra_epilogue_backward(dH, Z, "gelu", want_bias=True)
    want = dH.double() * slope(Z.double(), "gelu")
    off = 8 * F32 * dH.double().abs() + 4 * F32 * want.abs()
    agree(dZ, want, off * (1 + HALF) + HALF * want.abs(), "dZ")
    agree(db1, want.sum(0), off.sum(0) + (M + 16) * F32 * want.abs().sum(0), "db1")
    _, _, db2 = lw.lowra_epilogue_backward(dY, want_bias=True)
    agree(db2, dY.double().sum(0), (M + 16) * F32 * dY.double().abs().sum(0), "db2")
    dX = lw.lowra_lora_backward_input(*w1.head(), dZ, A1, B1, S)
    agree(dX, *input_gradient(w1.W_hat[0], dZ, A1, B1), "dX")
    grads = [*lw.lowra_lora_backward_adapters(X, dZ, A1, B1, S), *lw.lowra_lora_backward_adapters(H, dY, A2, B2, S)]
    for name, got, ref in zip(("dA1", "dB1", "dA2", "dB2"), grads, (*factor_gradients(X, dZ, A1, B1), *factor_gradients(H, dY, A2, B2))):
        agree(got, *ref, name)

    members = [dict(grad=g, momentum=torch.zeros(g.shape, device="cuda"), master=f.float(), weight=f, update=torch.empty(g.shape, device="cuda")) for g, f in zip(grads, (A1, B1, A2, B2))]
    before = [m["master"].clone() for m in members]
    lw.lowra_update_factors(members, 0.02, rank=r)
    for m, old in zip(members, before):
        new, u = momentum_of(torch.zeros_like(old), m["grad"])
        assert torch.equal(m["momentum"], new)
        x, far = update(u, m["grad"].shape[1] == r)
        agree(m["update"], x, far, "update")
        want = old.double() - 0.02 * m["update"].double()
        agree(m["master"], want, F32 * (old.double().abs() + want.abs() + 0.02 * m["update"].double().abs()), "weights")
        assert torch.equal(m["weight"], m["master"].bfloat16())
