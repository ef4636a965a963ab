"""Arrays of more than 2^31 elements: the epilogue, its gradient and the update of the factors reach their last rows, and those are right."""
import pytest
import torch

from epilogue_reference import HALF, Weight, forward, slope

pytestmark = pytest.mark.gpu


def test_forward_and_its_gradient():
    import paper_2502_08141_b200 as lw

    N, K, M, r = 8192, 128, 270001, 16
    assert M * N > 2 ** 31
    w = Weight(N, K, {1: 0.5, 2: 0.5}, r)
    X = w.draw(M, K).bfloat16()
    Z, Y = (torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bias = w.draw(N)
    residual = torch.empty(M, N, dtype=torch.bfloat16, device="cuda").normal_()
    lw.lowra_lora_forward_epilogue(*w.head(), X, w.A[0], w.B[0], 2.0, bias=bias, activation="silu", residual=residual, pre=Z, Y=Y)
    rows = torch.tensor([0, 1, 131071, 131072, 262143, 262144, 262145, M - 257, M - 2, M - 1], device="cuda")
    y, z, y_off, z_off = forward(w.W_hat[0], X[rows], w.A[0], w.B[0], 2.0, bias=bias, activation="silu", residual=residual[rows])
    assert ((Y[rows].double() - y).abs() <= y_off).all() and ((Z[rows].double() - z).abs() <= z_off).all()
    for want_bias in (False, True):
        dZ, _, dbias = lw.lowra_epilogue_backward(residual, Z, "silu", dZ=Y, want_bias=want_bias)
        g = residual[rows].double()
        dz = g * slope(Z[rows].double(), "silu")
        assert ((dZ[rows].double() - dz).abs() <= 1.01 * HALF * dz.abs() + 1e-6 * g.abs() + 1e-30).all()
    total = torch.zeros(N, dtype=torch.float64, device="cuda")
    size = torch.zeros(N, dtype=torch.float64, device="cuda")
    for at in range(0, M, 30000):
        part = residual[at:at + 30000].double() * slope(Z[at:at + 30000].double(), "silu")
        total += part.sum(0)
        size += part.abs().sum(0)
    # a run's sums are chains of up to M / 13 / 8 additions (13 runs of 32 tiles, a warp every eighth row), and the slopes are good to 1e-6
    assert ((dbias.double() - total).abs() <= (M / 100 + 100) * 2.0 ** -24 * size + 1e-6 * size).all()


def test_update():
    import paper_2502_08141_b200 as lw

    r, L = 128, 1 << 24
    gen = torch.Generator(device="cuda").manual_seed(1)
    for shape in ((L, r), (r, L)):
        grad = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        update = torch.empty(shape, device="cuda")
        lw.lowra_update_factors([dict(grad=grad, update=update)], 0.02, rank=r)
        tall = grad if shape[0] == L else grad.t()
        out = update if shape[0] == L else update.t()
        s = torch.zeros(r, r, dtype=torch.float64, device="cuda")
        for at in range(0, L, 1 << 20):
            part = tall[at:at + (1 << 20)].double()
            s += part.t() @ part
        norm = s.trace().sqrt() + 1e-7
        g, q = s / norm ** 2, torch.eye(r, dtype=torch.float64, device="cuda")
        for _ in range(5):
            p = 3.4445 * torch.eye(r, dtype=torch.float64, device="cuda") - 4.775 * g + 2.0315 * g @ g
            g, q = g @ p @ p, q @ p
        rows = torch.cat([torch.arange(0, L, 65537, device="cuda"), torch.arange(L - 40, L, device="cuda")])
        want = tall[rows].double() @ q / norm
        off = (r + 4) * 2.0 ** -24 * (tall[rows].double().abs() @ q.abs() / norm) + 1e-12
        assert ((out[rows].double() - want).abs() <= off).all(), shape
        del grad, update, tall, out
