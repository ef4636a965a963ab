"""Arrays of more than 2^31 elements: what lies past that is read and written in its place."""
import numpy as np
import pytest
import torch

import paper_2502_08141_b200 as lw

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB of free device memory")
    yield
    torch.cuda.empty_cache()


def test_norm():
    M, N = 140001, 16384
    tail = 5
    X = torch.ones((M, N), dtype=torch.bfloat16, device="cuda")
    part = torch.randn((tail, N), device="cuda").bfloat16()
    X[-tail:] = part
    w, b = torch.rand(N, device="cuda") + 0.5, torch.rand(N, device="cuda")
    Y, rstd, mean, _ = lw.lowra_norm_forward(X, w, b)
    want = lw.lowra_norm_forward(part, w, b)
    assert torch.equal(Y[-tail:], want[0]) or (Y[-tail:].float() - want[0].float()).abs().max() <= 2.0 ** -7 * want[0].float().abs().max()
    assert torch.allclose(mean[-tail:], want[2], rtol=0, atol=1e-6) and torch.allclose(rstd[-tail:], want[1], rtol=1e-6)
    assert torch.equal(Y[0], Y[M // 2]) and torch.equal(Y[0], Y[-tail - 1])
    dX, _, _ = lw.lowra_norm_backward(Y, X, w, rstd, mean=mean, dX=Y)             # in place, to the last row
    small, _, _ = lw.lowra_norm_backward(want[0], part, w, want[1], mean=want[2])
    assert (dX[-tail:].float() - small.float()).abs().max() <= 2.0 ** -6 * small.float().abs().max()


def test_rotary():
    M, H, D = 70001, 8, 128
    wide = torch.empty((M, 260, D), dtype=torch.bfloat16, device="cuda")          # a token's row is 33 280 values
    q = wide[:, 250:258]
    q.copy_(torch.randn((1, H, D), device="cuda").bfloat16().expand(M, H, D))
    positions = torch.arange(M, device="cuda", dtype=torch.int32)
    turns = torch.from_numpy(lw.lowra_rotary_turns(D)[0].view(np.int64)).cuda()
    want = lw.lowra_rotary(q[-7:].contiguous(), positions[-7:].contiguous(), turns)
    lw.lowra_rotary(q, positions, turns, out=q)
    assert torch.equal(q[-7:], want)


@pytest.mark.parametrize("eight", [False, True])
def test_adamw(eight):
    n = (1 << 31) + 1000
    state = lambda: torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) if eight else torch.zeros(n, device="cuda")  # noqa: E731
    m = dict(grad=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), master=torch.ones(n, device="cuda"), m=state(), v=state())
    if eight:
        m["m_scale"], m["v_scale"] = (torch.zeros((n + 255) // 256, device="cuda") for _ in range(2))
    m["grad"][-1], m["grad"][5], m["grad"][1 << 31] = 1.0, -1.0, 2.0
    lw.lowra_adamw([m], 0.5, step=1, weight_decay=0.0)
    for i, want in ((-1, 0.5), (5, 1.5), (1 << 31, 0.5), (-2, 1.0), ((1 << 31) - 1, 1.0), (0, 1.0)):
        assert abs(m["master"][i].item() - want) <= 1e-6, i
    if eight:
        assert abs(m["m"][-1].float().item() * m["m_scale"][-1].item() - 0.1) <= 0.1 * 2.0 ** -4


def test_cross_entropy():
    M, V, K = 64, 600001, 4096
    g = torch.Generator(device="cuda").manual_seed(1)
    W = torch.zeros((V, K), dtype=torch.bfloat16, device="cuda")
    far = torch.randint(V - 3000, V, (200,), generator=g, device="cuda").unique()
    W[far] = (torch.randn((far.numel(), K), generator=g, device="cuda") * 3 / 64).bfloat16()
    X = torch.randn((M, K), generator=g, device="cuda").bfloat16()
    labels = far[torch.randint(0, far.numel(), (M,), generator=g, device="cuda")]
    loss, dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True)
    only, _ = lw.lowra_cross_entropy(X, W, labels)
    l = X.double() @ W[far].double().t()
    lse = torch.logaddexp(torch.logsumexp(l, 1), torch.full((M,), float(np.log(V - far.numel())), dtype=torch.float64, device="cuda"))
    own = torch.searchsorted(far, labels)
    want = lse - l.gather(1, own[:, None])[:, 0]
    p = torch.exp(l - lse[:, None])
    p.scatter_add_(1, own[:, None], torch.full((M, 1), -1.0, dtype=torch.float64, device="cuda"))
    dwant = p @ W[far].double()
    assert (loss.double() - want).abs().max() <= 1e-4 and (only.double() - want).abs().max() <= 1e-4
    assert torch.linalg.norm(dX.double() - dwant) <= 2.0 ** -8 * torch.linalg.norm(dwant)
