"""A block's training step as a program runs it: fc1 with bias and GELU, fc2 with bias onto the residual stream, the gradient through both, the factors' gradients and their update -
against the same step in 64 bits; a gated block's gradients; the step captured into a graph and replayed beside an eager one."""
import pytest
import torch

from epilogue_reference import Weight, activate, slope

pytestmark = pytest.mark.gpu

MIX = {1: 0.3, 2: 0.5, 4: 0.2}
S = 2.0


class Block:
    """fc1 [F, D] with bias and GELU, fc2 [D, F] with bias and residual, rank r."""

    def __init__(self, D, F, M, r, seed=1):
        import paper_2502_08141_b200 as lw

        self.D, self.F, self.M, self.r = D, F, M, r
        self.w1, self.w2 = Weight(F, D, MIX, r, seed=seed), Weight(D, F, MIX, r, seed=seed + 1)
        self.b1, self.b2 = self.w1.draw(F).bfloat16() * 0.1, self.w2.draw(D) * 0.1
        ws = lambda w: lw.lowra_workspace_init(torch.empty(lw.lowra_workspace_bytes(w.layout, M, r), dtype=torch.uint8, device="cuda"))
        self.ws = [ws(w) for w in (self.w1, self.w2, self.w1, self.w2)]
        shapes = [f.shape for f in self.factors()]
        self.momentum = [torch.zeros(s, device="cuda") for s in shapes]
        self.master = [f.float() for f in self.factors()]
        self.ws_update = torch.empty(lw.lowra_update_workspace_bytes(shapes, r), dtype=torch.uint8, device="cuda")
        self.ws_epilogue = torch.empty(lw.lowra_epilogue_workspace_bytes(M, F), dtype=torch.uint8, device="cuda")

    def factors(self):
        return [self.w1.A[0], self.w1.B[0], self.w2.A[0], self.w2.B[0]]

    def step(self, X, dY, update=True):
        import paper_2502_08141_b200 as lw

        w1, w2, ws = self.w1, self.w2, self.ws
        Z = torch.empty(self.M, self.F, dtype=torch.bfloat16, device="cuda")
        H = lw.lowra_lora_forward_epilogue(*w1.head(), X, w1.A[0], w1.B[0], S, bias=self.b1, activation="gelu", pre=Z, workspace=ws[0])
        Y = lw.lowra_lora_forward_epilogue(*w2.head(), H, w2.A[0], w2.B[0], S, bias=self.b2, residual=X, workspace=ws[1])
        dH = lw.lowra_lora_backward_input(*w2.head(), dY, w2.A[0], w2.B[0], S, workspace=ws[3])
        _, _, db2 = lw.lowra_epilogue_backward(dY, want_bias=True)
        dZ, _, db1 = lw.lowra_epilogue_backward(dH, Z, "gelu", want_bias=True, workspace=self.ws_epilogue)
        dX = lw.lowra_lora_backward_input(*w1.head(), dZ, w1.A[0], w1.B[0], S, workspace=ws[2])
        grads = [*lw.lowra_lora_backward_adapters(X, dZ, w1.A[0], w1.B[0], S), *lw.lowra_lora_backward_adapters(H, dY, w2.A[0], w2.B[0], S)]
        if update:
            members = [dict(grad=g, momentum=m, master=p, weight=f) for g, m, p, f in zip(grads, self.momentum, self.master, self.factors())]
            lw.lowra_update_factors(members, 0.02, rank=self.r, workspace=self.ws_update)
        return Y, dX, db1, db2, grads

    def exact(self, X, dY):
        W1, W2, x, g = self.w1.W_hat[0].double(), self.w2.W_hat[0].double(), X.double(), dY.double()
        leaves = [f.double().requires_grad_(True) for f in self.factors()]
        A1, B1, A2, B2 = leaves
        b1, b2 = self.b1.double().requires_grad_(True), self.b2.double().requires_grad_(True)
        x.requires_grad_(True)
        z = x @ W1.t() + S * (x @ A1) @ B1 + b1
        h = activate(z, "gelu")
        y = h @ W2.t() + S * (h @ A2) @ B2 + b2
        (y * g).sum().backward()                       # (the residual's share of dX is dY itself: the program adds it where it adds the streams)
        return (y + x).detach(), x.grad, b1.grad, b2.grad, [t.grad for t in leaves]


def close(got, want, what):
    """Two roundings to bf16 lie between the inputs and Y, three before dX and the factors' gradients, each half a step (2^-8) of values whose squares add up; the
    norm of the error is a few of them at most."""
    d = torch.linalg.norm(got.double() - want) / torch.linalg.norm(want)
    assert d.item() <= 4 * 2.0 ** -8, (what, d.item())


@pytest.mark.parametrize("D,F,M,r", [(256, 1032 - 8, 40, 16), (512, 1408, 333, 64), (1024, 4096, 777, 128)])
def test_step_against_64_bits(D, F, M, r):
    block = Block(D, F, M, r)
    X, dY = block.w1.draw(M, D).bfloat16(), block.w1.draw(M, D).bfloat16() * 1e-3
    want = block.exact(X, dY)
    before = [p.clone() for p in block.master]
    got = block.step(X, dY)
    for name, a, b in zip(("Y", "dX", "db1", "db2"), got, want):
        close(a, b, name)
    for name, a, b in zip(("dA1", "dB1", "dA2", "dB2"), got[4], want[4]):
        close(a, b, name)
    for p, old, f, g in zip(block.master, before, block.factors(), got[4]):
        assert torch.equal(f, p.bfloat16()) and not torch.equal(p, old)
        # against the gradient: the update is near orthogonal and points along it
        assert ((old - p).double() * g.double()).sum().item() > 0


@pytest.mark.parametrize("M", [5, 300])
def test_gated_block(M):
    """H = silu(gate(X)) * up(X): the gradients of both factors of the product, by the formula and by differences of the loss along random directions."""
    import paper_2502_08141_b200 as lw

    N, K, r = 1032, 384, 32
    gate, up = Weight(N, K, MIX, r, seed=3), Weight(N, K, MIX, r, seed=4)
    X, dH = gate.draw(M, K).bfloat16(), gate.draw(M, N).bfloat16() * 1e-2
    U = lw.lowra_lora_forward(*up.head(), X, up.A[0], up.B[0], S)
    Z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    H = lw.lowra_lora_forward_epilogue(*gate.head(), X, gate.A[0], gate.B[0], S, activation="silu", multiply=U, pre=Z)
    dZ, dU, _ = lw.lowra_epilogue_backward(dH, Z, "silu", multiply=U)
    z, u, g = Z.double(), U.double(), dH.double()
    close(H, activate(z, "silu") * u, "H")
    close(dZ, g * u * slope(z, "silu"), "dZ")
    close(dU, g * activate(z, "silu"), "dU")
    loss = lambda z, u: (g * activate(z, "silu") * u).sum().item()
    for seed in range(3):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        vz, vu = (torch.randn(M, N, device="cuda", generator=gen, dtype=torch.float64) for _ in range(2))
        h = 1e-4
        slope_along = (loss(z + h * vz, u + h * vu) - loss(z - h * vz, u - h * vu)) / (2 * h)
        got = ((dZ.double() * vz).sum() + (dU.double() * vu).sum()).item()
        size = (torch.linalg.norm(dZ.double()) + torch.linalg.norm(dU.double())).item()
        assert abs(got - slope_along) <= 6 * 2.0 ** -8 * size          # (a random direction: six standard deviations of the roundings)


def test_captured_step_beside_an_eager_one():
    D, F, M, r = 512, 1408, 100, 32
    a, b = Block(D, F, M, r), Block(D, F, M, r)
    X, dY = a.w1.draw(M, D).bfloat16(), a.w1.draw(M, D).bfloat16() * 1e-3
    Block(D, F, M, r, seed=7).step(X, dY)                # launch configurations, outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = a.step(X, dY)
    for _ in range(3):
        graph.replay()
        eager = b.step(X, dY)
        assert torch.equal(captured[0], eager[0]) and torch.equal(captured[1], eager[1])
        for x, y in zip(a.master + a.momentum + a.factors(), b.master + b.momentum + b.factors()):
            assert torch.equal(x, y)


def test_two_streams():
    """Two blocks' calls for few tokens, their gradients and updates, on two streams at once: the results of one after the other."""
    blocks = [Block(256, 1024, 9, 16, seed=s) for s in (1, 5)]
    data = [(b.w1.draw(9, 256).bfloat16(), b.w1.draw(9, 256).bfloat16() * 1e-3) for b in blocks]
    import paper_2502_08141_b200 as lw

    def small(b, X, dY):
        Z = torch.empty(9, 1024, dtype=torch.bfloat16, device="cuda")
        H = lw.lowra_lora_forward_epilogue(*b.w1.head(), X, b.w1.A[0], b.w1.B[0], S, bias=b.b1, activation="gelu", pre=Z, workspace=b.ws[0])
        out = [H, Z, *lw.lowra_epilogue_backward(H, Z, "gelu", want_bias=True)[::2]]
        members = [dict(grad=f * 0.5, momentum=m.clone(), master=p.clone(), update=torch.empty_like(p)) for f, m, p in zip(b.factors(), b.momentum, b.master)]
        lw.lowra_update_factors(members, 0.02, rank=16, workspace=b.ws_update)
        return out + [m["update"] for m in members]

    want = [small(b, *d) for b, d in zip(blocks, data)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        got = []
        for b, d, s in zip(blocks, data, streams):
            with torch.cuda.stream(s):
                got.append(small(b, *d))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w))
