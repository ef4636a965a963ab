"""A training step from the hidden states to the new factors, as a program runs it: residual addition and norm, the query and key products, their positions, a product back to the residual
stream, the last norm, the loss over the vocabulary with its gradient, and all the way back to an update of the factors - against the same step in 64 bits; captured and replayed beside an eager one."""
import pytest
import torch

import paper_2502_08141_b200 as lw
from epilogue_reference import Weight

pytestmark = pytest.mark.gpu

MIX = {1: 0.3, 2: 0.5, 4: 0.2}
S, EPS = 2.0, 1e-5


class Net:
    """h = X + R; n = norm(h); q, k = n Wq, n Wk with positions; o = (q k) Wo + h (token by token: what mixes the tokens is not what is tested); loss of norm(o) W^T."""

    def __init__(self, D, H, M, V, r, kind, bits, seed=1):
        self.D, self.H, self.M, self.kind = D, H, M, kind
        self.q, self.k, self.o = (Weight(D, D, MIX, r, seed=seed + i) for i in range(3))
        draw = self.q.draw
        self.norms = [(1 + 0.1 * draw(D), 0.1 * draw(D) if kind == "layer" else None) for _ in range(2)]
        self.head = (draw(V, D) * 2.0 / D ** 0.5).bfloat16()
        self.labels = torch.randint(0, V, (M,), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
        self.labels[::7] = -100
        self.positions = torch.arange(M, device="cuda", dtype=torch.int32) + 300
        self.turns = torch.from_numpy(lw.lowra_rotary_turns(D // H)[0].view("int64")).cuda()
        self.scale = 1.0 / int((self.labels != -100).sum())
        ws = lambda: lw.lowra_workspace_init(torch.empty(lw.lowra_workspace_bytes(self.q.layout, M, r), dtype=torch.uint8, device="cuda"))  # noqa: E731
        self.ws = [ws() for _ in range(6)]
        self.step_number = torch.ones(1, dtype=torch.int32, device="cuda")
        self.members = []
        for f in self.factors():
            m = dict(master=f.float(), weight=f)
            zeros = torch.zeros(f.shape, device="cuda")
            m["m"], m["v"] = (zeros.clone().to(torch.float8_e4m3fn), zeros.clone().to(torch.float8_e4m3fn)) if bits == 8 else (zeros.clone(), zeros.clone())
            if bits == 8:
                n = (f.numel() + lw.LOWRA_ADAMW_BLOCK - 1) // lw.LOWRA_ADAMW_BLOCK
                m["m_scale"], m["v_scale"] = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
            self.members.append(m)

    def factors(self):
        return [f for w in (self.q, self.k, self.o) for f in (w.A[0], w.B[0])]

    def heads(self, t):
        return t.view(self.M, self.H, self.D // self.H)

    def step(self, X, R, update=True):
        (g1, b1), (g2, b2), ws = self.norms[0], self.norms[1], self.ws
        n1, rstd1, mean1, h = lw.lowra_norm_forward(X, g1, b1, eps=EPS, kind=self.kind, residual=R)
        q = lw.lowra_lora_forward(*self.q.head(), n1, self.q.A[0], self.q.B[0], S, workspace=ws[0])
        k = lw.lowra_lora_forward(*self.k.head(), n1, self.k.A[0], self.k.B[0], S, workspace=ws[1])
        lw.lowra_rotary(self.heads(q), self.positions, self.turns, k=self.heads(k), out=self.heads(q), k_out=self.heads(k))
        mixed = q * k
        o = lw.lowra_lora_forward_epilogue(*self.o.head(), mixed, self.o.A[0], self.o.B[0], S, residual=h, workspace=ws[2])
        n2, rstd2, mean2, _ = lw.lowra_norm_forward(o, g2, b2, eps=EPS, kind=self.kind)
        loss, dn2 = lw.lowra_cross_entropy(n2, self.head, self.labels, scale=self.scale, want_grad=True)
        do, dg2, _ = lw.lowra_norm_backward(dn2, o, g2, rstd2, mean=mean2, want_params=True)
        dmixed = lw.lowra_lora_backward_input(*self.o.head(), do, self.o.A[0], self.o.B[0], S, workspace=ws[3])
        grads_o = lw.lowra_lora_backward_adapters(mixed, do, self.o.A[0], self.o.B[0], S)
        dq, dk = dmixed * k, dmixed * q
        lw.lowra_rotary(self.heads(dq), self.positions, self.turns, k=self.heads(dk), inverse=True, out=self.heads(dq), k_out=self.heads(dk))
        dn1 = lw.lowra_lora_backward_input(*self.q.head(), dq, self.q.A[0], self.q.B[0], S, workspace=ws[4])
        dn1 = dn1 + lw.lowra_lora_backward_input(*self.k.head(), dk, self.k.A[0], self.k.B[0], S, workspace=ws[5])
        dX, dg1, _ = lw.lowra_norm_backward(dn1, h, g1, rstd1, mean=mean1, dsum=do, want_params=True)
        grads = [*lw.lowra_lora_backward_adapters(n1, dq, self.q.A[0], self.q.B[0], S), *lw.lowra_lora_backward_adapters(n1, dk, self.k.A[0], self.k.B[0], S), *grads_o]
        if update:
            for m, g in zip(self.members, grads):
                m["grad"] = g
            lw.lowra_adamw(self.members, 1e-3, step=self.step_number)
            self.step_number += 1
        return loss, dX, dg1, dg2, grads

    def exact(self, X, R):
        leaves = [f.double().requires_grad_(True) for f in self.factors()]
        Aq, Bq, Ak, Bk, Ao, Bo = leaves
        params = [(g.double().requires_grad_(True), None if b is None else b.double()) for g, b in self.norms]
        x = X.double().requires_grad_(True)

        def norm(h, g, b):
            d = h - h.mean(1, keepdim=True) if self.kind == "layer" else h
            y = d / torch.sqrt((d * d).mean(1, keepdim=True) + EPS) * g
            return y if b is None else y + b

        def turn(t):
            t, half = self.heads(t), self.D // self.H // 2
            angle = self.positions.double()[:, None, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
            a, b, c, s = t[..., :half], t[..., half:], torch.cos(angle), torch.sin(angle)
            return torch.cat([a * c - b * s, b * c + a * s], -1).reshape(self.M, self.D)

        layer = lambda w, t, A, B: t @ w.W_hat[0].double().t() + S * (t @ A) @ B  # noqa: E731
        h = x + R.double()
        n1 = norm(h, *params[0])
        o = layer(self.o, turn(layer(self.q, n1, Aq, Bq)) * turn(layer(self.k, n1, Ak, Bk)), Ao, Bo) + h
        logp = torch.log_softmax(norm(o, *params[1]) @ self.head.double().t(), 1)
        counts = self.labels != -100
        loss = torch.where(counts, -logp.gather(1, self.labels.clamp_min(0)[:, None])[:, 0], 0.0)
        (loss.sum() * self.scale).backward()
        return loss.detach(), x.grad, params[0][0].grad, params[1][0].grad, [t.grad for t in leaves]


def close(got, want, roundings, what):
    """`roundings` values rounded to bf16 lie between the inputs and this one on any way, each off by half a step (2^-8) at most, in the mean by less than a third of it; their squares add up, a
    product carries on those of both its factors, and a norm or a softmax those of its input, hardly enlarged at these sizes."""
    d = (torch.linalg.norm(got.double() - want) / torch.linalg.norm(want)).item()
    assert d <= 2.0 ** -8 * roundings ** 0.5, (what, d)


@pytest.mark.parametrize("kind, bits", [("rms", 32), ("layer", 8)])
@pytest.mark.parametrize("D, H, M, V, r", [(256, 2, 40, 1000, 16), (512, 8, 333, 5003, 32), (1024, 8, 600, 32000, 64)])
def test_step_against_64_bits(D, H, M, V, r, kind, bits):
    net = Net(D, H, M, V, r, kind, bits)
    X, R = net.q.draw(M, D).bfloat16(), net.q.draw(M, D).bfloat16()
    want = net.exact(X, R)
    old = [m["master"].clone() for m in net.members]
    loss, dX, dg1, dg2, grads = net.step(X, R)
    close(loss, want[0], 9, "loss")
    close(dX, want[1], 24, "dX")
    close(dg1, want[2], 24, "dweight of the first norm")
    close(dg2, want[3], 16, "dweight of the last norm")
    for name, g, w in zip(("dAq", "dBq", "dAk", "dBk", "dAo", "dBo"), grads, want[4]):
        close(g, w, 24, name)
    for m, before, g in zip(net.members, old, grads):
        # the first step from zero: lr g / (|g| + eps), and the decay
        moved = (before.double() * (1 - 1e-5) - m["master"].double())
        big = g.double().abs() > 1e-5 * g.double().abs().max()
        assert torch.equal(m["weight"], m["master"].bfloat16()) and ((moved - 1e-3 * g.double().sign())[big & (g.double().abs() > 1e-4)].abs() <= 1e-6).all()


def test_captured_step_beside_an_eager_one():
    a, b = (Net(256, 4, 100, 2000, 16, "rms", 8) for _ in range(2))
    X, R = a.q.draw(100, 256).bfloat16(), a.q.draw(100, 256).bfloat16()
    Net(256, 4, 100, 2000, 16, "rms", 8, seed=9).step(X, R)                # launch configurations, outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = a.step(X, R)
    for _ in range(3):
        graph.replay()
        eager = b.step(X, R)
        torch.cuda.synchronize()
        assert torch.equal(captured[0], eager[0]) and torch.equal(captured[1], eager[1])
        for x, y in zip(a.members, b.members):
            assert all(torch.equal(x[k].float(), y[k].float()) for k in x)
    assert int(a.step_number) == 4


def test_two_streams():
    """The calls that stand beside the products, on two streams at once: the results of one after the other."""
    nets = [Net(512, 8, 200, 3000, 16, "layer", 32, seed=s) for s in (1, 5)]
    data = [(n.q.draw(200, 512).bfloat16(), n.q.draw(200, 512).bfloat16()) for n in nets]

    def calls(net, X, R):
        (g, b), _ = net.norms
        y, rstd, mean, h = lw.lowra_norm_forward(X, g, b, residual=R)
        t = lw.lowra_rotary(net.heads(y), net.positions, net.turns)
        loss, dX = lw.lowra_cross_entropy(y, net.head, net.labels, want_grad=True)
        out = [y, t, loss, dX, *lw.lowra_norm_backward(dX, h, g, rstd, mean=mean, want_params=True)]
        members = [{**m, "grad": f * 0.5, **{k: m[k].clone() for k in ("master", "m", "v", "weight")}} for m, f in zip(net.members, net.factors())]
        lw.lowra_adamw(members, 1e-3, step=3)
        return out + [m["master"] for m in members]

    want = [calls(n, *d) for n, d in zip(nets, data)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in nets]
    for _ in range(5):
        got = []
        for n, d, s in zip(nets, data, streams):
            with torch.cuda.stream(s):
                got.append(calls(n, *d))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w))
