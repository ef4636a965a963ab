"""What stands behind a product, in 64 bits, with bounds on what fp32 arithmetic and the roundings to bf16 may be off by."""
import math

import torch

import synth_inputs as si

HALF = torch.finfo(torch.bfloat16).eps / 2     # a rounding to bf16, relative: 2^-8
F32 = torch.finfo(torch.float32).eps           # twice a rounding to fp32: 2^-23, for sums that are cut off rather than rounded
ACT_ERROR = 5e-4                               # of an activation, relative (gelu's polynomial 4e-4; the others 1e-6)
STEEPEST = 1.13                                # no activation is steeper


def activate(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "gelu":
        return 0.5 * z * torch.special.erfc(-z * math.sqrt(0.5))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z)


def slope(z, kind):
    if kind == "none":
        return torch.ones_like(z)
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return 0.5 * torch.special.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    if kind == "gelu_tanh":
        th = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * c * (1 + 3 * 0.044715 * z * z)
    p = torch.sigmoid(z)
    return p * (1 + z * (1 - p))


def forward(W_hat, X, A, B, s, bias=None, activation="none", multiply=None, residual=None):
    """-> Y, Z and how far the outputs may be off.  Sums of K + r products in fp32; s X A is rounded to bf16 once."""
    W, x, a, b = (t.double() for t in (W_hat, X, A, B))
    T = s * (x @ a)
    z = x @ W.t() + T @ b
    off = (W.shape[1] + A.shape[1] + 4) * F32 * (x.abs() @ W.abs().t() + T.abs() @ b.abs()) + HALF * (T.abs() @ b.abs())
    if bias is not None:
        z = z + bias.double()
        off = off + F32 * z.abs()
    h = activate(z, activation)
    h_off = off if activation == "none" else STEEPEST * off + ACT_ERROR * h.abs()
    y, y_off = h, h_off
    if multiply is not None:
        y, y_off = h * multiply.double(), h_off * multiply.double().abs()
    if residual is not None:
        y = y + residual.double()
    y_off = y_off + 4 * F32 * (y.abs() + (0 if residual is None else residual.double().abs()))
    return y, z, y_off * (1 + HALF) + HALF * y.abs() + 1e-30, off * (1 + HALF) + HALF * z.abs() + 1e-30


class Weight:
    """A quantised weight with tables for `n` adapters, its decoded values and low-rank factors."""

    def __init__(self, N, K, mix, r, n=1, natural=False, deal=True, seed=1):
        import paper_2502_08141_b200 as lw

        gen = torch.Generator(device="cuda").manual_seed(1000 * seed + N + K + r)
        self.draw = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)
        precs = si.precisions(N, mix, matrix_id=seed)
        self.layout = lw.Layout(precs, K, natural=natural)
        if deal:
            self.layout.build_deal()
        maps, thr = (torch.from_numpy(t).cuda() for t in si.standin_codebooks(precs))
        self.packed, self.absmax = lw.lowra_encode(self.layout, self.draw(N, K) * 0.02, thr)
        self.maps = (maps.unsqueeze(0) * (1.0 + 0.1 * torch.arange(n, device="cuda").view(n, 1, 1))).contiguous()
        self.W_hat = [lw.lowra_decode(self.layout, self.packed, self.absmax, t) for t in self.maps]
        self.A, self.B = self.draw(n, K, r).bfloat16() * 0.05, self.draw(n, r, N).bfloat16() * 0.05
        self.N, self.K, self.r = N, K, r

    def head(self, a=0):
        return self.layout, self.packed, self.absmax, self.maps[a]
