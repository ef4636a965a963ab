"""The norm and its gradient against the formulas in fp64, within bounds that count roundings: u = 2^-24 for an operation in fp32, 2^-8 relative for one to bf16."""
import pytest
import torch

import paper_2502_08141_b200 as lw

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


def make(M, N, kind, params, residual, seed=0, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + M * 31 + N)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X = (r(M, N) * torch.exp(0.5 * r(N)) * scale + shift).bfloat16()
    return dict(X=X, weight=(1 + 0.3 * r(N)).to(params), bias=r(N).to(params) if kind == "layer" else None, residual=r(M, N).bfloat16() if residual else None,
                dY=r(M, N).bfloat16(), dsum=r(M, N).bfloat16() if residual else None)


def statistics(h, layer):
    h = h.double()
    mean = h.mean(1, keepdim=True) if layer else torch.zeros_like(h[:, :1])
    return mean, 1 / torch.sqrt(((h - mean) ** 2).mean(1, keepdim=True) + EPS)


def check_forward(c, kind, Y, rstd, mean, h):
    layer = kind == "layer"
    want_h = c["X"] if c["residual"] is None else (c["X"].float() + c["residual"].float()).bfloat16()
    if c["residual"] is not None:
        assert torch.equal(h, want_h)
    x = want_h.double()
    mu, rs = statistics(want_h, layer)
    w = c["weight"].double()
    d = (x - mu) * rs * w
    y = d + (c["bias"].double() if layer else 0.0)
    # a sum of N values by 8 or 16 to a thread and trees: fewer than 32 roundings on any way, of the mean of magnitudes; the variance likewise, halved by the root
    wide = x.abs().mean(1, keepdim=True)
    assert ((rstd.double()[:, None] - rs).abs() <= 48 * U * rs * (1 + rs * wide * layer)).all()
    if layer:
        assert ((mean.double()[:, None] - mu).abs() <= 34 * U * wide).all()
    tol = 2.0 ** -8 * y.abs() + U * (60 * d.abs() * (1 + rs * wide * layer) + 34 * layer * rs * wide * w.abs() + 2 * y.abs())
    assert ((Y.double() - y).abs() <= tol).all()


SHAPES = [(1, 8), (1, 4096), (3, 256), (5, 1024), (17, 264), (333, 5120), (149, 8192), (150, 8200), (7, 16384), (1000, 1800), (2000, 32), (700, 512)]


@pytest.mark.parametrize("M, N", SHAPES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("params", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_forward(M, N, kind, params, residual):
    c = make(M, N, kind, params, residual)
    Y, rstd, mean, h = lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS, kind=kind, residual=c["residual"])
    assert (mean is None) == (kind == "rms") and (h is None) == (not residual)
    check_forward(c, kind, Y, rstd, mean, h)


def test_forward_far_from_zero_and_in_place():
    """A mean a thousand times the spread; sum and Y in the places of the inputs."""
    c = make(40, 1024, "layer", torch.float32, True, shift=1000.0)
    Y, rstd, mean, h = lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS, residual=c["residual"])
    check_forward(c, "layer", Y, rstd, mean, h)
    X, residual = c["X"].clone(), c["residual"].clone()
    got = lw.lowra_norm_forward(X, c["weight"], c["bias"], eps=EPS, residual=residual, sum=residual, Y=X)
    assert got[0] is X and got[3] is residual and torch.equal(X, Y) and torch.equal(residual, h) and torch.equal(got[1], rstd) and torch.equal(got[2], mean)
    X = c["X"].clone()
    lw.lowra_norm_forward(X, c["weight"], c["bias"], eps=EPS, Y=X)
    assert torch.equal(X, lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS)[0])


def test_rows_of_zeros_and_bad_values():
    """A row of zeros gives the bias; a NaN or an infinity stays in its row."""
    c = make(6, 512, "layer", torch.bfloat16, False)
    c["X"][1] = 0
    good = lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS)[0]
    assert torch.equal(good[1], c["bias"])
    bad = c["X"].clone()
    bad[2, 5], bad[4, 100] = float("nan"), float("inf")
    Y = lw.lowra_norm_forward(bad, c["weight"], c["bias"], eps=EPS)[0]
    assert Y[2].isnan().all() and Y[4].isnan().all() and torch.equal(Y[[0, 1, 3, 5]], good[[0, 1, 3, 5]])
    dX, dw, db = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], *reversed(statistics32(c["X"])), want_params=True)
    assert dX.isfinite().all() and dw.isfinite().all() and db.isfinite().all()


def statistics32(h, layer=True):
    mean, rstd = statistics(h, layer)
    return (mean[:, 0].float().contiguous() if layer else None), rstd[:, 0].float().contiguous()


def check_backward(c, kind, mean, rstd, dX, dw, db):
    layer, N, M = kind == "layer", c["X"].shape[1], c["X"].shape[0]
    rs, dY, w = rstd.double()[:, None], c["dY"].double(), c["weight"].double()
    d = c["X"].double() - (mean.double()[:, None] if layer else 0.0)
    xh, g = d * rs, dY * w
    along, level = (g * xh).mean(1, keepdim=True), g.mean(1, keepdim=True) * layer
    dx = rs * (g - xh * along - level)
    total = dx + (c["dsum"].double() if c["dsum"] is not None else 0.0)
    # the two means as sums of N products, 32 roundings and their own three; the rest a handful each
    slack = rs * (g.abs() * 4 + xh.abs() * (40 * (g * xh).abs().mean(1, keepdim=True)) + 40 * g.abs().mean(1, keepdim=True) * layer) + 4 * total.abs()
    assert ((dX.double() - total).abs() <= 2.0 ** -8 * total.abs() + U * slack).all()
    if dw is not None:
        assert ((dw.double() - (dY * xh).sum(0)).abs() <= (M + 8) * U * (dY * xh).abs().sum(0)).all()
    if db is not None:
        assert ((db.double() - dY.sum(0)).abs() <= (M + 4) * U * dY.abs().sum(0)).all()


@pytest.mark.parametrize("M, N", SHAPES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("params, residual, sums", [(torch.bfloat16, False, True), (torch.float32, True, True), (torch.bfloat16, True, False)])
def test_backward(M, N, kind, params, residual, sums):
    c = make(M, N, kind, params, residual, seed=1)
    mean, rstd = statistics32(c["X"], kind == "layer")
    dX, dw, db = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, dsum=c["dsum"], want_params=sums)
    assert (dw is not None) == sums and (db is not None) == (sums and kind == "layer")
    check_backward(c, kind, mean, rstd, dX, dw, db)
    again = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, dsum=c["dsum"], want_params=sums)
    assert all(a is b or torch.equal(a, b) for a, b in zip((dX, dw, db), again))


@pytest.mark.parametrize("place", ["dY", "X", "dsum"])
def test_backward_in_place_and_one_gradient(place):
    c = make(300, 1288, "layer", torch.bfloat16, True, seed=2)
    mean, rstd = statistics32(c["X"])
    dX, dw, db = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, dsum=c["dsum"], want_params=True)
    only = torch.empty(1288, device="cuda")
    a = {k: c[k].clone() for k in ("dY", "X", "dsum")}
    got = lw.lowra_norm_backward(a["dY"], a["X"], c["weight"], rstd, mean=mean, dsum=a["dsum"], dX=a[place], dbias=only)
    assert got[0] is a[place] and got[1] is None and torch.equal(got[0], dX) and torch.equal(only, db)


def test_gradient_against_differences():
    """A step along a direction changes sum(dY * Y) as dX, dweight and dbias say: in fp64 by the formula, whose value the forward call agrees with above."""
    c = make(9, 256, "layer", torch.float32, False, seed=3)
    X, w, b, dY = (c[k].double() for k in ("X", "weight", "bias", "dY"))
    f = lambda X, w, b: (dY * ((X - X.mean(1, keepdim=True)) / torch.sqrt(X.var(1, unbiased=False, keepdim=True) + EPS) * w + b)).sum()  # noqa: E731
    mean, rstd = statistics32(c["X"])
    dX, dw, db = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, want_params=True)
    g = torch.Generator(device="cuda").manual_seed(5)
    for i, grad in enumerate((dX, dw, db)):
        at = [X, w, b]
        v = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * v, at[i] - h * v
        slope = (f(*up) - f(*down)) / (2 * h)
        # roundings of dX to bf16 (2^-8 each, of all elements); of the differences 1e-16 |f| / h and h^2
        assert (slope - (grad.double() * v).sum()).abs() <= 2.0 ** -8 * (grad.double() * v).abs().sum() + 1e-6 * dY.abs().sum()


def test_other_stream_and_graph():
    c = make(333, 4096, "rms", torch.bfloat16, True, seed=4)
    want = lw.lowra_norm_forward(c["X"], c["weight"], eps=EPS, kind="rms", residual=c["residual"])
    want_b = lw.lowra_norm_backward(c["dY"], want[3], c["weight"], want[1], dsum=c["dsum"], want_params=True)
    out = dict(sum=torch.empty_like(c["X"]), Y=torch.empty_like(c["X"]), rstd=torch.empty(333, device="cuda"))
    back = dict(dX=torch.empty_like(c["X"]), dweight=torch.empty(4096, device="cuda"), workspace=torch.empty(lw.lowra_norm_workspace_bytes(333, 4096), dtype=torch.uint8, device="cuda"))

    def both(stream=None):
        lw.lowra_norm_forward(c["X"], c["weight"], eps=EPS, kind="rms", residual=c["residual"], stream=stream, **out)
        lw.lowra_norm_backward(c["dY"], out["sum"], c["weight"], out["rstd"], dsum=c["dsum"], stream=stream, **back)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    torch.cuda.synchronize()
    assert torch.equal(out["Y"], want[0]) and torch.equal(back["dX"], want_b[0]) and torch.equal(back["dweight"], want_b[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for t in (*out.values(), back["dX"], back["dweight"]):
        t.fill_(7)
    back["workspace"].fill_(255)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out["Y"], want[0]) and torch.equal(back["dX"], want_b[0]) and torch.equal(back["dweight"], want_b[1])


def test_refusals():
    c = make(4, 64, "layer", torch.bfloat16, False)
    mean, rstd = statistics32(c["X"])
    for bad in (dict(kind="batch"), dict(X=c["X"].float()), dict(X=c["X"][:, ::2]), dict(X=c["X"][0]), dict(weight=c["weight"].float()), dict(weight=c["weight"][:32]),
                dict(weight=c["weight"].double(), bias=None), dict(residual=c["X"][:2]), dict(Y=c["X"].cpu()), dict(mean=mean[:3]), dict(rstd=rstd.double())):
        with pytest.raises(ValueError):
            lw.lowra_norm_forward(**{**dict(X=c["X"], weight=c["weight"], bias=c["bias"]), **bad})
    for bad in (dict(dY=None), dict(dY=c["X"][:3]), dict(rstd=rstd[:2]), dict(dweight=torch.empty(63, device="cuda")), dict(dsum=c["X"].float()), dict(dX=c["X"].cpu())):
        with pytest.raises(ValueError):
            lw.lowra_norm_backward(**{**dict(dY=c["dY"], X=c["X"], weight=c["weight"], rstd=rstd, mean=mean), **bad})
    for call in (lambda: lw.lowra_norm_forward(c["X"], c["weight"]), lambda: lw.lowra_norm_forward(c["X"], c["weight"], sum=torch.empty_like(c["X"]), kind="rms"),
                 lambda: lw.lowra_norm_forward(c["X"][:0], c["weight"], c["bias"]), lambda: lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], Y=c["X"].view(-1)[:0].view(0, 64)),
                 lambda: lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, dbias=torch.empty(64, device="cuda"))):
        with pytest.raises((lw.LowraError, ValueError)):
            call()


@pytest.mark.parametrize("M, N", [(1, 8), (3, 40), (832, 256), (833, 256), (208, 256), (209, 256), (320, 256), (321, 256), (1280, 256), (1281, 256), (700, 504), (1024, 1024), (1025, 1024), (513, 1024), (2048, 1288), (2049, 1288), (149, 2056), (300, 4104), (1536, 8200), (1537, 8200), (77, 16384)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_backward_of_few_rows_and_of_more(M, N, kind):
    """Sizes about which columns and rows become CTAs of one launch, of two where dX takes an input's place, or of none; odd ends of the columns; one gradient of the two."""
    c = make(M, N, kind, torch.float32, True, seed=6)
    mean, rstd = statistics32(c["X"], kind == "layer")
    dX, dw, db = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, dsum=c["dsum"], want_params=True)
    check_backward(c, kind, mean, rstd, dX, dw, db)
    alone = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, dsum=c["dsum"])
    check_backward(c, kind, mean, rstd, *alone)
    for place in ("dY", "X", "dsum"):
        a = {k: c[k].clone() for k in ("dY", "X", "dsum")}
        only = torch.full((N,), 7.0, device="cuda")
        out = lw.lowra_norm_backward(a["dY"], a["X"], c["weight"], rstd, mean=mean, dsum=a["dsum"], dX=a[place], dweight=only)
        assert out[0] is a[place] and out[1] is only and out[2] is None
        check_backward(c, kind, mean, rstd, *out)
        assert all(torch.equal(a[k], c[k]) for k in a if k != place)
