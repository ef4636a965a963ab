"""What the norm, the rotary positions and the optimiser of adaptive moments refuse before any GPU is asked for, through the C interface; the table of rotary frequencies."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest

import paper_2502_08141_b200 as lw


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2502_08141_b200 import build
    build.build()


AT = 1 << 20        # addresses that are never used: every call here ends at a check


def test_norm_forward():
    def call(X=AT, residual=None, weight=2 * AT, bias=3 * AT, fp32=0, M=4, N=64, kind=0, eps=1e-5, sum=None, Y=4 * AT, mean=5 * AT, rstd=6 * AT):
        return lw.lib().lowra_norm_forward(X, residual, weight, bias, fp32, M, N, kind, eps, sum, Y, mean, rstd, None)

    for bad in (dict(X=None), dict(weight=None), dict(Y=None), dict(bias=None), dict(residual=AT), dict(sum=7 * AT)):
        assert call(**bad) == lw.LOWRA_ERR_NULL, bad
    for bad in (dict(M=0), dict(M=(1 << 30) + 1), dict(N=0), dict(N=60), dict(N=16392), dict(kind=2), dict(kind=-1), dict(eps=-1.0), dict(eps=math.nan), dict(kind=1),
                dict(kind=1, bias=None), dict(Y=AT + 64), dict(Y=2 * AT), dict(mean=AT), dict(rstd=5 * AT), dict(residual=7 * AT, sum=4 * AT),
                dict(residual=7 * AT, sum=AT + 16), dict(residual=7 * AT, sum=7 * AT, Y=7 * AT)):
        assert call(**bad) == lw.LOWRA_ERR_SHAPE, bad
    for name in ("X", "weight", "bias", "Y", "mean", "rstd"):
        assert call(**{name: 8 * AT + 8}) == lw.LOWRA_ERR_ALIGN, name


def test_norm_backward():
    def call(dY=AT, X=2 * AT, weight=3 * AT, fp32=0, mean=4 * AT, rstd=5 * AT, dsum=None, M=4, N=64, dX=6 * AT, dw=7 * AT, db=None, ws=8 * AT, n=0):
        return lw.lib().lowra_norm_backward(dY, X, weight, fp32, mean, rstd, dsum, M, N, dX, dw, db, ws, n, None)

    for name in ("dY", "X", "weight", "rstd", "dX"):
        assert call(**{name: None}) == lw.LOWRA_ERR_NULL, name
        assert call(**{name: 9 * AT + 8}) == lw.LOWRA_ERR_ALIGN, name
    assert call() == lw.LOWRA_ERR_WORKSPACE and call(ws=None, n=1 << 20) == lw.LOWRA_ERR_WORKSPACE and call(ws=8 * AT + 16, n=1 << 20) == lw.LOWRA_ERR_WORKSPACE
    for bad in (dict(M=0), dict(N=12), dict(N=16400), dict(mean=None, db=9 * AT), dict(dX=AT + 16), dict(dX=3 * AT), dict(dw=AT), dict(dw=6 * AT + 256), dict(db=7 * AT),
                dict(dsum=9 * AT, dX=9 * AT + 32), dict(dX=8 * AT), dict(dw=8 * AT), dict(X=8 * AT), dict(rstd=8 * AT)):
        assert call(**{"n": 1 << 20, **bad}) == lw.LOWRA_ERR_SHAPE, bad
    assert lw.lowra_norm_workspace_bytes(0, 64) == 0 and lw.lowra_norm_workspace_bytes(4, 60) == 0 and lw.lowra_norm_workspace_bytes(4, 16392) == 0
    for M, N in ((1, 8), (17, 264), (8192, 512), (100000, 16384)):
        size = lw.lowra_norm_workspace_bytes(M, N)
        assert size % 256 == 0 and 8 * N <= size <= 148 * 8 * N + 256


def part(x=AT, out=2 * AT, heads=4, xt=512, xh=128, ot=512, oh=128):
    return lw._CRotaryPart(x, out, xt, xh, ot, oh, heads)


def rotary(*parts, count=None, M=8, D=128, dim=128, positions=16 * AT, turns=17 * AT):
    arr = (lw._CRotaryPart * 3)(*parts)
    return lw.lib().lowra_rotary(arr, len(parts) if count is None else count, M, D, dim, positions, turns, 1.0, 0, 0, None)


def test_rotary():
    assert lw.lib().lowra_rotary(None, 1, 8, 128, 128, AT, AT, 1.0, 0, 0, None) == lw.LOWRA_ERR_NULL
    assert rotary(part(), positions=None) == lw.LOWRA_ERR_NULL and rotary(part(), turns=None) == lw.LOWRA_ERR_NULL
    assert rotary(part(x=None)) == lw.LOWRA_ERR_NULL and rotary(part(), part(out=None)) == lw.LOWRA_ERR_NULL
    for bad in (dict(count=0), dict(count=3), dict(M=0), dict(D=8, dim=8), dict(D=132), dict(dim=120), dict(dim=0), dict(D=64, dim=128), dict(D=4104, dim=16), dict(D=2048, dim=1040)):
        assert rotary(part(), **bad) == lw.LOWRA_ERR_SHAPE, bad
    for bad in (dict(heads=0), dict(heads=65537), dict(xt=516), dict(xh=-128), dict(ot=0), dict(oh=0), dict(oh=120), dict(ot=504), dict(ot=128, oh=512)):
        assert rotary(part(**bad)) == lw.LOWRA_ERR_SHAPE, bad
    assert rotary(part(x=AT + 2)) == lw.LOWRA_ERR_ALIGN and rotary(part(), positions=AT + 2) == lw.LOWRA_ERR_ALIGN and rotary(part(), turns=AT + 8) == lw.LOWRA_ERR_ALIGN
    # memory shared: with the input but not in place, with the other part, the positions, the table
    for bad in (part(out=AT + 16), part(out=AT, ot=1024), part(out=16 * AT), part(out=17 * AT - 512)):
        assert rotary(bad) == lw.LOWRA_ERR_SHAPE
    assert rotary(part(), part(x=4 * AT)) == lw.LOWRA_ERR_SHAPE and rotary(part(), part(x=4 * AT, out=AT)) == lw.LOWRA_ERR_SHAPE
    # slices of one projection: in place beside each other is fine (the call then ends at the alignment of the table), one value over is not
    q, k = part(out=AT, xt=1536, ot=1536), part(x=AT + 1024, out=AT + 1024, xt=1536, ot=1536)
    assert rotary(q, k, turns=AT + 8) == lw.LOWRA_ERR_ALIGN
    assert rotary(q, part(x=4 * AT, out=AT + 1008, xt=1536, ot=1536)) == lw.LOWRA_ERR_SHAPE
    assert rotary(q, part(x=4 * AT, out=AT + 2064, xt=1536, ot=1536)) == lw.LOWRA_ERR_SHAPE


def test_turns():
    for bad in (dict(dim=0), dict(dim=63), dict(dim=1026), dict(base=1.0), dict(base=math.nan), dict(kind="linear", factor=0.5), dict(kind="yarn", factor=2.0, original=0.0),
                dict(kind="bands", factor=2.0, low=4.0, high=4.0), dict(kind="yarn", factor=2.0, beta_slow=0.0)):
        with pytest.raises(lw.LowraError) as e:
            lw.lowra_rotary_turns(**{"dim": 64, **bad})
        assert e.value.code == lw.LOWRA_ERR_SHAPE, bad
    with pytest.raises(ValueError, match="kind"):
        lw.lowra_rotary_turns(64, kind="longer")


@pytest.mark.parametrize("kind, options", [("none", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)), ("yarn", dict(factor=16.0, original=4096)),
                                           ("bands", dict(factor=8.0, original=8192, low=1.0, high=4.0))])
@pytest.mark.parametrize("dim, base", [(2, 1e4), (128, 1e4), (64, 5e5), (1024, 1e6)])
def test_turns_table(kind, options, dim, base):
    """The table against the formulas in fp64, to their rounding (2^-48 relative: a power's exponent of up to 14 is off by 2^-50) and the table's own, half of 2^-64 (which for the
    lowest frequencies, 2^-17 of a turn and less, is more than the relative part)."""
    turns, scale = lw.lowra_rotary_turns(dim, base, kind, **options)
    i, f = np.arange(dim // 2), options.get("factor", 1.0)
    b = base * f ** (dim / (dim - 2)) if kind == "ntk" and dim > 2 else base
    w = b ** (-2.0 * i / dim)
    if kind == "linear":
        w = w / f
    if kind == "yarn":
        place = lambda t: dim * math.log(4096 / (t * 2 * math.pi)) / (2 * math.log(b))  # noqa: E731
        low, high = max(math.floor(place(32.0)), 0), min(math.ceil(place(1.0)), dim - 1)
        t = np.clip((i - low) / max(high - low, 0.001), 0, 1)
        w = w * (1 - t) + w / f * t
    if kind == "bands":
        t = np.clip((8192 * w / (2 * math.pi) - 1.0) / 3.0, 0, 1)
        w = w * t + w / f * (1 - t)
    assert turns.shape == (dim // 2,) and turns.dtype == np.uint64
    for got, want in zip(turns, w):
        want = Fraction(float(want)) / Fraction(2 * math.pi)
        assert abs(Fraction(int(got), 1 << 64) - want) <= Fraction(1, 1 << 48) * want + Fraction(1, 1 << 65)
    assert scale == pytest.approx(0.1 * math.log(16.0) + 1.0 if kind == "yarn" else 1.0, rel=2.0 ** -23)


def test_adamw():
    def call(count=1, members=True, with_step=True, step={}, **fields):
        arr = (lw._CAdamwMember * 4200)()
        base = dict(grad_dev=AT, master_dev=2 * AT, master_out_dev=2 * AT, weight_dev=None, m_dev=3 * AT, m_out_dev=3 * AT, v_dev=4 * AT, v_out_dev=4 * AT, m_scale_dev=5 * AT,
                    m_scale_out_dev=5 * AT, v_scale_dev=6 * AT, v_scale_out_dev=6 * AT, n=1000)
        for i, m in enumerate(arr[:min(max(count, 1), 2)]):
            for k, v in {**base, **fields}.items():
                setattr(m, k, v + (i << 30) if v and k != "n" else v)
        s = lw._CAdamwStep(1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None, 8, 0)
        for k, v in step.items():
            setattr(s, k, v)
        return lw.lib().lowra_adamw(arr if members else None, count, ctypes.byref(s) if with_step else None, None)

    assert call(members=False) == lw.LOWRA_ERR_NULL and call(with_step=False) == lw.LOWRA_ERR_NULL
    for name in ("grad_dev", "master_dev", "master_out_dev", "m_dev", "m_out_dev", "v_dev", "v_out_dev", "m_scale_dev", "m_scale_out_dev", "v_scale_dev", "v_scale_out_dev"):
        assert call(**{name: None}) == lw.LOWRA_ERR_NULL, name
        assert call(**{name: 9 * AT + (2 if "scale" in name else 8)}) == lw.LOWRA_ERR_ALIGN, name
    assert call(weight_dev=AT + 4) == lw.LOWRA_ERR_ALIGN and call(count=2, weight_dev=9 * AT + 2) == lw.LOWRA_ERR_ALIGN
    for bad in (dict(count=0), dict(count=4097), dict(n=0), dict(n=-1), dict(n=(1 << 36) + 1), dict(weight_dev=AT), dict(m_out_dev=2 * AT), dict(master_out_dev=2 * AT + 16),
                dict(v_out_dev=AT + 1984), dict(m_scale_out_dev=6 * AT + 12), dict(v_scale_out_dev=4 * AT + 996)):
        assert call(**bad) == lw.LOWRA_ERR_SHAPE, bad
    for bad in (dict(bits=16), dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(eps=-1.0), dict(eps=math.nan), dict(lr_dev=3 * AT + 4), dict(step_dev=5 * AT),
                dict(grad_scale_dev=2 * AT)):
        assert call(step=bad) == lw.LOWRA_ERR_SHAPE, bad
    for name in ("lr_dev", "step_dev", "grad_scale_dev"):
        assert call(step={name: 9 * AT + 2}) == lw.LOWRA_ERR_ALIGN


def test_cross_entropy():
    def call(X=AT, W=2 * AT, labels=3 * AT, weights=None, M=4, V=100, K=64, loss=4 * AT, dX=5 * AT, ws=64 * AT, n=1 << 40):
        return lw.lib().lowra_cross_entropy(X, W, labels, weights, M, V, K, -100, 1.0, loss, dX, ws, n, None)

    for name in ("X", "W", "labels", "loss", "ws"):
        assert call(**{name: None}) == lw.LOWRA_ERR_NULL, name
    for name in ("X", "W", "labels", "weights", "loss", "dX"):
        assert call(**{name: 9 * AT + 8}) == lw.LOWRA_ERR_ALIGN, name
    for bad in (dict(M=0), dict(M=(1 << 30) + 1), dict(V=0), dict(V=(1 << 24) + 1), dict(K=56), dict(K=68), dict(K=65544), dict(dX=AT), dict(loss=AT + 16), dict(loss=5 * AT), dict(dX=2 * AT + 128),
                dict(weights=4 * AT), dict(loss=3 * AT + 16), dict(dX=64 * AT), dict(W=64 * AT)):
        assert call(**bad) == lw.LOWRA_ERR_SHAPE, bad
    size = lw.lowra_cross_entropy_workspace_bytes(4, 100, 64, True)
    assert call(n=size - 1) == lw.LOWRA_ERR_WORKSPACE and call(ws=64 * AT + 64) == lw.LOWRA_ERR_WORKSPACE
    for M, V, K in ((0, 100, 64), (4, 0, 64), (4, 100, 60), (4, 100, 32)):
        assert lw.lowra_cross_entropy_workspace_bytes(M, V, K, True) == 0
    # the logits are never kept: however many tokens and words, a piece of exponentials of 128 MB and O
    assert lw.lowra_cross_entropy_workspace_bytes(4096, 32000, 4096, False) < 20 << 20
    for M, V in ((4096, 32000), (100000, 32000), (4096, 1 << 24), (64, 1 << 24)):
        assert lw.lowra_cross_entropy_workspace_bytes(M, V, 1024, True) < (160 << 20) + 17 * 4096 * 1024 * 4
