"""The gradient through bias, activation, second factor and residual (lowra_epilogue_backward) against the formula in 64 bits, against differences, and at values where it can go
wrong; in place, repeated, beside other rows, and its refusals."""
import pytest
import torch

from epilogue_reference import F32, HALF, activate, slope

pytestmark = pytest.mark.gpu

ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
SLOPE_ERROR = 8 * F32          # act and act', absolute for |z| <= 8: a handful of fp32 operations on values below 2


def inputs(M, N, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda scale: (torch.randn(M, N, device="cuda", generator=gen) * scale).bfloat16()
    return draw(1e-3), draw(1.5).clamp(-8, 8), draw(1.0)


@pytest.mark.parametrize("M,N", [(1, 8), (1, 1024), (16, 1024), (17, 264), (333, 4104), (1001, 520), (2500, 1032), (40, 13824)])
@pytest.mark.parametrize("activation", ACTIVATIONS)
def test_against_the_formula(M, N, activation):
    import paper_2502_08141_b200 as lw

    dY, pre, mul = inputs(M, N)
    for with_mul in (False, True):
        m = mul if with_mul else None
        dh = dY.double() * (mul.double() if with_mul else 1.0)
        dz = dh * slope(pre.double(), activation)
        dz_off = SLOPE_ERROR * dh.abs() + 4 * F32 * dz.abs()
        for bias in (False, True):
            out = [torch.full((M + 1, N), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            got = lw.lowra_epilogue_backward(dY, pre, activation, multiply=m, dZ=out[0][:M], dmultiply=out[1][:M] if with_mul else None, want_bias=bias)
            assert ((got[0].double() - dz).abs() <= dz_off * (1 + HALF) + HALF * dz.abs() + 1e-38).all()
            assert (got[1] is None) == (not with_mul) and (got[2] is None) == (not bias)
            if with_mul:
                dm = dY.double() * activate(pre.double(), activation)
                off = SLOPE_ERROR * (1 + pre.double().abs()) * dY.double().abs()
                assert ((got[1].double() - dm).abs() <= off * (1 + HALF) + HALF * dm.abs() + 1e-38).all()
            if bias:
                total = dz.sum(0)
                off = dz_off.sum(0) + (M + 16) * F32 * dz.abs().sum(0) / 8 + 16 * F32 * dz.abs().sum(0)     # (no chain of additions is longer than M / 8 + 16)
                assert got[2].dtype == torch.float32 and ((got[2].double() - total).abs() <= off + 1e-38).all()
            assert bool((out[0][M:] == 7.0).all()) and bool((out[1][M:] == 7.0).all())
            again = lw.lowra_epilogue_backward(dY, pre, activation, multiply=m, want_bias=bias, stream=torch.cuda.current_stream())
            assert all(a is None or torch.equal(a, b) for a, b in zip(again, got))


@pytest.mark.parametrize("M,N", [(2, 72), (63, 8), (65, 136), (127, 4104), (128, 9472), (129, 9472), (128, 9480)])
def test_few_rows(M, N):
    """On both sides of the bounds of the narrow CTAs, which hold all rows each."""
    import paper_2502_08141_b200 as lw

    test_against_the_formula(M, N, "silu")
    dY, pre, mul = inputs(M, N)
    whole = lw.lowra_epilogue_backward(dY, pre, "gelu", multiply=mul, want_bias=True)
    if M <= 128 and N <= 9472:
        assert lw.lowra_epilogue_workspace_bytes(M, N) == (4 * N + 255) // 256 * 256
    place = dY.clone()
    got = lw.lowra_epilogue_backward(place, pre, "gelu", multiply=mul, dZ=place, want_bias=True)
    assert got[0].data_ptr() == place.data_ptr() and torch.equal(got[0], whole[0]) and torch.equal(got[2], whole[2])


@pytest.mark.parametrize("activation", ACTIVATIONS)
def test_against_differences(activation):
    import paper_2502_08141_b200 as lw

    M, N, h = 7, 520, 1e-5
    dY, pre, mul = inputs(M, N, seed=3)
    if activation == "relu":
        pre = torch.where(pre.abs() < 0.01, torch.ones_like(pre), pre)       # (away from the corner)
    z, m, g = pre.double(), mul.double(), dY.double()
    loss = lambda z, m: (g * activate(z, activation) * m)                     # elementwise: every output depends on its own inputs only
    dz = (loss(z + h, m) - loss(z - h, m)) / (2 * h)
    dm = (loss(z, m + h) - loss(z, m - h)) / (2 * h)
    got = lw.lowra_epilogue_backward(dY, pre, activation, multiply=mul)
    # a central difference is off by h^2 / 6 times the third derivative (below 3) and by the rounding of its terms over h
    far = 3 * h * h * (g * m).abs() + 2.0 ** -52 * 10 * g.abs() * (1 + m.abs()) / h
    assert ((got[0].double() - dz).abs() <= far + (SLOPE_ERROR * (g * m).abs()) + HALF * 1.01 * dz.abs() + 1e-38).all()
    assert ((got[1].double() - dm).abs() <= far + SLOPE_ERROR * (1 + z.abs()) * g.abs() + HALF * 1.01 * dm.abs() + 1e-38).all()


def test_far_out_and_no_numbers():
    import paper_2502_08141_b200 as lw

    z = torch.tensor([0.0, -0.0, 30.0, -30.0, 1e4, -1e4, 3e38, -3e38, float("nan")] + [1.0] * 7, device="cuda").bfloat16().repeat(3, 1)
    dY = torch.full_like(z, 2.0)
    for activation in ACTIVATIONS[1:]:
        dZ, _, dbias = lw.lowra_epilogue_backward(dY, z, activation, want_bias=True)
        want = {"relu": [0.0, 0.0]}.get(activation, [1.0, 1.0])
        assert dZ[0, :2].tolist() == want, activation
        assert dZ[0, 2].item() == 2.0 and dZ[0, 4].item() == 2.0 and dZ[0, 3].abs().item() < 1e-9 and dZ[0, 5].item() == 0.0
        assert dZ[0, 6].item() == 2.0 and dZ[0, 7].item() == 0.0
        assert bool(dbias[9:].isfinite().all()) and bool(dZ[:, 9:].isfinite().all())
        assert activation == "relu" or (bool(dZ[0, 8].isnan()) and bool(dbias[8].isnan()))


@pytest.mark.parametrize("M,N", [(5, 264), (700, 1032)])
def test_in_place(M, N):
    import paper_2502_08141_b200 as lw

    for place in ("dY", "pre"):
        dY, pre, mul = inputs(M, N, seed=5)
        want = lw.lowra_epilogue_backward(dY, pre, "silu", multiply=mul, want_bias=True)
        a = dict(dY=dY.clone(), pre=pre.clone())
        m = mul.clone()
        got = lw.lowra_epilogue_backward(a["dY"], a["pre"], "silu", multiply=m, dZ=a[place], dmultiply=m, want_bias=True)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_only_the_bias():
    import paper_2502_08141_b200 as lw

    dY, _, _ = inputs(900, 264)
    dZ, _, dbias = lw.lowra_epilogue_backward(dY, want_bias=True)
    assert torch.equal(dZ, dY)
    off = (900 + 16) * F32 * dY.double().abs().sum(0)
    assert ((dbias.double() - dY.double().sum(0)).abs() <= off).all()


def test_refusals():
    import paper_2502_08141_b200 as lw

    dY, pre, mul = inputs(40, 264)
    run = lambda **kw: lw.lowra_epilogue_backward(**{**dict(dY=dY, pre=pre, activation="gelu", multiply=mul, want_bias=True), **kw})
    run()
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")
    for change, says in ((dict(activation="swish"), "activation"), (dict(dY=dY.float()), "bfloat16"), (dict(dY=dY.flatten()), "dY"), (dict(pre=pre[:-1]), "pre"),
                         (dict(pre=pre.cpu()), "CUDA"), (dict(multiply=mul[:, ::2]), "contiguous|multiply"), (dict(dZ=new(41, 264)), "dZ"), (dict(dmultiply=new(40, 264, dtype=torch.float32)), "bfloat16"),
                         (dict(dbias=new(264)), "float32"), (dict(dbias=new(256, dtype=torch.float32)), "dbias"), (dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8)), "CUDA")):
        with pytest.raises(ValueError, match=says):
            run(**change)
    one = new(40, 264)
    for change, code in ((dict(pre=None), lw.LOWRA_ERR_NULL), (dict(pre=None, activation="none"), lw.LOWRA_ERR_NULL), (dict(dZ=one, dmultiply=one), lw.LOWRA_ERR_SHAPE),
                         (dict(dY=new(40, 260), pre=new(40, 260), multiply=None), lw.LOWRA_ERR_SHAPE), (dict(dZ=new(40 * 264 + 4)[4:].view(40, 264)), lw.LOWRA_ERR_ALIGN),
                         (dict(workspace=torch.empty(128, dtype=torch.uint8, device="cuda")), lw.LOWRA_ERR_WORKSPACE)):
        with pytest.raises(lw.LowraError) as e:
            run(**change)
        assert e.value.code == code, change.keys()
