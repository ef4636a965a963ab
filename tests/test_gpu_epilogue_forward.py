"""Products with bias, activation, second factor and residual (lowra_lora_forward_epilogue, its batch and adapters forms) against the formula in 64 bits: every path
that forms a product (one launch, slices, units, shared tiles, cut tiles, whole tiles), every option, in place, and what lies behind the last row."""
import itertools

import pytest
import torch

from epilogue_reference import Weight, forward

pytestmark = pytest.mark.gpu

MIX, FEW = {1: 0.3, 2: 0.5, 4: 0.2}, {1: 0.5, 2: 0.5}
# N, K, M, r, mix, what the call has to take
SHAPES = [
    (264, 384, 1, 16, MIX, "few"),            # a small weight, one launch
    (512, 512, 16, 16, FEW, "few"),
    (1032, 1024, 1, 64, MIX, "few"),          # one token, slices of a cluster
    (2048, 2048, 33, 48, MIX, "few"),         # more tokens than a unit
    (4104, 1664, 7, 80, {4: 1.0}, "few"),
    (640, 1152, 130, 32, MIX, "tiles"),       # few whole tiles
    (1800, 2304, 65, 48, FEW, "shared"),      # few tiles, each shared by clusters
    (1032, 4096, 600, 64, MIX, "shared"),
    (1800, 2304, 777, 48, FEW, "tiles"),      # channels that end inside 16 columns
    (1032, 256, 300, 128, MIX, "tiles"),
    (1800, 2304, 4300, 80, MIX, "tiles"),     # tiles cut between clusters
    (8, 128, 65, 16, {2: 1.0}, "any"),        # the smallest weight
]
OPTIONS = [
    dict(),
    dict(bias=torch.float32),
    dict(bias=torch.bfloat16, activation="gelu", pre=True),
    dict(activation="silu", multiply=True),
    dict(bias=torch.bfloat16, residual=True),
    dict(bias=torch.float32, activation="gelu_tanh", multiply=True, residual=True, pre=True),
    dict(activation="relu", residual=True, pre=True),
]


def arrays(w, M, bias=None, activation="none", multiply=False, residual=False, pre=False):
    new = lambda: w.draw(M, w.N).bfloat16()
    return dict(bias=None if bias is None else w.draw(w.N).to(bias), activation=activation, multiply=new() if multiply else None,
                residual=new() if residual else None), pre


def agrees(got, want, off, what):
    excess = ((got.double() - want).abs() / off).max().item()
    assert excess <= 1.0, (what, excess)


@pytest.mark.parametrize("N,K,M,r,mix,path", SHAPES)
def test_against_the_formula(N, K, M, r, mix, path):
    import paper_2502_08141_b200 as lw

    for k, options in enumerate(OPTIONS):
        w = Weight(N, K, mix, r, natural=k == 1, deal=k != 2, seed=k + 1)
        c = lw.lowra_diag_choose(w.layout, False, [M], r)
        if path != "any":
            assert (path == "few") == (c["few_tokens"] == 1) and (path != "shared" or c["w_split"] > 1), c
        X = w.draw(M, K).bfloat16()
        e, pre = arrays(w, M, **options)
        Y = torch.full((M + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
        Z = torch.full((M + 2, N), 7.0, dtype=torch.bfloat16, device="cuda") if pre else None
        ws = torch.empty(lw.lowra_workspace_bytes(w.layout, M, r), dtype=torch.uint8, device="cuda")
        lw.lowra_workspace_init(ws)
        got = lw.lowra_lora_forward_epilogue(*w.head(), X, w.A[0], w.B[0], 2.0, **e, pre=None if Z is None else Z[:M], Y=Y, workspace=ws)
        assert got is Y and lw.lowra_device_status(ws) == lw.LOWRA_OK
        y, z, y_off, z_off = forward(w.W_hat[0], X, w.A[0], w.B[0], 2.0, **e)
        agrees(Y[:M], y, y_off, (options, "Y"))
        assert bool((Y[M:] == 7.0).all())
        if pre:
            agrees(Z[:M], z, z_off, (options, "pre"))
            assert bool((Z[M:] == 7.0).all())


@pytest.mark.parametrize("N,K,M,r,mix,path", [s for s in SHAPES if s[2] in (1, 33, 65, 130, 777)])
def test_nothing_behind_is_the_product_and_places_make_no_difference(N, K, M, r, mix, path):
    import paper_2502_08141_b200 as lw

    w = Weight(N, K, mix, r)
    X = w.draw(M, K).bfloat16()
    run = lambda **kw: lw.lowra_lora_forward_epilogue(*w.head(), X, w.A[0], w.B[0], 2.0, **kw)
    assert torch.equal(run(), lw.lowra_lora_forward(*w.head(), X, w.A[0], w.B[0], 2.0))
    residual, multiply = w.draw(M, N).bfloat16(), w.draw(M, N).bfloat16()
    want = run(activation="silu", multiply=multiply, residual=residual)
    for name in ("residual", "multiply"):                      # the output in the place of an input
        own = dict(residual=residual, multiply=multiply)
        own[name] = own[name].clone()
        assert torch.equal(run(activation="silu", **own, Y=own[name]), want), name
    again = run(activation="silu", multiply=multiply, residual=residual, stream=torch.cuda.current_stream())    # the interpreted way
    assert torch.equal(again, want)
    # outputs and arrays that are 16-byte aligned only
    odd = lambda t: torch.cat([torch.zeros(8, dtype=torch.bfloat16, device="cuda"), t.flatten()])[8:].view(M, N)
    shifted, Z, Z2 = odd(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")), odd(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")), torch.empty_like(want)
    assert torch.equal(run(activation="silu", multiply=odd(multiply), residual=odd(residual), pre=Z, Y=shifted), want)
    assert torch.equal(run(activation="silu", multiply=multiply, residual=residual, pre=Z2), want) and torch.equal(Z, Z2)


@pytest.mark.parametrize("M", [3, 300])
def test_values_out_of_the_ordinary_stay_where_they_are(M):
    import paper_2502_08141_b200 as lw

    w = Weight(520, 384, MIX, 16)
    X, N = w.draw(M, 384).bfloat16(), w.N
    residual = w.draw(M, N).bfloat16()
    run = lambda **kw: lw.lowra_lora_forward_epilogue(*w.head(), X, w.A[0], w.B[0], 2.0, **kw)
    want = run(residual=residual)
    bad = residual.clone()
    bad[1, 5], bad[2, 6] = float("nan"), float("inf")
    got = run(residual=bad)
    assert bool(got[1, 5].isnan()) and bool(got[2, 6].isinf())
    got[1, 5], got[2, 6] = want[1, 5], want[2, 6]
    assert torch.equal(got, want)
    # a channel far out on either side, and one that is no number, through every activation
    bias = torch.zeros(N, device="cuda")
    bias[:4] = torch.tensor([1e4, -1e4, float("nan"), -40.0])
    for activation in ("relu", "gelu", "gelu_tanh", "silu"):
        y = run(bias=bias, activation=activation)
        assert bool((y[:, 0] > 9e3).all()) and bool((y[:, 1] == 0).all()) and bool(y[:, 2].isnan().all()) and bool((y[:, 3].abs() < 1e-9).all()), activation
        assert bool(y[:, 4:].isfinite().all())


@pytest.mark.parametrize("N,K,M,r,count,shared", [(256, 384, 300, 32, 3, True), (1800, 2304, 900, 48, 4, False), (520, 512, 9, 16, 2, True)])
def test_batch(N, K, M, r, count, shared):
    import paper_2502_08141_b200 as lw

    ws_w = [Weight(N, K, MIX, r, seed=i + 1) for i in range(count)]
    X = [ws_w[0].draw(M, K).bfloat16()] * count if shared else [w.draw(M, K).bfloat16() for w in ws_w]
    members, checks = [], []
    for i, (w, x) in enumerate(zip(ws_w, X)):
        e, pre = arrays(w, M, **OPTIONS[(i + 2) % len(OPTIONS)])
        members.append(dict(layout=w.layout, packed=w.packed, absmax=w.absmax, maps=w.maps[0], act=x, A=w.A[0], B=w.B[0],
                            out=torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda"), **e, pre=torch.empty(M, N, dtype=torch.bfloat16, device="cuda") if pre else None))
        checks.append(forward(w.W_hat[0], x, w.A[0], w.B[0], 2.0, **e))
    ws = lw.lowra_workspace_init(torch.empty(lw.lowra_batch_workspace_bytes(ws_w[0].layout, count, M, r), dtype=torch.uint8, device="cuda"))
    for _ in range(2):
        outs = lw.lowra_lora_forward_batch_epilogue(members, 2.0, ws)
    assert lw.lowra_device_status(ws) == lw.LOWRA_OK
    for i, (m, (y, z, y_off, z_off)) in enumerate(zip(members, checks)):
        agrees(outs[i], y, y_off, (i, "Y"))
        if m["pre"] is not None:
            agrees(m["pre"], z, z_off, (i, "pre"))


@pytest.mark.parametrize("N,K,r,counts", [
    (4096, 1664, 16, (17, 24, 0, 32, 1, 9)),          # units, an empty group
    (520, 384, 32, (1, 40, 0, 100, 3)),               # few tokens and tiles in one call
    (1032, 1024, 64, (5,)),
])
def test_adapters(N, K, r, counts):
    import paper_2502_08141_b200 as lw

    n, M = len(counts), sum(counts)
    w = Weight(N, K, MIX, r, n=n)
    start = list(itertools.accumulate(counts, initial=0))
    X = w.draw(M, K).bfloat16()
    ws = lw.lowra_workspace_init(torch.empty(lw.lowra_batch_workspace_bytes(w.layout, 4, M, r), dtype=torch.uint8, device="cuda"))
    for options in OPTIONS:
        e, pre = arrays(w, M, **options)
        Y = torch.full((M + 1, N), 7.0, dtype=torch.bfloat16, device="cuda")
        Z = torch.empty(M, N, dtype=torch.bfloat16, device="cuda") if pre else None
        lw.lowra_lora_forward_adapters_epilogue(w.layout, w.packed, w.absmax, w.maps, X, start, w.A, w.B, 2.0, **e, pre=Z, Y=Y, workspace=ws)
        for a in range(n):
            rows = slice(start[a], start[a + 1])
            part = {k: v[rows] if k in ("multiply", "residual") and v is not None else v for k, v in e.items()}
            if start[a] < start[a + 1]:
                y, z, y_off, z_off = forward(w.W_hat[a], X[rows], w.A[a], w.B[a], 2.0, **part)
                agrees(Y[rows], y, y_off, (options, a))
                if pre:
                    agrees(Z[rows], z, z_off, (options, a, "pre"))
        assert bool((Y[M:] == 7.0).all())


@pytest.mark.parametrize("native", [False, True])
def test_refusals(native):
    import paper_2502_08141_b200 as lw

    N, K, M, r = 264, 384, 5, 16
    w = Weight(N, K, MIX, r)
    X = w.draw(M, K).bfloat16()
    stream = None if native else torch.cuda.current_stream()
    run = lambda **kw: lw.lowra_lora_forward_epilogue(*w.head(), X, w.A[0], w.B[0], 2.0, stream=stream, **kw)
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")
    for change, says in ((dict(bias=new(N, dtype=torch.float16)), "bias"), (dict(bias=new(N - 8)), "bias"), (dict(bias=torch.zeros(N)), "CUDA"), (dict(bias=new(2 * N)[::2]), "bias"),
                         (dict(activation="tanh"), "activation"), (dict(multiply=new(M, N, dtype=torch.float32)), "bfloat16"), (dict(multiply=new(M - 1, N)), "multiply"),
                         (dict(residual=new(M, 2 * N)[:, ::2]), "contiguous"), (dict(residual=new(M + 1, N)), "residual"), (dict(pre=torch.zeros(M, N).bfloat16()), "CUDA"),
                         (dict(pre=new(M * N)), "pre"), (dict(Y=new(M - 1, N)), "elements")):
        with pytest.raises(ValueError, match=says):
            run(**change)
    one = new(M, N)
    for change, code in ((dict(pre=one, Y=one), lw.LOWRA_ERR_SHAPE), (dict(pre=one, residual=one), lw.LOWRA_ERR_SHAPE), (dict(pre=one, multiply=one), lw.LOWRA_ERR_SHAPE),
                         (dict(residual=new(M * N + 4)[4:].view(M, N)), lw.LOWRA_ERR_ALIGN), (dict(bias=new(N + 4)[4:]), lw.LOWRA_ERR_ALIGN)):
        with pytest.raises(lw.LowraError) as e:
            run(**change)
        assert e.value.code == code, change.keys()
