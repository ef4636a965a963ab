"""The step of adaptive moments: bit for bit the formula in fp32, operation by operation, where states are concerned; against fp64 within counted roundings; tails, places, captured steps."""
import math

import pytest
import torch

import paper_2502_08141_b200 as lw

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn
BLOCK = lw.LOWRA_ADAMW_BLOCK


def blocks_of(n):
    return (n + BLOCK - 1) // BLOCK


def rows(t):
    return torch.nn.functional.pad(t.flatten(), (0, -t.numel() % BLOCK)).view(-1, BLOCK)


def encode(t, root):
    """fp32 values -> e4m3 codes and scales, every operation rounded to fp32 by itself."""
    x = rows(t)
    scale = x.abs().amax(1) * torch.tensor(1 / 448, dtype=torch.float32, device="cuda")
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    x = x * torch.where(scale > 0, 1 / scale, torch.zeros_like(scale))[:, None]
    if root:
        x = torch.where(x > 0, x.clamp_min(2.0 ** -9), x)
    return x.clamp(-448, 448).flatten()[:t.numel()].view(t.shape).to(E4M3), scale


def decode(codes, scale):
    return (rows(codes.float()) * scale[:, None]).flatten()[:codes.numel()].view(codes.shape)


def make(shapes, eight, grad=torch.bfloat16, weight=True, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 11)
    r = lambda s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    members = []
    for s in shapes:
        size = torch.exp(2 * r(s)) * 1e-3
        m = dict(grad=(r(s) * size).to(grad), master=r(s), m=r(s) * size * 0.3, v=(r(s) * size) ** 2)
        if eight:
            m["m"], m["m_scale"] = encode(m["m"], False)
            m["v"], m["v_scale"] = encode(torch.sqrt(m["v"]), True)
        if weight:
            m["weight"] = torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        members.append(m)
    return members


def copy(members):
    return [{k: t.clone() for k, t in m.items()} for m in members]


def states32(w, betas, factor=None):
    """m', v' and v's root as fp32 operations one by one."""
    g = w["grad"].float()
    if factor is not None:
        g = g * factor
    f = lambda x: torch.tensor(x, dtype=torch.float32, device="cuda")  # noqa: E731
    m, v = w["m"], w["v"]
    if m.dtype == E4M3:
        m, root = decode(m, w["m_scale"]), decode(v, w["v_scale"])
        v = root * root
    m = f(betas[0]) * m + f(1 - betas[0]) * g
    v = f(betas[1]) * v + (f(1 - betas[1]) * g) * g
    return m, v, torch.sqrt(v)


def check(before, after, lr, betas, eps, wd, t, factor=None):
    for w, a in zip(before, after):
        m, v, root = states32(w, betas, factor)
        if w["m"].dtype == E4M3:
            for got, values, is_root in (("m", m, False), ("v", root, True)):
                codes, scale = encode(values, is_root)
                assert torch.equal(a[got].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(a[got + "_scale"], scale)
                # and what the codes stand for: half a step of e4m3 (2^-4 relative, 2^-10 of a scale below its normal numbers), two roundings of the value over the scale;
                # a root kept off zero is up to a step, 2^-9, too large; a block with a scale under 2^-126 is zero, its values under 448 * 2^-126
                off = (decode(a[got], a[got + "_scale"]).double() - values.double()).abs()
                least = rows(torch.ones_like(values)) * scale[:, None] * 2.0 ** (-9 if is_root else -10)
                least = least.flatten()[:values.numel()].view(values.shape).double()
                assert (off <= torch.maximum(2.0 ** -4 * values.double().abs(), least) * (1 + 8 * U) + 448 * 2.0 ** -126).all()
                assert not is_root or ((a[got].float() > 0) == ((values > 0) & (least > 0))).all()
        else:
            assert torch.equal(a["m"], m) and torch.equal(a["v"], v)
        # the weights: from the states in fp64, whose roundings above are four each; a quotient good to 2^-22, its factors and sums to a few u
        b = [float(x) for x in betas]
        step = lr / (1 - b[0] ** t) * m.double() / (v.double().sqrt() / math.sqrt(1 - b[1] ** t) + eps)
        want = w["master"].double() * (1 - lr * wd) - step
        tol = 3 * U * w["master"].double().abs() + 16 * U * step.abs() + U * want.abs()
        assert ((a["master"].double() - want).abs() <= tol).all()
        if "weight" in a:
            assert torch.equal(a["weight"], a["master"].bfloat16())


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shapes", [[(1,)], [(7,), (8,), (9,)], [(255,), (256,), (257,), (3, 85)], [(1024, 16), (16, 4096)], [(77, 131)] * 5, [(64, 11008), (1, 1), (4096, 64)]])
def test_step(shapes, grad, eight):
    members = make(shapes, eight, grad)
    before = copy(members)
    assert lw.lowra_adamw(members, 1e-3, step=5, weight_decay=0.1) is members
    check(before, members, 1e-3, (0.9, 0.999), 1e-8, 0.1, 5)
    assert all(torch.equal(m["grad"], b["grad"]) for m, b in zip(members, before))


@pytest.mark.parametrize("eight", [False, True])
def test_many_steps_from_zero(eight):
    """States that begin as zeros, and options; a gradient factor on the device; blocks without a gradient stay as they are but for the decay."""
    s = (300, 24)
    members = make([s, (1000,)], eight, weight=False)
    for m in members:
        for k in ("m", "v", "m_scale", "v_scale"):
            if k in m:
                m[k] = torch.zeros_like(m[k].float()).to(m[k].dtype)
        m["grad"].view(-1)[:512] = 0
    factor = torch.full((1,), 0.25, device="cuda")
    for t in range(1, 6):
        before = copy(members)
        lw.lowra_adamw(members, 0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.0, step=t, grad_scale=factor)
        check(before, members, 0.01, (0.8, 0.95), 1e-6, 0.0, t, 0.25)
        assert all(torch.equal(m["master"].view(-1)[:512], b["master"].view(-1)[:512]) for m, b in zip(members, before))
        for m in members:
            m["grad"].mul_(-0.7)


@pytest.mark.parametrize("eight", [False, True])
def test_many_factors_and_outputs_of_their_own(eight):
    """More factors than a launch describes, of all sizes; outputs beside the inputs; memory around the arrays stays."""
    sizes = [1 + (i * 37) % 700 for i in range(500)]
    members = make([(n,) for n in sizes], eight, seed=1)
    before = copy(members)
    names = ("master", "m", "v") + (("m_scale", "v_scale") if eight else ())
    pads = []
    for m in members:
        for k in names:
            n = m[k].numel()
            big = torch.full((n + 64,), 5.0, device="cuda").to(m[k].dtype)
            pads.append((big, n))
            m[k + "_out"] = big[16:16 + n] if m[k].dtype == torch.float32 else big[32:32 + n] if m[k].dtype == E4M3 else None
    lw.lowra_adamw(members, 1e-2, step=3)
    check(before, [{k: m.get(k + "_out", m[k]) for k in m if not k.endswith("_out")} for m in members], 1e-2, (0.9, 0.999), 1e-8, 0.01, 3)
    for m, b in zip(members, before):
        assert all(torch.equal(m[k].float(), b[k].float()) for k in names)
    for big, n in pads:
        start = 16 if big.dtype == torch.float32 else 32
        assert (big[:start].float() == 5).all() and (big[start + n:].float() == 5).all()


@pytest.mark.parametrize("eight", [False, True])
def test_bad_gradients(eight):
    """A NaN or an infinity stays with its weight (and, in 8 bits, with the block's states); nothing else is touched."""
    members = make([(1000,)], eight)
    members[0]["grad"][300] = float("nan")
    members[0]["grad"][700] = float("inf")
    clean = copy(members)
    clean[0]["grad"][[300, 700]] = 0
    lw.lowra_adamw(members, 1e-3, step=2)
    lw.lowra_adamw(clean, 1e-3, step=2)
    a, b = members[0], clean[0]
    hit = torch.zeros(1000, dtype=torch.bool, device="cuda")
    hit[[300, 700]] = True
    assert a["master"][hit].isnan().all() and torch.equal(a["master"][~hit], b["master"][~hit])
    if eight:
        m = decode(a["m"], a["m_scale"])
        assert m[256:512].isnan().all() and m[512:768].isnan().all() and torch.equal(m[:256], decode(b["m"], b["m_scale"])[:256])
        assert a["m_scale"].isfinite().tolist() == [True, False, False, True]
    else:
        assert torch.equal(a["m"][~hit], b["m"][~hit])


def test_tiny_blocks_in_8_bits():
    """Magnitudes whose scale has no reciprocal in fp32: the block is zero, not NaN."""
    m = make([(512,)], True)[0]
    m["m"], m["v"], m["m_scale"], m["v_scale"] = torch.zeros(512, device="cuda").to(E4M3), torch.zeros(512, device="cuda").to(E4M3), torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    m["grad"] = torch.full((512,), 1e-36, device="cuda").bfloat16()
    before = copy([m])
    lw.lowra_adamw([m], 1e-3, step=1)
    check(before, [m], 1e-3, (0.9, 0.999), 1e-8, 0.01, 1)
    assert m["m_scale"].eq(0).all() and m["m"].float().eq(0).all() and m["master"].isfinite().all()


@pytest.mark.parametrize("eight", [False, True])
def test_captured_step(eight):
    """A captured step whose count, rate and factor are on the device, replayed while they change, against calls with the same numbers from the host."""
    a = make([(100, 16), (16, 333)], eight, seed=2)
    b = copy(a)
    step, lr, factor = torch.ones(1, dtype=torch.int32, device="cuda"), torch.full((1,), 1e-3, device="cuda"), torch.full((1,), 0.5, device="cuda")
    warm = copy(a)
    lw.lowra_adamw(warm, lr, step=step, grad_scale=factor)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lw.lowra_adamw(a, lr, step=step, grad_scale=factor)
        step += 1
    for t in range(1, 5):
        rate = float(torch.tensor(1e-3 / t))
        lr.fill_(rate)
        graph.replay()
        before = copy(b)
        lw.lowra_adamw(b, rate, step=t, grad_scale=factor)
        torch.cuda.synchronize()
        for x, y, w in zip(a, b, before):
            assert all(torch.equal(x[k].float(), y[k].float()) for k in ("m", "v"))
            assert ((x["master"] - y["master"]).abs() <= 2.0 ** -20 * ((y["master"] - w["master"]).abs() + w["master"].abs())).all()
            x["master"].copy_(y["master"])
    assert int(step) == 5
    only_lr, only_step = copy(b), copy(b)
    lw.lowra_adamw(only_lr, lr, step=7)
    step.fill_(7)
    lw.lowra_adamw(only_step, float(lr), step=step)
    lw.lowra_adamw(b, float(lr), step=7)
    for x, y, z in zip(only_lr, only_step, b):
        assert torch.allclose(x["master"], z["master"], rtol=2.0 ** -21, atol=1e-9) and torch.allclose(y["master"], z["master"], rtol=2.0 ** -21, atol=1e-9)


def test_other_stream():
    a = make([(500, 64)], True, seed=3)
    b = copy(a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lw.lowra_adamw(a, 1e-3, step=2, stream=side)
    torch.cuda.synchronize()
    lw.lowra_adamw(b, 1e-3, step=2)
    assert all(torch.equal(a[0][k].float(), b[0][k].float()) for k in a[0])


def test_refusals():
    good = make([(64, 16)], True)[0]
    wide = make([(64, 16)], False)[0]
    with pytest.raises(ValueError, match="no members"):
        lw.lowra_adamw([], 1e-3)
    for bad in (dict(grad=good["grad"].half()), dict(m=good["m"].half()), dict(v=wide["v"]), dict(master=good["grad"]), dict(master=good["master"][:32]), dict(m_scale=good["m_scale"][:3]),
                dict(v_scale=None), dict(weight=good["master"]), dict(m_out=wide["m"]), dict(master=good["master"].t()), dict(master=good["master"].cpu()),
                dict(master_out=good["master"][:1])):
        with pytest.raises(ValueError):
            lw.lowra_adamw([{**good, **bad}], 1e-3)
    with pytest.raises(ValueError, match="scales"):
        lw.lowra_adamw([{**wide, "m_scale": good["m_scale"]}], 1e-3)
    with pytest.raises(ValueError):
        lw.lowra_adamw([good, wide], 1e-3)
    for options in (dict(step=0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -1.0)), dict(eps=-1.0)):
        with pytest.raises(lw.LowraError):
            lw.lowra_adamw([good], 1e-3, **options)
    for options in (dict(step=torch.ones(1, device="cuda")), dict(step=torch.ones(2, dtype=torch.int32, device="cuda")), dict(grad_scale=torch.ones(1)),
                    dict(lr=torch.ones(1, dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            lw.lowra_adamw([good], **{"lr": 1e-3, **options})
    with pytest.raises(lw.LowraError):
        lw.lowra_adamw([good, good], 1e-3)                                       # one factor twice
    with pytest.raises(lw.LowraError):
        lw.lowra_adamw([{**wide, "m_out": wide["v"]}], 1e-3)
