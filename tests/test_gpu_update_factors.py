"""Momentum and orthogonalised updates of the low-rank factors (lowra_update_factors) against the definition in 64 bits: every rank, both orientations, lengths down to 8, gradients of
both types, with and without momentum, master and update; in place; factors of low rank, of zeros, of very small and very large values, with a NaN; many factors; refusals."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF32 = torch.finfo(torch.float32).eps / 2      # 2^-24
COEFFICIENTS = (3.4445, -4.775, 2.0315)


def make(shapes, r, grad=torch.bfloat16, seed=1, size=1e-3, fall=5.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    members = []
    for rows, cols in shapes:
        L, tall = (rows, True) if rows != r else (cols, False)
        spread = torch.exp(-torch.arange(r, device="cuda") * (fall / r))
        body = lambda scale: ((draw(L, r) * spread) @ (draw(r, r) / math.sqrt(r)) * scale)
        turn = lambda t: (t if tall else t.t()).contiguous()
        members.append(dict(grad=turn(body(size)).to(grad), momentum=turn(body(10 * size)), master=turn(draw(L, r) * 0.01), scale=1.0 + 0.25 * len(members)))
    return members


def definition(m, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    g = m["grad"].double()
    new = None
    u, u_off = g, torch.zeros_like(g)
    if m.get("momentum") is not None:
        old = m["momentum"].double()
        new = momentum * old + g
        u = g + momentum * new if nesterov else new
        u_off = 4 * HALF32 * (old.abs() + 2 * g.abs())              # three roundings, and that of `momentum`
    side = min(u.shape)
    x = u if u.shape[0] == side else u.t()
    norm = torch.linalg.norm(x) + eps
    x = x / norm
    q = torch.eye(side, dtype=torch.float64, device=x.device)
    for _ in range(steps):
        s = x @ x.t()
        p = coefficients[0] * torch.eye(side, dtype=torch.float64, device=x.device) + coefficients[1] * s + coefficients[2] * s @ s
        x, q = p @ x, p @ q
    x = x if u.shape[0] == side else x.t()
    return new, u, u_off, x, q, norm


def bounds(m, **step):
    """-> momentum, update and weights with how far they may be off.  u Q is a sum of r products in fp32 of u (whose roundings the iteration lifts by at most a^steps) and
    Q / |u| (rounded once)."""
    lr, wd, steps, a = step.get("lr", 0.02), step.get("weight_decay", 0.0), step.get("steps", 5), step.get("coefficients", COEFFICIENTS)[0]
    new, u, u_off, x, q, norm = definition(m, **step)
    side = q.shape[0]
    product = (q.abs() @ u.abs() if u.shape[0] == side else u.abs() @ q.abs()) / norm
    lifted = abs(a) ** steps * torch.linalg.norm(u_off) / norm      # in the Frobenius norm; an element cannot be off by more
    off = lifted + (max(side, 128) + 4) * HALF32 * product + 1e-12
    out = dict(update=(x, off))
    if new is not None:
        out["momentum"] = (new, 3 * HALF32 * (m["momentum"].double().abs() + m["grad"].double().abs()) + 1e-42)
    if m.get("master") is not None:
        w = m["master"].double()
        rate = lr * m.get("scale", 1.0)
        out["master"] = (w * (1 - lr * wd) - rate * x, rate * off + 4 * HALF32 * (w.abs() + rate * x.abs()))
    return out


def check(members, r, step=None, names=("momentum", "master", "update")):
    import paper_2502_08141_b200 as lw

    step = step or {}
    want = [bounds(m, **step) for m in members]
    for m in members:
        shape = m["grad"].shape
        new = lambda dtype=torch.float32: torch.full(shape, 7.0, dtype=dtype, device="cuda")
        if m.get("momentum") is not None:
            m["momentum_out"] = new()
        if m.get("master") is not None:
            m["master_out"], m["weight"] = new(), new(torch.bfloat16)
        m["update"] = new()
    lw.lowra_update_factors(members, **{"lr": 0.02, **step}, rank=r)
    for i, (m, w) in enumerate(zip(members, want)):
        for name, (ref, off) in w.items():
            got = m["update"] if name == "update" else m[name + "_out"]
            excess = ((got.double() - ref).abs() / off).max().item()
            assert excess <= 1.0, (i, name, tuple(m["grad"].shape), excess)
        if "weight" in m:
            assert torch.equal(m["weight"], m["master_out"].bfloat16())


@pytest.mark.parametrize("r", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_every_rank(r, grad):
    shapes = [(8, r), (r, 8), (r, r), (1000, r), (r, 1000), (2056, r), (r, 4104), (r, 40), (24, r)]
    check(make(shapes, r, grad), r)
    check(make(shapes[3:6], r, grad, seed=2), r, dict(nesterov=False, weight_decay=0.1, lr=0.05))


@pytest.mark.parametrize("r,length", [(16, 13824), (64, 11008), (128, 13824)])
def test_long_factors(r, length):
    check(make([(length, r), (r, length)], r), r)


@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("r,longest", [(16, 8192), (32, 2048)])
def test_both_sides_of_one_launch(r, longest, grad):
    """Short factors of small rank go through one kernel: its longest, the next length, its most factors, one more, and lengths that leave CTAs of a cluster without rows."""
    check(make([(longest, r), (r, longest)], r, grad), r)
    check(make([(longest + 8, r), (r, longest + 8)], r, grad), r)
    shapes = [(8 * (1 + 5 * i), r) if i % 2 else (r, 8 * (1 + 9 * i)) for i in range(15)]
    check(make(shapes[:14], r, grad), r)
    check(make(shapes, r, grad), r)
    members = make([(264, r), (r, 520), (r, 72)], r, grad)
    members[0]["momentum"] = members[2]["momentum"] = None
    check(members, r, dict(nesterov=False, steps=3))


@pytest.mark.parametrize("r", [16, 32])
def test_one_launch_in_a_graph_and_in_place(r):
    import paper_2502_08141_b200 as lw

    start = make([(520, r), (r, 1032), (8, r)], r)
    copy = lambda: [{k: v.clone() if torch.is_tensor(v) else v for k, v in m.items()} for m in start]
    eager, replayed = copy(), copy()
    lw.lowra_update_factors(replayed, 0.02, rank=r)          # loads the kernel
    for m, s in zip(replayed, start):
        for k, v in s.items():
            if torch.is_tensor(v):
                m[k].copy_(v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lw.lowra_update_factors(replayed, 0.02, rank=r)
    for _ in range(3):
        graph.replay()
        lw.lowra_update_factors(eager, 0.02, rank=r)
    torch.cuda.synchronize()
    for a, b in zip(eager, replayed):
        for k, v in a.items():
            if torch.is_tensor(v):
                assert torch.equal(v, b[k]), k


@pytest.mark.parametrize("steps,coefficients", [(1, COEFFICIENTS), (2, COEFFICIENTS), (3, (1.5, -0.5, 0.0)), (9, (1.875, -1.25, 0.375))])
def test_steps_and_coefficients(steps, coefficients):
    check(make([(520, 48), (48, 264)], 48, fall=2.0), 48, dict(steps=steps, coefficients=coefficients))
    check(make([(520, 128), (128, 264)], 128, fall=2.0), 128, dict(steps=steps, coefficients=coefficients))


@pytest.mark.parametrize("r", [16, 64, 128])
def test_without_momentum_and_without_weights(r):
    members = make([(264, r), (r, 520), (96, r), (r, 96)], r)
    members[0]["momentum"] = members[1]["momentum"] = None
    members[1]["master"] = members[2]["master"] = None
    check([m for m in members], r)


@pytest.mark.parametrize("r", [32, 64, 112])
def test_the_result_is_near_orthogonal(r):
    import paper_2502_08141_b200 as lw

    members = make([(2048, r), (r, 1032)], r, fall=3.0)
    for m in members:
        m["update"] = torch.empty_like(m["momentum"])
    lw.lowra_update_factors(members, 0.02, rank=r)
    for m in members:
        values = torch.linalg.svdvals(m["update"].double())
        assert values.max().item() < 1.3 and values.min().item() > 0.4       # (u's are within exp(-3) or so of each other, which five steps lift to this)


@pytest.mark.parametrize("r", [16, 64, 128])
@pytest.mark.parametrize("size", [1e-25, 1e-12, 1e10])
def test_very_small_and_very_large(r, size):
    members = make([(520, r), (r, 264)], r, torch.float32, size=size)
    check(members, r, dict(eps=1e-40))


@pytest.mark.parametrize("r", [16, 64, 128])
def test_low_rank_zeros_and_no_numbers(r):
    import paper_2502_08141_b200 as lw

    gen = torch.Generator(device="cuda").manual_seed(3)
    low = torch.randn(1000, 3, device="cuda", generator=gen) @ torch.randn(3, r, device="cuda", generator=gen)
    members = make([(1000, r), (1000, r), (1000, r), (r, 520)], r)
    members[0]["grad"] = low.bfloat16() * 0 + low.bfloat16()
    members[0]["momentum"] = torch.zeros_like(members[0]["momentum"])
    members[1]["grad"], members[1]["momentum"] = torch.zeros_like(members[1]["grad"]), torch.zeros_like(members[1]["momentum"])
    alone = [dict(m) for m in members]
    check(members, r)
    assert bool((members[1]["update"] == 0).all()) and torch.equal(members[1]["master_out"], members[1]["master"])
    # a NaN in one factor: that factor is NaN, the others are as before, bit for bit
    bad = [dict(m) for m in alone]
    bad[2]["grad"] = bad[2]["grad"].clone()
    bad[2]["grad"][999, r - 1] = float("nan")
    for m in bad:
        m["update"], m["momentum_out"], m["master_out"] = (torch.empty_like(m["master"]) for _ in range(3))
    lw.lowra_update_factors(bad, 0.02, rank=r)
    assert bool(bad[2]["update"].isnan().all())
    for i in (0, 1, 3):
        assert torch.equal(bad[i]["update"], members[i]["update"]) and torch.equal(bad[i]["master_out"], members[i]["master_out"])


@pytest.mark.parametrize("r,count", [(16, 64), (48, 40), (64, 64), (80, 40), (96, 20), (128, 33)])
def test_many_factors(r, count):
    shapes = [((8 * (3 + 7 * i % 50), r) if i % 2 else (r, 8 * (1 + 11 * i % 60))) for i in range(count)]
    check(make(shapes, r, torch.float32 if r == 48 else torch.bfloat16), r)


@pytest.mark.parametrize("r", [32, 128])
def test_in_place_repeated_and_on_another_stream(r):
    import paper_2502_08141_b200 as lw

    shapes = [(1032, r), (r, 2048), (r, 264)]
    a, b, c = (make(shapes, r) for _ in range(3))
    for m in a:
        m["momentum_out"], m["master_out"], m["weight"] = torch.empty_like(m["momentum"]), torch.empty_like(m["master"]), torch.empty_like(m["grad"])
    lw.lowra_update_factors(a, 0.02, weight_decay=0.1, rank=r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for members, stream in ((b, None), (c, side)):
        lw.lowra_update_factors(members, 0.02, weight_decay=0.1, stream=stream)
    torch.cuda.synchronize()
    for members in (b, c):
        for m, want in zip(members, a):
            assert torch.equal(m["momentum"], want["momentum_out"]) and torch.equal(m["master"], want["master_out"])


def test_captured_and_replayed():
    import paper_2502_08141_b200 as lw

    r, shapes = 64, [(1032, 64), (64, 2048)]
    a, b = make(shapes, r), make(shapes, r)
    size = lw.lowra_update_workspace_bytes(shapes, r)
    workspaces = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    lw.lowra_update_factors(make(shapes, r, seed=9), 0.02, workspace=workspaces[0])      # (launch configuration is looked up once, outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lw.lowra_update_factors(a, 0.02, workspace=workspaces[0])
    for _ in range(3):
        graph.replay()
        lw.lowra_update_factors(b, 0.02, workspace=workspaces[1])
    for x, y in zip(a, b):
        assert torch.equal(x["momentum"], y["momentum"]) and torch.equal(x["master"], y["master"])


def test_refusals():
    import paper_2502_08141_b200 as lw

    base = make([(264, 32)], 32)[0]
    base["update"] = torch.empty_like(base["master"])
    run = lambda step=None, **change: lw.lowra_update_factors([{**base, **change}], **{"lr": 0.02, **(step or {})})
    new = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
    for change, says in ((dict(grad=new(264, 32, dtype=torch.float16)), "grad"), (dict(grad=new(264 * 32)), "matrix"), (dict(momentum=new(264, 31)), "momentum"),
                         (dict(momentum=new(264, 32, dtype=torch.bfloat16)), "float32"), (dict(master=torch.zeros(264, 32)), "CUDA"), (dict(weight=new(264, 32)), "bfloat16"),
                         (dict(update=new(264, 64)[:, ::2]), "contiguous"), (dict(master_out=new(256, 32)), "master")):
        with pytest.raises(ValueError, match=says):
            run(**change)
    for wrong in ((3.4, -4.7), [1.0, 2.0, 3.0, 4.0]):
        with pytest.raises(ValueError, match="three"):
            run(dict(coefficients=wrong))
    with pytest.raises(ValueError, match="no members"):
        lw.lowra_update_factors([], 0.02)
    with pytest.raises(ValueError, match="common"):
        lw.lowra_update_factors(make([(264, 32)], 32) + make([(264 + 8, 16)], 16), 0.02)
    odd = lambda t: torch.cat([torch.zeros(1, dtype=t.dtype, device="cuda"), t.flatten()])[1:].view(t.shape)
    for step, change, code in ((None, dict(momentum=None, master=None, update=None), lw.LOWRA_ERR_NULL), (None, dict(master=None, weight=new(264, 32, dtype=torch.bfloat16)), lw.LOWRA_ERR_NULL),
                               (dict(steps=0), {}, lw.LOWRA_ERR_SHAPE), (dict(steps=33), {}, lw.LOWRA_ERR_SHAPE), (dict(rank=264), {}, lw.LOWRA_ERR_SHAPE),
                               (None, dict(master=odd(base["master"])), lw.LOWRA_ERR_ALIGN),
                               (dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), {}, lw.LOWRA_ERR_WORKSPACE)):
        with pytest.raises(lw.LowraError) as e:
            run(step, **change)
        assert e.value.code == code, (step, change.keys())
    with pytest.raises(lw.LowraError):
        lw.lowra_update_factors(make([(260, 32)], 32), 0.02, rank=32)
    with pytest.raises(lw.LowraError):
        lw.lowra_update_factors(make([(16, 16)] * 65, 16), 0.02)
