"""States in 8 bits that are rounded up or down by their place between two codes: one of the two about the value, with no bias; scales, weights, NaNs and zeros as without; and over thousands of steps the
kept moments follow those in fp32, which rounding to nearest does not."""
import pytest
import torch

import paper_2502_08141_b200 as lw
from test_gpu_adamw import copy, decode, encode, make, rows, states32

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
BETAS = (0.9, 0.999)


def over_scale(values, scale, root):
    """What is rounded, fp32 as the formula has it."""
    x = rows(values) * torch.where(scale > 0, 1 / scale, torch.zeros_like(scale))[:, None]
    if root:
        x = torch.where(x > 0, x.clamp_min(2.0 ** -9), x)
    return x.clamp(-448, 448).flatten()[:values.numel()].view(values.shape).double()


def distance(x):
    """Of the codes about x (the upper of a power of two)."""
    return 2.0 ** (torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)


@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shapes", [[(1,)], [(7,), (256,), (257,), (3, 85)], [(1024, 16), (16, 4096)], [(77, 131)] * 5, [(1 + 31 * i % 700,) for i in range(300)]])
def test_one_of_two_codes(shapes, grad):
    members = make(shapes, True, grad)
    nearest, before = copy(members), copy(members)
    assert lw.lowra_adamw(members, 1e-3, step=5, dither=True) is members
    lw.lowra_adamw(nearest, 1e-3, step=5)
    places, count = {"m": 0.0, "v": 0.0}, 0
    for w, a, b in zip(before, members, nearest):
        assert all(torch.equal(a[k], b[k]) for k in ("master", "weight", "m_scale", "v_scale"))
        m, _, root = states32(w, BETAS)
        for name, values, is_root in (("m", m, False), ("v", root, True)):
            x, got = over_scale(values, a[name + "_scale"], is_root), a[name].float().double()
            off = (got - x) / distance(x)
            assert (off.abs() < 1).all() and (got * x >= 0).all() and torch.equal(got[x == 0], x[x == 0])
            assert not is_root or (got[x > 0] > 0).all()
            places[name] += off.sum().item()
        count += m.numel()
    # each is off by under a distance, by nothing on average: half of one at most for its spread, six of them over the root of their number
    assert all(abs(p) <= 6 * 0.5 * count ** 0.5 for p in places.values()), (places, count)
    again = copy(before)
    lw.lowra_adamw(again, 1e-3, step=5, dither=True)
    other = copy(before)
    lw.lowra_adamw(other, 1e-3, step=6, dither=True)
    assert all(torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)) for a, b in zip(members, again) for k in ("m", "v"))
    assert count < 1000 or any(not torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)) for a, b in zip(members, other) for k in ("m", "v"))


def test_zeros_tiny_blocks_and_bad_gradients():
    members = make([(1024,)], True)
    w = members[0]
    w["grad"][:256], w["m"][:256], w["v"][:256], w["m_scale"][0], w["v_scale"][0] = 0, torch.zeros(256, device="cuda").to(E4M3), torch.zeros(256, device="cuda").to(E4M3), 0, 0
    w["grad"][300], w["grad"][700] = float("nan"), float("inf")
    near = copy(members)
    lw.lowra_adamw(members, 1e-3, step=2, dither=True)
    lw.lowra_adamw(near, 1e-3, step=2)
    a, b = members[0], near[0]
    assert (a["m"][:256].float() == 0).all() and (a["v"][:256].float() == 0).all()
    for k in ("m", "v"):
        values = decode(a[k], a[k + "_scale"])
        assert values[256:768].isnan().all() and values[768:].isfinite().all() and torch.equal(values.isnan(), decode(b[k], b[k + "_scale"]).isnan())
    assert torch.equal(a["master"].isnan(), b["master"].isnan())


@pytest.mark.parametrize("noisy", [False, True])
def test_moments_follow_over_thousands_of_steps(noisy):
    """Gradients that change size, beside one of 1 in every block that keeps its scale.  A change of the root by a share p of the distance of two codes happens once in 1 / p steps; p is some 0.006 at rest (b2 =
    0.999, distances of 6 to 12 %), which over the thousand steps that b2 remembers leaves about two codes, an eighth of the root: so every root is within a factor of two, four times that, and the mean over
    1020 elements within a tenth of it, twice that while it falls, when the steps on which it may fall are those just past where it was before."""
    n = 1024
    g = torch.Generator(device="cuda").manual_seed(3)
    zeros = lambda k=n: torch.zeros(k, device="cuda")  # noqa: E731
    eight = dict(grad=zeros(), master=zeros(), m=zeros().to(E4M3), v=zeros().to(E4M3), m_scale=zeros(4), v_scale=zeros(4))
    full = dict(grad=eight["grad"], master=zeros(), m=zeros(), v=zeros())
    small = torch.arange(n, device="cuda") % 256 != 0
    t = 0
    for size, steps in ((0.1, 3000), (0.5, 3000), (0.01, 6000), (0.1, 3000)):
        eight["grad"].copy_(torch.where(small, size, 1.0))
        for _ in range(steps):
            t += 1
            if noisy:
                eight["grad"].copy_(torch.where(small, size * torch.randn(n, generator=g, device="cuda"), 1.0))
            lw.lowra_adamw([eight], 1e-4, step=t, dither=True)
            lw.lowra_adamw([full], 1e-4, step=t)
        ratio = (decode(eight["v"], eight["v_scale"]) / full["v"].sqrt())[small]
        assert 0.5 < ratio.min() and ratio.max() < 2.0 and 0.8 < ratio.mean() < 1.1, (size, ratio.min(), ratio.mean(), ratio.max())
        if not noisy:      # m has a tenth of every gradient: within a code, 2^-3, of it
            m = decode(eight["m"], eight["m_scale"])[small]
            assert (m / full["m"][small] - 1).abs().max() <= 2.0 ** -3 * 1.01


def test_captured_step_counts_on_the_device():
    a = make([(100, 16), (16, 333)], True, seed=2)
    b = copy(a)
    step = torch.ones(1, dtype=torch.int32, device="cuda")
    lw.lowra_adamw(copy(a), 1e-3, step=step, dither=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lw.lowra_adamw(a, 1e-3, step=step, dither=True)
        step += 1
    for t in range(1, 4):
        graph.replay()
        lw.lowra_adamw(b, 1e-3, step=t, dither=True)
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            assert all(torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)) for k in ("m", "v"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lw.lowra_adamw(a, 1e-3, step=4, dither=True, stream=side)      # (the other way through the binding)
    torch.cuda.synchronize()
    lw.lowra_adamw(b, 1e-3, step=4, dither=True)
    assert all(torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)) for x, y in zip(a, b) for k in ("m", "v"))


def test_without_it_the_codes_are_the_nearest_and_states_in_fp32_refuse_it():
    members = make([(300, 24)], True)
    before = copy(members)
    lw.lowra_adamw(members, 1e-3, step=5, dither=False)
    m, _, root = states32(before[0], BETAS)
    for name, values, is_root in (("m", m, False), ("v", root, True)):
        assert torch.equal(members[0][name].view(torch.uint8), encode(values, is_root)[0].view(torch.uint8))
    wide = make([(64, 16)], False)
    for way in (dict(), dict(stream=torch.cuda.current_stream())):
        with pytest.raises(lw.LowraError):
            lw.lowra_adamw(wide, 1e-3, step=1, dither=True, **way)
