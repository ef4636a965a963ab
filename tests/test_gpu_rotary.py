"""Rotary positions against the formula in fp64: 2^-8 relative for the rounding to bf16 and, of the pair's magnitudes, 8 * 2^-24 for the angle (rounded to fp32: pi * 2^-25 twice), its
cosine and sine (two steps of 2^-24), and the products."""
import numpy as np
import pytest
import torch

import paper_2502_08141_b200 as lw

pytestmark = pytest.mark.gpu


def reference(x, positions, dim, base, interleaved, inverse, scale, factor=1.0):
    x = x.double()
    f = torch.tensor(base, dtype=torch.float64) ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim) / factor
    t = positions.double()[:, None, None] * f.cuda()
    c, s = torch.cos(t) * scale, torch.sin(t) * (-scale if inverse else scale)
    i = torch.arange(dim // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
    a, b = x[..., first], x[..., second]
    y, wide = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    wide[..., first] = wide[..., second] = (a.abs() + b.abs()) * scale
    return y, wide


def close(got, want):
    y, wide = want
    return ((got.double() - y).abs() <= 2.0 ** -8 * y.abs() + 8 * 2.0 ** -24 * wide).all()


def table(dim, base=10000.0, kind="none", **options):
    turns, scale = lw.lowra_rotary_turns(dim, base, kind, **options)
    return torch.from_numpy(turns.view(np.int64)).cuda(), scale


def heads(M, H, D, seed=0):
    return torch.randn((M, H, D), generator=torch.Generator(device="cuda").manual_seed(seed + M * H + D), device="cuda").bfloat16()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("M, q, k, D, dim", [(1, 1, 1, 16, 16), (1, 32, 8, 128, 128), (3, 5, 1, 80, 32), (16, 32, 8, 128, 64), (777, 12, 12, 64, 64), (2500, 40, 40, 128, 128),
                                            (130, 3, 2, 1032, 1024), (600, 64, 1, 256, 128), (9000, 2, 1, 96, 48), (5, 7, 0, 64, 16)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(M, q, k, D, dim, interleaved, inverse):
    turns, scale = table(dim, 5e5, "linear", factor=2.0)
    positions = torch.randint(0, 200000, (M,), device="cuda", dtype=torch.int32)
    x, y = heads(M, q, D), heads(M, k, D, 1) if k else None
    got = lw.lowra_rotary(x, positions, turns, k=y, interleaved=interleaved, inverse=inverse, scale=1.25 * scale)
    for a, b in zip(got if k else (got,), (x, y)):
        assert a.is_contiguous() and close(a, reference(b, positions, dim, 5e5, interleaved, inverse, 1.25, 2.0))
        assert torch.equal(a[..., dim:], b[..., dim:])


def test_far_and_negative_positions():
    """Angles of every 32-bit position: the product with the frequency wraps by whole turns."""
    turns, _ = table(128)
    positions = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 7, 123456789, -987654321], dtype=torch.int32, device="cuda")
    x = heads(8, 4, 128)
    y, wide = reference(x, positions, 128, 10000.0, False, False, 1.0)
    got = lw.lowra_rotary(x, positions, turns)
    # the reference's own angles, in fp64: 2^31 * 2^-52
    assert ((got.double() - y).abs() <= 2.0 ** -8 * y.abs() + (8 * 2.0 ** -24 + 2.0 ** -20) * wide).all()
    assert torch.equal(got[0], x[0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_in_place_and_rows_beside(interleaved):
    """Queries and keys as slices of one projection, in place: the values' part and what lies between stays; heads before tokens; one head or token of odd strides."""
    M, D = 50, 64
    turns, _ = table(32)
    positions = torch.arange(M, device="cuda", dtype=torch.int32) + 1000
    qkv = heads(M, 12, D)
    before = qkv.clone()
    q, k = qkv[:, :6], qkv[:, 6:9]
    want = lw.lowra_rotary(before[:, :6].contiguous(), positions, turns, k=before[:, 6:9].contiguous(), interleaved=interleaved)
    got = lw.lowra_rotary(q, positions, turns, k=k, interleaved=interleaved, out=q, k_out=k)
    assert got[0] is q and got[1] is k and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, 9:], before[:, 9:])
    across = before[:, :6].transpose(0, 1).contiguous().transpose(0, 1)      # [tokens, heads, D] over memory [heads, tokens, D]
    assert torch.equal(lw.lowra_rotary(across, positions, turns, interleaved=interleaved), want[0])
    out = torch.zeros((6, M, D), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    lw.lowra_rotary(across, positions, turns, interleaved=interleaved, out=out)
    assert torch.equal(out, want[0])
    assert torch.equal(lw.lowra_rotary(before[:, 2:3], positions, turns, interleaved=interleaved), want[0][:, 2:3])
    assert torch.equal(lw.lowra_rotary(before[7:8, :6], positions[7:8], turns, interleaved=interleaved), want[0][7:8])
    assert torch.equal(lw.lowra_rotary(before[:1, :1].expand(M, 6, D), positions, turns, interleaved=interleaved),
                       lw.lowra_rotary(before[:1, :1].expand(M, 6, D).contiguous(), positions, turns, interleaved=interleaved))
    wide = torch.full((M, 20, D), 3.0, dtype=torch.bfloat16, device="cuda")
    lw.lowra_rotary(before[:, :6], positions, turns, interleaved=interleaved, out=wide[:, 4:10])
    assert torch.equal(wide[:, 4:10], want[0]) and (wide[:, :4] == 3).all() and (wide[:, 10:] == 3).all()


def test_gradient_turns_back():
    """The inverse is the transpose: <turn(x), y> = <x, inverse(y)>, and turning back gives x to the two roundings."""
    turns, scale = table(64, kind="yarn", factor=4.0)
    positions = torch.randint(0, 9000, (100,), device="cuda", dtype=torch.int32)
    x, y = heads(100, 8, 96), heads(100, 8, 96, 3)
    a = lw.lowra_rotary(x, positions, turns, scale=scale)
    b = lw.lowra_rotary(y, positions, turns, scale=scale, inverse=True)
    left, right = (a.double() * y.double()), (x.double() * b.double())
    assert (left.sum() - right.sum()).abs() <= 2.0 ** -8 * 1.01 * (left.abs().sum() + right.abs().sum())
    back = lw.lowra_rotary(lw.lowra_rotary(x, positions, turns), positions, turns, inverse=True)
    size = torch.maximum(x.double().abs(), x.double().norm(dim=-1, keepdim=True))
    assert ((back.double() - x.double()).abs() <= 2.0 ** -7 * size).all()


def test_graph_with_positions_that_change():
    turns, _ = table(128)
    positions = torch.arange(4, device="cuda", dtype=torch.int32)
    x, out = heads(4, 32, 128), torch.empty((4, 32, 128), dtype=torch.bfloat16, device="cuda")
    lw.lowra_rotary(x, positions, turns, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lw.lowra_rotary(x, positions, turns, out=out)
    positions += 5000
    graph.replay()
    torch.cuda.synchronize()
    assert close(out, reference(x, positions, 128, 10000.0, False, False, 1.0))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = torch.empty_like(out)
    lw.lowra_rotary(x, positions, turns, out=other, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, other)


def test_unsigned_table():
    turns, _ = table(64)
    x, positions = heads(8, 4, 64), torch.arange(8, device="cuda", dtype=torch.int32)
    assert torch.equal(lw.lowra_rotary(x, positions, turns.view(torch.uint64)), lw.lowra_rotary(x, positions, turns))


def test_refusals():
    turns, _ = table(64)
    x, positions = heads(8, 4, 64), torch.arange(8, device="cuda", dtype=torch.int32)
    for bad in (dict(q=x.float()), dict(q=x[0]), dict(q=x.transpose(1, 2)), dict(q=x.cpu()), dict(positions=positions.long()), dict(positions=positions[:7]), dict(turns=turns.int()),
                dict(turns=turns.double()), dict(turns=turns.view(torch.complex64)), dict(turns=turns.cpu()), dict(k=x[:, :, :32]), dict(k=x[:7]), dict(out=x[:, :3]), dict(k_out=x)):
        with pytest.raises(ValueError):
            lw.lowra_rotary(**{**dict(q=x, positions=positions, turns=turns), **bad})
    both = heads(8, 5, 64)
    for bad in (dict(out=both[:, 1:]), dict(q=both[:, :4, 8:40], turns=turns), dict(q=x[:, :1].expand(8, 4, 64), out=x[:, :1].expand(8, 4, 64)), dict(turns=turns[:30]),
                dict(q=x[:0], positions=positions[:0]), dict(k=both[:, :4], k_out=x, out=x)):
        with pytest.raises(lw.LowraError):
            lw.lowra_rotary(**{**dict(q=both[:, :4], positions=positions, turns=turns), **bad})
