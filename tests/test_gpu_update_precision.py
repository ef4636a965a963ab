"""The update of the factors to the last bits that fp32 products leave, at every rank, in both orientations, on both sides of the one launch: with directions so weak that S or the steps in fp32 would
be outside of the bound many times over (which tests/test_update_reference_host.py shows)."""
import pytest
import torch

from update_reference import U, graded, momentum_of, update

pytestmark = pytest.mark.gpu

RANKS = [16, 32, 48, 64, 80, 96, 112, 128]


def run(members, r, **step):
    import paper_2502_08141_b200 as lw

    lw.lowra_update_factors(members, 0.02, rank=r, **step)
    return members


def agree(got, want, off, what):
    excess = ((got.double() - want).abs() / off).max().item()
    assert excess <= 1.0, (what, excess)


@pytest.mark.parametrize("r", RANKS)
@pytest.mark.parametrize("lengths", [(264, 1000, 2048), (8, 4104, 13824)])
def test_gradients_alone(r, lengths):
    turned = [(L, tall) for L in lengths for tall in (True, False)]
    us = [graded(L, r, L + r, "cuda") for L, _ in turned]
    members = [dict(grad=(u if tall else u.t()).contiguous()) for u, (_, tall) in zip(us, turned)]
    for m in members:
        m["update"] = torch.empty_like(m["grad"])
    for alone in (False, True):                                # together, and each by itself
        for m in members:
            m["update"].fill_(7.0)
        for group in ([members] if not alone else [[m] for m in members]):
            run(group, r)
        for m, (L, tall) in zip(members, turned):
            agree(m["update"], *update(m["grad"], tall), (L, tall, alone))


@pytest.mark.parametrize("r", RANKS)
@pytest.mark.parametrize("nesterov", [True, False])
def test_with_momentum_and_weights(r, nesterov):
    """Gradients of both types, far smaller than the momentum; u is that of the kernels, rounding for rounding, and the weights follow from the update that they return."""
    members = []
    for i, (L, tall) in enumerate([(520, True), (2056, False), (5120, True), (11008, False)]):
        turn = lambda t: (t if tall else t.t()).contiguous()
        m = dict(grad=turn(graded(L, r, 3 * i + r, "cuda") * 1e-2), momentum=turn(graded(L, r, i + r, "cuda")), master=turn(graded(L, r, i, "cuda") * 1e3), scale=1.0 + i)
        if i % 2 == 0:
            m["grad"] = m["grad"].bfloat16()
        for name in ("momentum_out", "master_out", "update"):
            m[name] = torch.empty_like(m["master"])
        members.append(m)
    run(members, r, nesterov=nesterov, weight_decay=0.1)
    for m in members:
        tall = m["grad"].shape[1] == r
        new, u = momentum_of(m["momentum"], m["grad"], nesterov=nesterov)
        agree(m["momentum_out"], new.double(), 2 * U * new.double().abs() + 1e-42, "momentum")
        agree(m["update"], *update(u, tall), ("update", tuple(u.shape)))
        w, x, rate = m["master"].double(), m["update"].double(), 0.02 * m["scale"]
        want = (1 - 0.02 * 0.1) * w - rate * x
        agree(m["master_out"], want, U * (2 * w.abs() + rate * x.abs() + want.abs()) * 1.01 + 1e-42, "weights")        # the decay and its product rounded, the rate, the sum
