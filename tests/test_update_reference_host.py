"""The bound on the update notices what S and the steps are held in: mistakes planted in the oracle are outside of it, and what the kernels compute is inside."""
import pytest
import torch

from update_reference import graded, iterate, momentum_of, update


@pytest.mark.parametrize("r", [16, 48, 64, 128])
@pytest.mark.parametrize("L", [264, 1000, 4104])
def test_the_bound_shows_the_precision(r, L):
    u = graded(L, r, L + r, "cpu")
    x, off = update(u, True)
    excess = lambda got: ((got.double() - x).abs() / off).max().item()
    S = u.double().t() @ u.double()
    assert excess(u @ iterate(S).float()) < 0.5                                       # as the kernels do it
    assert excess(u @ iterate(S.float().double()).float()) > 4                        # S rounded to fp32, the steps in 64 bits
    assert excess(u @ iterate(u.t() @ u).float()) > 20                                # all of it in fp32
    assert excess((u.double() @ iterate(S.float().double()))) > 4                     # (and not by the product)


def test_momentum():
    m, g = torch.tensor([1.0, -3.0, 0.1]), torch.tensor([0.5, 0.25, -0.7]).bfloat16()
    new, u = momentum_of(m, g)
    want = 0.95 * m.double() + g.double()
    assert (new.double() - want).abs().max() < 2.0 ** -22 and (u.double() - (g.double() + 0.95 * want)).abs().max() < 2.0 ** -22
    assert torch.equal(momentum_of(m, g, nesterov=False)[1], new)
