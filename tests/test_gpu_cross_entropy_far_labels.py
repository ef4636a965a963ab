"""A label so far above the token's lift that its exponential under it is no fp32 number, with the others far above it too: the gradient is small, not zero.  Elementwise against fp64."""
import pytest
import torch

from test_gpu_cross_entropy import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M, V, K", [(40, 2000, 512), (300, 40000, 128), (2048, 33001, 2560)])
@pytest.mark.parametrize("label, others", [(88.0, 36.0), (89.0, 36.0), (95.0, 36.0), (100.0, 20.0), (80.0, -8.0), (120.0, 40.0)])
def test_label_beyond_the_range_of_an_exponential(M, V, K, label, others):
    X, W, labels, weights = make(M, V, K, ignored=0.1, spread=0.5)
    X[:, 0], W[:, 0], W[V // 3, 0] = 8.0, others / 8, label / 8
    labels[labels >= 0] = V // 3
    _, dX, want = check(X, W, labels, weights, scale=1.0 / 64)
    counts = labels >= 0
    assert (want[0][counts] < 1e-12).all() and want[2][counts].abs().amax(1).gt(1e-38).all() and (dX[counts] != 0).any(1).all()
