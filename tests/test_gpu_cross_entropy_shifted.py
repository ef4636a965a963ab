"""Cross entropy of logits far from zero, all alike: the loss does not depend on what is added to every logit of a token, so a sure token's small loss keeps its digits there too, with a gradient and
without one.  Elementwise against fp64 within the bounds of the other tests."""
import pytest
import torch

from test_gpu_cross_entropy import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [40, 300])
@pytest.mark.parametrize("known", [0.0, 14.0, 26.0])
@pytest.mark.parametrize("shift", [-200.0, -35.0, -20.0, -10.0, 20.0, 35.0, 200.0])
def test_logits_about_another_level(M, known, shift):
    X, W, labels, weights = make(M, 2000, 512, known=known)
    X[:, 0], W[:, 0] = 8.0, shift / 8
    _, _, want = check(X, W, labels, weights)
    small = (want[0] > 0) & (want[0] < 1e-5)
    assert known < 26 or small.sum() > M / 2


def test_two_words_of_negative_logits():
    """The label at -30, the other word at -30 - d: log(1 + exp(-d)), to the digits of an fp32 number."""
    K = 64
    d = torch.tensor([0.0, 0.125, 0.5, 1.0, 4.0, 9.5, 14.5, 20.0, 25.0, -0.125, -1.0, -14.0, -25.0], dtype=torch.float64, device="cuda")
    for level in (-30.0, -5.0, 0.0, 30.0):
        X = torch.zeros((d.numel(), K), device="cuda").bfloat16()
        W = torch.zeros((2, K), device="cuda").bfloat16()
        X[:, 0], X[:, 1], W[:, 0], W[0, 1] = 1.0, d.bfloat16(), level, -1.0       # l = (level - d, level)
        labels = torch.ones(d.numel(), dtype=torch.int64, device="cuda")
        loss, _, want = check(X, W, labels)
        exact = torch.log1p(torch.exp(-d))
        # the exponentials of a logit 55 from zero: 2^-18 of an octave at most for its rounding, 2^-22 for the function; a handful of roundings of the loss itself
        assert ((loss.double() - exact).abs() <= (2.0 ** -18 * 0.7 + 2.0 ** -20) * (1 - torch.exp(-exact)) + 2.0 ** -21 * exact).all()
