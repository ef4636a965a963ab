"""The gradient's whole tiles over several pieces of the vocabulary: more than 74 tiles of 256 tokens by 256 features, kept in fp32 from piece to piece and finished in the last one, with the lift of some
tokens changing between the pieces.  Elementwise against fp64."""
import pytest
import torch

from test_gpu_cross_entropy import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M, V, K", [(2048, 70001, 2560), (1900, 40001, 2824)])
@pytest.mark.parametrize("far", [False, True])
def test_whole_tiles_over_pieces(M, V, K, far):
    X, W, labels, weights = make(M, V, K, known=8.0, ignored=0.1)
    if far:
        X[:, 0], W[:, 0] = 0, 0
        X[::4, 0], X[1::4, 0], X[2::4, 0] = 16.0, -16.0, 8.0
        # the first kind's largest logits rise from piece to piece (in steps of some 130 and 60, twice that in octaves and less), the second's fall; the third's rise once, by more than its headroom
        W[5, 0], W[V // 2, 0], W[V - 3, 0], W[V // 3, 0] = 4.0, 12.0, 16.0, -10.0
        labels[::16], labels[4::16], labels[8::16] = V - 3, V // 2, 5
    loss, dX, want = check(X, W, labels, weights, scale=1 / M)
    if far:
        assert (want[0] > 100).any() and (want[0] < 1e-20).any()
    ws = torch.full((1,), 0, dtype=torch.uint8, device="cuda")  # (another allocation between the two calls)
    again, dX2, _ = check(X, W, labels, weights, scale=1 / M)
    assert torch.equal(loss, again) and torch.equal(dX, dX2) and ws.numel() == 1
