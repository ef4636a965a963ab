"""The cross entropy's waits run out, made so on the host: tiles that are not loaded.  Every kind of product gives up after the limit, says so by the status word, which the launches behind it leave, and the
next call on the same workspace is right.  Nothing traps, faults or waits without a limit."""
import pytest
import torch

import paper_2502_08141_b200 as lw
from test_gpu_cross_entropy import make

pytestmark = pytest.mark.gpu


@pytest.fixture
def short_waits():
    lw.lowra_set_wait_limit(2_000_000)      # 2 ms
    yield
    lw.lowra_diag_drop_tiles(0)
    lw.lowra_set_wait_limit(0)


# few tokens, loss alone; many; the gradient's two products, in parts of the contraction, and as whole tiles over two pieces of the vocabulary
@pytest.mark.parametrize("M, V, K, grad, products", [(40, 5000, 512, False, 1), (64, 40000, 1096, False, 3), (300, 20000, 1096, False, 1), (300, 5000, 512, True, 1), (300, 20000, 512, True, 2),
                                                     (12, 20000, 512, True, 3), (2048, 40001, 2560, True, 2), (4200, 5000, 256, True, 2), (4200, 5000, 256, False, 1)])
def test_timeout_and_the_next_call(short_waits, M, V, K, grad, products):
    X, W, labels, weights = make(M, V, K, known=5.0)
    ws = torch.empty(lw.lowra_cross_entropy_workspace_bytes(M, V, K, grad), dtype=torch.uint8, device="cuda")

    def call():
        loss, dX = lw.lowra_cross_entropy(X, W, labels, weights=weights, want_grad=grad, workspace=ws)
        return lw.lowra_device_status(ws), loss, dX

    status, good, good_dX = call()
    assert status == lw.LOWRA_OK
    lw.lowra_diag_drop_tiles(2, products)
    for _ in range(2):
        assert call()[0] == lw.LOWRA_ERR_TIMEOUT
    for _ in range(2):
        status, loss, dX = call()
        assert status == lw.LOWRA_OK and torch.equal(loss, good) and (not grad or torch.equal(dX, good_dX))


def test_what_is_not_named_runs_on(short_waits):
    """The gradient's products withheld change nothing for a call without a gradient; disarmed, nothing for any."""
    X, W, labels, _ = make(300, 5000, 512)
    good, _ = lw.lowra_cross_entropy(X, W, labels)
    ws = torch.empty(lw.lowra_cross_entropy_workspace_bytes(300, 5000, 512, True), dtype=torch.uint8, device="cuda")
    lw.lowra_diag_drop_tiles(1, 2)
    assert torch.equal(lw.lowra_cross_entropy(X, W, labels, workspace=ws)[0], good) and lw.lowra_device_status(ws) == lw.LOWRA_OK
    lw.lowra_diag_drop_tiles(5, 3)
    lw.lowra_diag_drop_tiles(0)
    lw.lowra_cross_entropy(X, W, labels, want_grad=True, workspace=ws)
    assert lw.lowra_device_status(ws) == lw.LOWRA_OK
