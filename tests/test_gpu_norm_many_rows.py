"""The norm over many rows: the forward kernel that asks for its rows ahead, in every form and on either side of the number of rows from which it is taken, and the backward kernel with parameters in bf16
and 16 or 32 channels to a thread.  Against fp64 within the bounds of the other tests."""
import pytest
import torch

import paper_2502_08141_b200 as lw
from test_gpu_norm import EPS, check_backward, check_forward, make, statistics32

pytestmark = pytest.mark.gpu

# Rows from which the kernel is taken: two to a group of threads, on 148 SMs: 9472 up to 512 channels (groups of a warp), 4440 at 1024, 1184 at 4096, 296 above 8192.  Either side of it, and
# numbers that leave the last round of rows odd, or to some groups only.
SHAPES = [(9471, 256), (9472, 256), (9473, 256), (14300, 8), (9600, 264), (9473, 512), (4439, 1024), (4440, 1024), (5003, 1024), (1183, 4096), (1184, 4096), (1777, 4096), (592, 8192), (295, 8200),
          (296, 8200), (449, 8200), (301, 16384)]


@pytest.mark.parametrize("M, N", SHAPES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("params", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_forward(M, N, kind, params, residual):
    c = make(M, N, kind, params, residual, seed=21)
    Y, rstd, mean, h = lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS, kind=kind, residual=c["residual"])
    check_forward(c, kind, Y, rstd, mean, h)
    again = lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS, kind=kind, residual=c["residual"])
    assert all(a is b or torch.equal(a, b) for a, b in zip((Y, rstd, mean, h), again))


@pytest.mark.parametrize("M, N", [(9473, 256), (9601, 504), (4441, 1024), (1185, 4096), (301, 16384)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_forward_in_place_far_from_zero_and_bad_rows(M, N, kind):
    """sum and Y in the places of the inputs, either way round; a mean a thousand times the spread; a NaN, an infinity and a row of zeros stay in their rows."""
    c = make(M, N, kind, torch.float32, True, seed=22, shift=1000.0)
    want = lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS, kind=kind, residual=c["residual"])
    check_forward(c, kind, *want)
    for swap in (False, True):
        X, residual = c["X"].clone(), c["residual"].clone()
        a, b = (X, residual) if swap else (residual, X)
        got = lw.lowra_norm_forward(X, c["weight"], c["bias"], eps=EPS, kind=kind, residual=residual, sum=a, Y=b)
        assert got[3] is a and got[0] is b and all(x is y or torch.equal(x, y) for x, y in zip(got, want))
    c = make(M, N, kind, torch.bfloat16, False, seed=23)
    good = lw.lowra_norm_forward(c["X"], c["weight"], c["bias"], eps=EPS, kind=kind)
    X = c["X"].clone()
    assert torch.equal(lw.lowra_norm_forward(X, c["weight"], c["bias"], eps=EPS, kind=kind, Y=X)[0], good[0])
    hit = torch.zeros(M, dtype=torch.bool, device="cuda")
    hit[[7, M // 2, M - 1]] = True
    bad = c["X"].clone()
    bad[7, N - 1], bad[M // 2, 3], bad[M - 1] = float("nan"), float("inf"), 0
    Y, rstd, mean, _ = lw.lowra_norm_forward(bad, c["weight"], c["bias"], eps=EPS, kind=kind)
    assert torch.equal(Y[~hit], good[0][~hit]) and torch.equal(rstd[~hit], good[1][~hit])
    assert Y[7].isnan().all() and Y[M // 2].isnan().any() and torch.equal(Y[M - 1], c["bias"] if kind == "layer" else torch.zeros_like(Y[0]))


@pytest.mark.parametrize("M, N", [(1300, 256), (2049, 1288), (2100, 4096), (2049, 8192), (1537, 8200), (1600, 16384)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("residual", [False, True])
def test_backward_with_parameters_in_bf16(M, N, kind, residual):
    c = make(M, N, kind, torch.bfloat16, residual, seed=24)
    mean, rstd = statistics32(c["X"], kind == "layer")
    for sums in (True, False):
        dX, dw, db = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, dsum=c["dsum"], want_params=sums)
        check_backward(c, kind, mean, rstd, dX, dw, db)
    again = lw.lowra_norm_backward(c["dY"], c["X"], c["weight"], rstd, mean=mean, dsum=c["dsum"], dX=c["dY"].clone(), want_params=True)
    check_backward(c, kind, mean, rstd, *again)
