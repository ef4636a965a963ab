"""The norm, rotary positions, the cross entropy and the step of adaptive moments take no device memory beside what they are given.  (The first calls make the driver load the kernels' code.)

Collected last on purpose (file name), and written to pass both alone and after the other tests."""
import pytest
import torch

import paper_2502_08141_b200 as lw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [3, 2000])
def test_nothing_is_allocated(M):
    N, V = 512, 1000
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
    scratch = lambda size: new(size, dtype=torch.uint8)  # noqa: E731
    X, Y, h, dX, W = new(M, N) + 1, new(M, N), new(M, N), new(M, N), new(V, N)
    w, b, mean, rstd, dw, db = (new(n, dtype=torch.float32) + 1 for n in (N, N, M, M, N, N))
    ws_norm, ws_loss, ws_only = (scratch(n) for n in (lw.lowra_norm_workspace_bytes(M, N), lw.lowra_cross_entropy_workspace_bytes(M, V, N, True),
                                                      lw.lowra_cross_entropy_workspace_bytes(M, V, N, False)))
    labels, positions, loss = new(M, dtype=torch.int64), new(M, dtype=torch.int32), new(M, dtype=torch.float32)
    turns = torch.from_numpy(lw.lowra_rotary_turns(64)[0].view("int64")).cuda()
    factors = [dict(grad=new(n, 16), master=new(n, 16, dtype=torch.float32), weight=new(n, 16), m=new(n, 16, dtype=torch.float32), v=new(n, 16, dtype=torch.float32)) for n in (100, 3000)]

    def calls():
        lw.lowra_norm_forward(X, w, b, residual=dX, sum=h, Y=Y, mean=mean, rstd=rstd)
        lw.lowra_norm_backward(Y, h, w, rstd, mean=mean, dsum=X, dX=dX, dweight=dw, dbias=db, workspace=ws_norm)
        lw.lowra_rotary(Y.view(M, 8, 64), positions, turns, k=h.view(M, 8, 64), out=Y.view(M, 8, 64), k_out=h.view(M, 8, 64))
        lw.lowra_cross_entropy(X, W, labels, loss=loss, dX=dX, workspace=ws_loss)
        lw.lowra_cross_entropy(X, W, labels, loss=loss, workspace=ws_only)
        lw.lowra_adamw(factors, 1e-3, step=1)

    calls()
    torch.cuda.synchronize()
    free, allocated = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(5):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free and torch.cuda.memory_stats()["allocation.all.allocated"] == allocated
    assert lw.lowra_device_status(ws_loss) == lw.LOWRA_OK and lw.lowra_device_status(ws_only) == lw.LOWRA_OK
