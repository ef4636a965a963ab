"""Products with an epilogue, their gradient and the update of the factors take no device memory beside what they are given: free device memory is the same before and after
a run of calls with outputs and workspaces of the caller's.  (The first calls make the driver load the kernels' code.)

Collected last on purpose (file name), and written to pass both alone and after the other tests."""
import pytest
import torch

from epilogue_reference import Weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [3, 300])
def test_nothing_is_allocated(M):
    import paper_2502_08141_b200 as lw

    N, K, r = 640, 1152, 32
    w = Weight(N, K, {1: 0.5, 2: 0.3, 4: 0.2}, r, n=2)
    X, dY = w.draw(M, K).bfloat16(), w.draw(M, N).bfloat16()
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")
    scratch = lambda size: new(size, dtype=torch.uint8)
    bias, Y, Z, dZ, dmultiply, dbias = w.draw(N), new(M, N), new(M, N), new(M, N), new(M, N), new(N, dtype=torch.float32)
    ws, ws4 = scratch(lw.lowra_workspace_bytes(w.layout, M, r)), scratch(lw.lowra_batch_workspace_bytes(w.layout, 4, M, r))
    ws_back = scratch(lw.lowra_epilogue_workspace_bytes(M, N))
    factors = [dict(grad=new(*s), momentum=new(*s, dtype=torch.float32), master=new(*s, dtype=torch.float32), weight=new(*s)) for s in ((K, r), (r, N))]
    ws_update = scratch(lw.lowra_update_workspace_bytes([(K, r), (r, N)], r))
    rank64 = [dict(grad=new(*s), update=new(*s, dtype=torch.float32)) for s in ((K, 64), (64, N))]
    ws_64 = scratch(lw.lowra_update_workspace_bytes([(K, 64), (64, N)], 64))
    member = dict(layout=w.layout, packed=w.packed, absmax=w.absmax, maps=w.maps[0], act=X, A=w.A[0], B=w.B[0], out=Y, bias=bias, activation="gelu", pre=Z)

    def calls():
        lw.lowra_lora_forward_epilogue(*w.head(), X, w.A[0], w.B[0], 2.0, bias=bias, activation="gelu", pre=Z, Y=Y, workspace=ws)
        lw.lowra_lora_forward_batch_epilogue([member], 2.0, ws4)
        lw.lowra_lora_forward_adapters_epilogue(w.layout, w.packed, w.absmax, w.maps, X, [0, 1, M], w.A, w.B, 2.0, bias=bias, residual=dY, Y=Y, workspace=ws4)
        lw.lowra_epilogue_backward(dY, Z, "gelu", multiply=Y, dZ=dZ, dmultiply=dmultiply, dbias=dbias, workspace=ws_back)
        lw.lowra_update_factors(factors, 0.02, rank=r, workspace=ws_update)
        lw.lowra_update_factors(rank64, 0.02, rank=64, workspace=ws_64)

    calls()
    torch.cuda.synchronize()
    free, allocated = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(5):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free and torch.cuda.memory_stats()["allocation.all.allocated"] == allocated
    assert lw.lowra_device_status(ws) == lw.LOWRA_OK and lw.lowra_device_status(ws4) == lw.LOWRA_OK
