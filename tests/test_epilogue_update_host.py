"""What the epilogue, its gradient and the update of the factors refuse before any GPU is asked for, through the C interface, and the sizes of their scratch."""
import ctypes

import pytest

import paper_2502_08141_b200 as lw
import synth_inputs as si


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2502_08141_b200 import build
    build.build()


AT = 1 << 20        # addresses that are never used: every call here ends at a check


def epilogue(**fields):
    e = lw._CEpilogue()
    for k, v in fields.items():
        setattr(e, k, v)
    return e


def forward(e, Y=AT, X=2 * AT):
    layout = lw.Layout(si.precisions(64, {1: 0.5, 2: 0.5}), 128, device="cpu")
    return lw.lib().lowra_lora_forward_epilogue(layout.ref, AT, AT, AT, X, 4, AT, AT, 16, 2.0, None if e is None else ctypes.byref(e), Y, AT, 0, None)


def test_forward():
    assert forward(None) == lw.LOWRA_ERR_NULL
    assert forward(epilogue(activation=5)) == lw.LOWRA_ERR_SHAPE and forward(epilogue(activation=-1)) == lw.LOWRA_ERR_SHAPE
    for name in ("bias_dev", "multiply_dev", "residual_dev", "pre_dev"):
        assert forward(epilogue(**{name: AT + 8})) == lw.LOWRA_ERR_ALIGN
    for other in ("multiply_dev", "residual_dev"):
        assert forward(epilogue(**{other: AT + 64, "pre_dev": AT + 64})) == lw.LOWRA_ERR_SHAPE
    assert forward(epilogue(pre_dev=AT)) == lw.LOWRA_ERR_SHAPE
    assert forward(epilogue(residual_dev=AT), X=AT) == lw.LOWRA_ERR_SHAPE and forward(epilogue(pre_dev=2 * AT)) == lw.LOWRA_ERR_SHAPE
    assert forward(epilogue(residual_dev=2 * AT)) == lw.LOWRA_ERR_WORKSPACE and forward(epilogue(residual_dev=AT)) == lw.LOWRA_ERR_WORKSPACE
    assert forward(epilogue()) == lw.LOWRA_ERR_WORKSPACE           # everything else is in order
    assert lw.lib().lowra_lora_forward_batch_epilogue(None, None, 1, 4, 16, 2.0, AT, 0, None) == lw.LOWRA_ERR_NULL


def test_backward():
    call = lambda dY=AT, pre=AT, mul=None, M=4, N=64, act=1, dZ=AT, dm=None, db=None, ws=None, n=0: lw.lib().lowra_epilogue_backward(dY, pre, mul, M, N, act, dZ, dm, db, ws, n, None)
    assert call(dY=None) == lw.LOWRA_ERR_NULL and call(dZ=None) == lw.LOWRA_ERR_NULL and call(pre=None) == lw.LOWRA_ERR_NULL
    assert call(dm=AT + 64) == lw.LOWRA_ERR_NULL and call(pre=None, act=0, mul=AT, dm=AT + 64) == lw.LOWRA_ERR_NULL
    assert call(M=0) == lw.LOWRA_ERR_SHAPE and call(N=4) == lw.LOWRA_ERR_SHAPE and call(N=60) == lw.LOWRA_ERR_SHAPE and call(act=7) == lw.LOWRA_ERR_SHAPE
    assert call(mul=AT, dm=AT) == lw.LOWRA_ERR_SHAPE and call(dZ=AT + 2) == lw.LOWRA_ERR_ALIGN and call(M=4096, db=AT) == lw.LOWRA_ERR_WORKSPACE
    assert call(M=(1 << 30) + 1) == lw.LOWRA_ERR_SHAPE and call(N=(1 << 24) + 8) == lw.LOWRA_ERR_SHAPE
    assert lw.lowra_epilogue_workspace_bytes(0, 64) == 0 and lw.lowra_epilogue_workspace_bytes(4, 60) == 0
    for M, N in ((1, 8), (17, 264), (8192, 512), (100000, 13824)):
        size = lw.lowra_epilogue_workspace_bytes(M, N)
        assert size >= 4 * N and size % 256 == 0 and size <= 148 * 3 * 4 * max(N, 256) + 256


def test_update():
    step = lw._CUpdateStep(0.02, 0.95, 0.0, 1e-7, (ctypes.c_double * 3)(3.4, -4.7, 2.0), 1, 5)

    def call(r=16, count=1, steps=5, with_step=True, workspace=AT, **fields):
        arr = (lw._CFactor * 70)()
        for m in arr:
            for k, v in {**dict(rows=64, cols=16, grad_dev=AT, momentum_dev=AT, momentum_out_dev=AT, master_dev=AT, master_out_dev=AT, weight_dev=None, update_dev=None, scale=1.0), **fields}.items():
                setattr(m, k, v)
        step.steps = steps
        return lw.lib().lowra_update_factors(arr, count, r, ctypes.byref(step) if with_step else None, workspace, 0, None)

    assert lw.lib().lowra_update_factors(None, 1, 16, ctypes.byref(step), AT, 0, None) == lw.LOWRA_ERR_NULL
    for bad in (dict(r=8), dict(r=24), dict(r=144), dict(count=0), dict(count=65), dict(rows=60), dict(rows=0), dict(rows=(1 << 24) + 8), dict(rows=64, cols=24), dict(steps=0), dict(steps=33)):
        assert call(**bad) == lw.LOWRA_ERR_SHAPE, bad
    for bad in (dict(with_step=False), dict(workspace=None), dict(grad_dev=None), dict(momentum_dev=None), dict(momentum_out_dev=None), dict(master_out_dev=None),
                dict(master_dev=None, master_out_dev=None), dict(master_dev=None, master_out_dev=None, update_dev=AT, weight_dev=AT)):
        assert call(**bad) == lw.LOWRA_ERR_NULL, bad
    assert call(count=2) == lw.LOWRA_ERR_SHAPE                     # a factor named twice
    for name in ("grad_dev", "momentum_dev", "momentum_out_dev", "master_dev", "master_out_dev", "weight_dev", "update_dev"):
        assert call(**{name: AT + 8}) == lw.LOWRA_ERR_ALIGN, name
    assert call() == lw.LOWRA_ERR_WORKSPACE
    assert lw.lowra_update_workspace_bytes([(64, 16)], 32) == 0 and lw.lowra_update_workspace_bytes([], 16) == 0
    sizes = [lw.lowra_update_workspace_bytes([(11008, r), (r, 4096)], r) for r in range(16, 129, 16)]
    assert all(s % 256 == 0 and s > 0 for s in sizes) and sizes == sorted(sizes)


def test_activation_names():
    assert lw.ACTIVATIONS == {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
    with pytest.raises(ValueError, match="activation"):
        lw._activation("swish")
