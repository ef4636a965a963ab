"""The training step's calls by the binding's native way and by the interpreted one: the same results, the same objects back, and the native way leaves to the other what is not ordinary."""
import numpy as np
import pytest
import torch

import paper_2502_08141_b200 as lw

pytestmark = pytest.mark.gpu


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen(seed), device="cuda").to(dtype)


def turns_of(dim):
    return torch.from_numpy(lw.lowra_rotary_turns(dim)[0].view(np.int64)).cuda()


def norm_forward(new):
    x, out = rand(7, 256), {} if new else dict(Y=rand(7, 256), rstd=rand(7, dtype=torch.float32), mean=rand(7, dtype=torch.float32), sum=rand(7, 256))
    got = lw.lowra_norm_forward(x, rand(256, seed=1), rand(256, seed=2), residual=rand(7, 256, seed=3), **out)
    assert new or (got[0] is out["Y"] and got[1] is out["rstd"] and got[2] is out["mean"] and got[3] is out["sum"])
    return [*got, *(t for t in lw.lowra_norm_forward(x, rand(256, dtype=torch.float32), kind="rms") if t is not None)]


def norm_backward(new):
    x, out = rand(7, 256), {} if new else dict(dX=rand(7, 256), dweight=rand(256, dtype=torch.float32), dbias=rand(256, dtype=torch.float32),
                                               workspace=torch.empty(lw.lowra_norm_workspace_bytes(7, 256), dtype=torch.uint8, device="cuda"))
    rstd, mean = rand(7, seed=4, dtype=torch.float32), rand(7, seed=5, dtype=torch.float32)
    got = lw.lowra_norm_backward(rand(7, 256, seed=1), x, rand(256, seed=2), rstd, mean=mean, dsum=rand(7, 256, seed=3), want_params=new, **out)
    assert new or (got[0] is out["dX"] and got[1] is out["dweight"] and got[2] is out["dbias"])
    alone = lw.lowra_norm_backward(rand(7, 256, seed=1), x, rand(256, seed=2), rstd)
    assert alone[1] is None and alone[2] is None
    return [*got, alone[0]]


def rotary(new):
    q, k, at = rand(9, 4, 64), rand(9, 2, 64, seed=1), torch.arange(9, device="cuda", dtype=torch.int32)
    out = {} if new else dict(out=rand(9, 4, 64), k_out=rand(9, 2, 64))
    got = lw.lowra_rotary(q, at, turns_of(32), k=k, interleaved=True, scale=1.5, **out)
    assert type(got) is tuple and (new or (got[0] is out["out"] and got[1] is out["k_out"]))
    one = lw.lowra_rotary(q.transpose(0, 1).contiguous().transpose(0, 1), at, turns_of(64), inverse=True)
    assert one.is_contiguous()
    return [*got, one]


def cross_entropy(new):
    x, w, y = rand(20, 128), rand(300, 128, seed=1), torch.randint(0, 300, (20,), generator=gen(), device="cuda")
    out = {} if new else dict(loss=rand(20, dtype=torch.float32), dX=rand(20, 128), workspace=torch.empty(lw.lowra_cross_entropy_workspace_bytes(20, 300, 128, True), dtype=torch.uint8, device="cuda"))
    got = lw.lowra_cross_entropy(x, w, y, scale=0.5, weights=rand(20, seed=2, dtype=torch.float32), ignore_index=3, want_grad=new, **out)
    assert new or (got[0] is out["loss"] and got[1] is out["dX"])
    only = lw.lowra_cross_entropy(x, w, y)
    assert only[1] is None
    return [*got, only[0]]


def adamw(new):
    members = [dict(grad=rand(300, 3), master=rand(300, 3, dtype=torch.float32), m=torch.zeros(300, 3, device="cuda").to(torch.float8_e4m3fn), v=torch.zeros(300, 3, device="cuda").to(torch.float8_e4m3fn),
                    m_scale=torch.zeros(4, device="cuda"), v_scale=torch.zeros(4, device="cuda"), weight=None if new else rand(300, 3)) for _ in range(3)]
    assert lw.lowra_adamw(members, 1e-3, step=2) is members
    lw.lowra_adamw(members, torch.full((1,), 1e-2, device="cuda"), betas=(0.8, 0.9), step=torch.full((1,), 3, dtype=torch.int32, device="cuda"), grad_scale=torch.full((1,), 0.5, device="cuda"))
    return [t.float() for m in members for t in m.values() if t is not None]


@pytest.mark.parametrize("new", [True, False])
@pytest.mark.parametrize("call", [norm_forward, norm_backward, rotary, cross_entropy, adamw])
def test_both_ways(call, new, monkeypatch):
    lw.lib()
    native = getattr(lw._py_calls, call.__name__)
    answers = []

    class Listening:
        def __getattr__(self, name):
            inner = getattr(real, name)
            if name != call.__name__:
                return inner

            def ask(*args):
                answers.append(inner(*args))
                return answers[-1]
            return ask

    real = lw._py_calls
    monkeypatch.setattr(lw, "_py_calls", Listening())
    a = call(new)
    assert answers and all(x is not None and type(x) is not int for x in answers) and native is not None
    monkeypatch.setattr(lw, "_py_calls", None)
    b = call(new)
    assert len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


def test_statuses_come_through():
    """What the library refuses is an error of its status by either way."""
    x, at = rand(4, 2, 64), torch.arange(4, device="cuda", dtype=torch.int32)
    for call, code in ((lambda: lw.lowra_norm_forward(rand(4, 60), rand(60), rand(60)), lw.LOWRA_ERR_SHAPE), (lambda: lw.lowra_norm_forward(rand(4, 64), rand(64)), lw.LOWRA_ERR_NULL),
                       (lambda: lw.lowra_rotary(x, at, turns_of(8)), lw.LOWRA_ERR_SHAPE), (lambda: lw.lowra_rotary(x, at, turns_of(64), k=x, out=x, k_out=x), lw.LOWRA_ERR_SHAPE),
                       (lambda: lw.lowra_cross_entropy(rand(4, 60), rand(9, 60), torch.zeros(4, dtype=torch.int64, device="cuda")), lw.LOWRA_ERR_SHAPE),
                       (lambda: lw.lowra_adamw([dict(grad=rand(8), master=rand(8, dtype=torch.float32), m=rand(8, dtype=torch.float32), v=rand(8, dtype=torch.float32))], 1e-3, step=0),
                        lw.LOWRA_ERR_SHAPE)):
        for way in (lw._py_calls, None):
            keep, lw._py_calls = lw._py_calls, way
            try:
                with pytest.raises(lw.LowraError) as e:
                    call()
                assert e.value.code == code
            finally:
                lw._py_calls = keep
