"""Arrays of the factors' update that get in each other's way are refused before any GPU is asked for: every pair of them, within a member and between members."""
import ctypes
import itertools

import pytest

import paper_2502_08141_b200 as lw

AT, ROWS, R = 1 << 20, 64, 16          # addresses that are never used: every call here ends at a check
NAMES = ("grad", "momentum", "momentum_out", "master", "master_out", "weight", "update")
WRITTEN = ("momentum_out", "master_out", "weight", "update")
IN_PLACE = (("momentum_out", "momentum"), ("master_out", "master"))
SIZE = {name: ROWS * R * (2 if name in ("grad", "weight") else 4) for name in NAMES}


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2502_08141_b200 import build
    build.build()


def places(number=0, **change):
    return {**{name: AT * (2 + 8 * number + i) for i, name in enumerate(NAMES)}, **change}


def call(members, workspace_bytes):
    arr = (lw._CFactor * len(members))()
    for c, m in zip(arr, members):
        c.rows, c.cols, c.scale = ROWS, R, 1.0
        for name in NAMES:
            setattr(c, name + "_dev", m[name])
    step = lw._CUpdateStep(0.02, 0.95, 0.0, 1e-7, (ctypes.c_double * 3)(3.4, -4.7, 2.0), 1, 5)
    return lw.lib().lowra_update_factors(arr, len(members), R, ctypes.byref(step), AT, workspace_bytes, None)


def test_within_a_member():
    assert call([places()], 0) == lw.LOWRA_ERR_WORKSPACE
    for written, other in itertools.product(WRITTEN, NAMES):
        if written == other:
            continue
        for apart in (0, 16, SIZE[other] - 16, 16 - SIZE[written]):
            if apart != 0 or (written, other) not in IN_PLACE:
                assert call([places(**{written: places()[other] + apart})], 1 << 20) == lw.LOWRA_ERR_SHAPE, (written, other, apart)


@pytest.mark.parametrize("count", [2, 3, 64])
def test_between_members(count):
    in_order = lw.LOWRA_ERR_WORKSPACE              # (with a workspace of no bytes)
    usual = [places(i, momentum=places(i)["momentum_out"], master=places(i)["master_out"]) for i in range(count)]
    assert call(usual, 0) == in_order and call([places(i) for i in range(count)], 0) == in_order
    assert call([{**m, "grad": usual[0]["grad"]} for m in usual], 0) == in_order                  # one gradient for all: it is only read
    for i, j in ((0, count - 1), (count - 1, 0)):
        for written, other in itertools.product(WRITTEN, NAMES):
            for apart in (0, 16, SIZE[other] - 16, 16 - SIZE[written]):
                members = [dict(m) for m in usual]
                members[i][written] = usual[j][other] + apart
                if written == "momentum_out":
                    members[i]["momentum"] = members[i][written]
                if written == "master_out":
                    members[i]["master"] = members[i][written]
                assert call(members, 0) == lw.LOWRA_ERR_SHAPE, (i, j, written, other, apart)
            for apart in (SIZE[other], -SIZE[written]):
                members = [dict(m) for m in usual]
                members[i][written] = usual[j][other] + apart
                assert call(members, 0) == in_order
