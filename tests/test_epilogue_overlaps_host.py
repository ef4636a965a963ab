"""Arrays of products with an epilogue that get in each other's way are refused before any GPU is asked for: within a member, and between members that run side by side."""
import ctypes
import itertools

import pytest

import paper_2502_08141_b200 as lw
import synth_inputs as si

M, N, K, R = 4, 64, 128, 16
ROWS = 2 * M * N                 # bytes of an output
AT = 1 << 20                     # addresses that are never used: every call here ends at a check


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2502_08141_b200 import build
    build.build()


@pytest.fixture(scope="module")
def layout():
    layout = lw.Layout(si.precisions(N, {1: 0.5, 2: 0.5}), K, device="cpu")
    layout.c.deal_dev = AT
    return layout


class Arrays(dict):
    """Places far from each other, until they are changed."""

    def __init__(self, number=0, **places):
        super().__init__({name: AT * (2 + 8 * number + i) for i, name in enumerate(("X", "Y", "pre", "multiply", "residual"))}, **places)

    def epilogue(self):
        return lw._CEpilogue(None, self["multiply"], self["residual"], self["pre"], 1, 0)


def single(layout, a):
    return lw.lib().lowra_lora_forward_epilogue(layout.ref, AT, AT, AT, a["X"], M, AT, AT, R, 2.0, ctypes.byref(a.epilogue()), a["Y"], AT, 0, None)


def adapters(layout, a):
    start = (ctypes.c_int32 * 3)(0, 1, M)
    return lw.lib().lowra_lora_forward_adapters_epilogue(layout.ref, AT, AT, AT, 2, a["X"], M, start, AT, AT, R, 2.0, ctypes.byref(a.epilogue()), a["Y"], AT, 0, None)


def batch(layout, members):
    arr, behind = (lw._CMember * len(members))(), (lw._CEpilogue * len(members))()
    for i, a in enumerate(members):
        arr[i].layout = ctypes.pointer(layout.c)
        arr[i].packed_dev = arr[i].absmax_dev = arr[i].maps_dev = arr[i].A_dev = arr[i].B_dev = AT
        arr[i].act_dev, arr[i].out_dev = a["X"], a["Y"]
        behind[i] = a.epilogue()
    return lw.lib().lowra_lora_forward_batch_epilogue(arr, behind, len(members), M, R, 2.0, AT, 0, None)


@pytest.mark.parametrize("call", [single, adapters, lambda layout, a: batch(layout, [a])])
def test_within_a_member(layout, call):
    in_order = lw.LOWRA_ERR_WORKSPACE                    # what is left is the workspace, of no bytes
    assert call(layout, Arrays()) == in_order
    for written, other in (("Y", "X"), ("pre", "X"), ("pre", "Y"), ("pre", "multiply"), ("pre", "residual"), ("Y", "multiply"), ("Y", "residual")):
        for apart in (16, ROWS - 16, -16, 16 - ROWS):
            assert call(layout, Arrays(**{written: Arrays()[other] + apart})) == lw.LOWRA_ERR_SHAPE, (written, other, apart)
        for apart in (ROWS if other != "X" else 2 * M * K, -ROWS):
            assert call(layout, Arrays(**{written: Arrays()[other] + apart})) == in_order, (written, other, apart)
        assert call(layout, Arrays(**{written: Arrays()[other]})) == (in_order if (written, other) in (("Y", "multiply"), ("Y", "residual")) else lw.LOWRA_ERR_SHAPE)
    # what is only read may be the same
    assert call(layout, Arrays(residual=Arrays()["X"], multiply=Arrays()["X"])) == in_order


def test_between_members(layout):
    in_order = lw.LOWRA_ERR_WORKSPACE
    assert batch(layout, [Arrays(0), Arrays(1), Arrays(2)]) == in_order
    for i, j in itertools.permutations(range(3), 2):
        for written in ("Y", "pre"):
            for other in ("X", "Y", "pre", "multiply", "residual"):
                for apart in (0, 16, 16 - ROWS):
                    members = [Arrays(0), Arrays(1), Arrays(2)]
                    members[i][written] = members[j][other] + apart
                    assert batch(layout, members) == lw.LOWRA_ERR_SHAPE, (i, j, written, other, apart)
                members[i][written] = members[j][other] - ROWS
                assert batch(layout, members) == in_order
    # one input and one residual for all; each stream added to in place by its own member
    shared = Arrays(0)
    assert batch(layout, [Arrays(i, X=shared["X"], residual=shared["residual"], multiply=shared["multiply"]) for i in range(3)]) == in_order
    assert batch(layout, [Arrays(i, X=shared["X"], residual=Arrays(i)["Y"]) for i in range(3)]) == in_order
    # a gate whose second factor is what the up projection beside it writes; a stream that two members add to
    assert batch(layout, [Arrays(0, multiply=Arrays(1)["Y"]), Arrays(1)]) == lw.LOWRA_ERR_SHAPE
    assert batch(layout, [Arrays(0, residual=Arrays(0)["Y"]), Arrays(1, Y=Arrays(0)["Y"], residual=Arrays(0)["Y"])]) == lw.LOWRA_ERR_SHAPE
