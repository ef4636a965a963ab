"""Arrays of the epilogue's gradient that get in each other's way are refused before any GPU is asked for."""
import pytest

import paper_2502_08141_b200 as lw

M, N = 4, 64
ROWS = 2 * M * N                 # bytes of an array of rows
AT = 1 << 20                     # addresses that are never used: every call here ends at a check
PLACES = {name: AT * (i + 1) for i, name in enumerate(("dY", "pre", "multiply", "dZ", "dmultiply", "dbias"))}


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2502_08141_b200 import build
    build.build()


def call(**change):
    a = {**PLACES, **change}
    return lw.lib().lowra_epilogue_backward(a["dY"], a["pre"], a["multiply"], M, N, 1, a["dZ"], a["dmultiply"], a["dbias"], 32 * AT, 1 << 20, None)


@pytest.mark.parametrize("written", ["dZ", "dmultiply", "dbias"])
def test_in_each_others_way(written):
    size = lambda name: 4 * N if name == "dbias" else ROWS
    for other in PLACES:
        if other != written:
            for apart in (16, size(other) - 16, 16 - size(written)):
                assert call(**{written: PLACES[other] + apart}) == lw.LOWRA_ERR_SHAPE, (other, apart)
            if other in ("dZ", "dmultiply", "dbias") or written == "dbias":
                assert call(**{written: PLACES[other]}) == lw.LOWRA_ERR_SHAPE, other
