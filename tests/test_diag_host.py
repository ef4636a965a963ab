"""The diagnostic that withholds the cross entropy's tiles: what it refuses, on the host."""
import pytest

import paper_2502_08141_b200 as lw


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2502_08141_b200 import build
    build.build()


def test_drop_tiles_arguments():
    for calls, products in ((-1, 1), (1001, 1), (1, 0), (1, 4), (0, -1)):
        with pytest.raises(lw.LowraError) as e:
            lw.lowra_diag_drop_tiles(calls, products)
        assert e.value.code == lw.LOWRA_ERR_SHAPE
    lw.lowra_diag_drop_tiles(3, 2)
    lw.lowra_diag_drop_tiles(0)
