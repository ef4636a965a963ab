"""Which ways of rounding the step of adaptive moments takes, through the C interface, before any GPU is asked for."""
import ctypes

import pytest

import paper_2502_08141_b200 as lw


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2502_08141_b200 import build
    build.build()


@pytest.mark.parametrize("bits, taken", [(8, True), (8 | 0x100, True), (32, True), (32 | 0x100, False), (0x100, False), (8 | 0x200, False), (16, False), (-8, False)])
def test_bits(bits, taken):
    """What is taken ends at an address that is not aligned, the rest before that."""
    at = 1 << 20
    arr = (lw._CAdamwMember * 1)()
    for i, name in enumerate(("grad_dev", "master_dev", "m_dev", "v_dev", "m_scale_dev", "v_scale_dev")):
        setattr(arr[0], name, (i + 1) * at)
    arr[0].master_out_dev, arr[0].m_out_dev, arr[0].v_out_dev, arr[0].m_scale_out_dev, arr[0].v_scale_out_dev, arr[0].n = 2 * at + 8, 3 * at, 4 * at, 5 * at, 6 * at, 1000
    step = lw._CAdamwStep(1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None, bits, 0)
    assert lw.lib().lowra_adamw(arr, 1, ctypes.byref(step), None) == (lw.LOWRA_ERR_ALIGN if taken else lw.LOWRA_ERR_SHAPE)
