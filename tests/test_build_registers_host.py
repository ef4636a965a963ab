"""The build looks at the registers that kernels are launched with whose warps give registers to one another."""
import os
import re

from paper_2502_08141_b200 import build

REPORT = """ptxas info    : Compiling entry function '_ZN5lowra12_GLOBAL__N__114product_kernelILi{kind}EEEvNS0_8CeParamsE' for 'sm_100a'
ptxas info    : Function properties for _ZN5lowra12_GLOBAL__N__114product_kernelILi{kind}EEEvNS0_8CeParamsE
    0 bytes stack frame, 0 bytes spill stores, 0 bytes spill loads
ptxas info    : Used {used} registers, used 1 barriers
"""


def test_reports():
    assert build.wrong_registers("") == []
    assert build.wrong_registers(REPORT.format(kind=1, used=168) + REPORT.format(kind=2, used=168)) == []
    wrong = build.wrong_registers(REPORT.format(kind=1, used=168) + REPORT.format(kind=2, used=160) + REPORT.format(kind=3, used=168))
    assert len(wrong) == 1 and wrong[0][1] == 160 and "ILi2E" in wrong[0][0]
    other = REPORT.format(kind=1, used=72).replace("14product_kernel", "19other_product_kernel")
    assert build.wrong_registers(other.replace("19other_product_kernel", "11loss_kernel")) == []


def test_every_kernel_that_shares_out_registers_is_listed():
    found = set()
    for path in build.sources():
        text = open(path).read()
        if "setmaxnreg" not in text:
            continue
        # the kernel that a line stands in: the last one that began before it
        starts = [(m.start(), m.group(1)) for m in re.finditer(r"__global__[^;{]*?\b(\w+_kernel)\(", text)]
        found |= {max(s for s in starts if s[0] < m.start())[1] for m in re.finditer(r"setmaxnreg", text) if any(s[0] < m.start() for s in starts)}
    assert found == set(build.LAUNCH_REGISTERS), (found, os.path.basename(build.CSRC))
