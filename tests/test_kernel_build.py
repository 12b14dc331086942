"""What the kernels rely on and the compiler decides: read from what it reported when it built them."""
import os
import re

import pytest


@pytest.fixture(scope="module")
def reports():
    """{source: [(kernel, registers)]}"""
    from paper_2606_08804_b200 import build
    build.build()
    out = {}
    for name in sorted(os.listdir(build.CSRC)):
        log = os.path.join(build.OBJ_DIR, name[:-3] + ".log")
        if not name.endswith(".cu") or not os.path.exists(log):
            continue
        text = open(log).read()
        out[name] = [(m.group(1), int(m.group(2))) for m in
                     re.finditer(r"Compiling entry function '(\w+)' for 'sm_100a'(?:(?!Compiling entry).)*?Used (\d+) registers", text, re.S)]
    if not out:
        pytest.skip("the library was not built here")
    return out


def test_registers_handed_from_warps_to_warps(reports):
    """setmaxnreg.inc waits until the CTA's own registers, those of its launch, have room: the two halves of k_scan_bwd that share them out
    need a launch with half of the sum, or the walking warps would wait for good."""
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_08804_b200", "csrc", "scan_bwd.cu")).read()
    walk, prepare = map(int, re.search(r"kWalkRegs = (\d+), kPrepareRegs = (\d+)", src).groups())
    regs = {k: n for k, n in reports["scan_bwd.cu"] if "k_scan_bwd" in k and "ELb0E" in k}          # the end walk, ELb1E, shares nothing out
    assert len(regs) == 6 and src.count("setmaxnreg") == 2
    assert all(2 * n == walk + prepare for n in regs.values()), regs


def test_sizes_of_shared_memory_have_a_place(reports):
    """Each kernel that asks for dynamic shared memory has an entry in its device's table, or every launch would set the size anew."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_08804_b200", "csrc")
    read = lambda n: open(os.path.join(csrc, n)).read()  # noqa: E731
    kernels = {k for n, ks in reports.items() for k, _ in ks if "extern __shared__" in read(n) or "split_common.cuh" in read(n)}
    places = int(re.search(r"kKernels = (\d+)", read("tmap.cu")).group(1))
    assert 100 < len(kernels) <= places, len(kernels)
