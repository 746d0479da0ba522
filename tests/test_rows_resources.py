"""Registers and scratch memory of the operators on rows of logits, as their comments and the design notes state
them, from the built library's own metadata.  Needs no GPU."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401  (a fixture)


# (name, variants, most registers, most scratch bytes a lane)
@pytest.mark.parametrize("pattern,count,regs,spill", [
    (r"dk::row_groups_kernel<", 2, 64, 0),
    # two workgroups of eight waves a CU; the widest vocabularies one
    (r"dk::(top_select|draw_first)_kernel<\w+, (2|10)>", 8, 128, 0),
    (r"dk::(top_select|draw_first)_kernel<\w+, 20>", 4, 256, 0),
    # sixteen waves of all registers that a workgroup of them can have: one a CU, and it spills
    (r"dk::draw_whole_kernel<", 2, 128, 160),
    (r"dk::distill_(part|grad)_kernel<", 4, 64, 0),
    (r"dk::distill_row_kernel", 1, 128, 0),
])
def test_registers_and_scratch(kernels, pattern, count, regs, spill):  # noqa: F811
    found = {n: v for n, v in kernels.items() if re.match(pattern, n)}
    assert len(found) == count, sorted(kernels)
    for name, (vgprs, scratch) in found.items():
        assert vgprs <= regs and scratch <= spill, (name, vgprs, scratch)
