"""Registers and scratch memory of the paged kernels whose launches count on them.  Needs no GPU."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401  (the fixture)


# (name, instantiations, most registers, most scratch): 256 registers leave two waves a SIMD, 128 four
@pytest.mark.parametrize("pattern,count,regs,spill", [
    (r"dk::paged_chunk_kernel<", 16, 256, 16),
    (r"dk::paged_chunk_weights_kernel<", 4, 256, 0),
    (r"dk::paged_attn_kernel<bf16_t, \d+, 1", 8, 256, 0),
    (r"dk::paged_evict_(select|phase)_kernel<", 4, 128, 0),
    (r"dk::paged_commit_kernel<4>", 1, 64, 0),
    (r"dk::paged_append_kernel<", 4, 72, 0)])
def test_registers_and_scratch(kernels, pattern, count, regs, spill):  # noqa: F811
    found = {n: v for n, v in kernels.items() if re.match(pattern, n)}
    assert len(found) == count, sorted(kernels)
    for name, (vgprs, scratch) in found.items():
        assert vgprs <= regs and scratch <= spill, (name, vgprs, scratch)
