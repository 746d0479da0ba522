"""Temperatures that the distillation refuses and takes; needs no GPU."""
import pytest

import host_stub
from test_rows_refusals import DISTILL, INV, _call
from paper_2605_29707_amd import binding as bd


@pytest.mark.parametrize("T", [1.1e4, 1e5, 1e8, 1e30, float("inf"), float("nan"), 0.9e-30])
def test_temperatures_without_a_loss_are_refused(T):
    assert _call("domino_distill_loss", DISTILL, T=T) == INV and "1e4" in bd.last_error()


def test_the_ends_of_the_range_are_taken(tmp_path):
    host_stub.run('''
import paper_2605_29707_amd.binding as bd
lib, F = bd.load(), h.FAKE
n = lib.domino_distill_workspace_bytes(3, 100, 5)
for T in (1e-30, 1.0, 1e4):
    assert lib.domino_distill_loss(3, 100, 5, F, 1, 100, F, F, None, T, None, 1.0, F, None, None, 0, F, n, None) == 0
''', tmp_path)
