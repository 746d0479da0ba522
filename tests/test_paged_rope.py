"""The two rules of YaRN in domino_rope_frequencies, by numbers that were worked out apart from both.  Needs no GPU."""
import math

import numpy as np
import pytest

from paper_2605_29707_amd import binding as bd


# Borders by hand, c(r) = d ln(ctx / (2 pi r)) / (2 ln theta):
#   d 128, theta 1e6, ctx 32768   c(32) = 128 ln(162.97) / 27.631 = 23.60, c(1) = 128 ln(5215.2) / 27.631 = 39.65
#   d 64, theta 1e4, ctx 4096     c(32) = 64 ln(20.372) / 18.421 = 10.47, c(1) = 64 ln(651.90) / 18.421 = 22.51
#   d 64, theta 1e4, ctx 100      c(32) < 0, c(1) = 64 ln(15.915) / 18.421 = 9.61
#   d 16, theta 10, ctx 10000     c(32) = 16 ln(49.736) / 4.6052 = 13.57, c(1) = 16 ln(1591.5) / 4.6052 = 25.6, above d - 1
@pytest.mark.parametrize("d,theta,ctx,first,last", [(128, 1e6, 32768, 23, 40), (64, 1e4, 4096, 10, 23), (64, 1e4, 100, 0, 10),
                                                     (16, 10.0, 10000, 13, 15)])
@pytest.mark.parametrize("factor", [1.0, 4.0, 40.0])
def test_yarn_by_index(d, theta, ctx, first, last, factor):
    f, scale = bd.domino_rope_frequencies(d, theta, bd.DOMINO_ROPE_YARN_INDEX, factor, ctx, 32.0, 1.0)
    for i in range(d // 2):
        base = theta ** (-2.0 * i / d)
        part = min(max((i - first) / (last - first), 0.0), 1.0)       # of the way to a division by `factor`
        assert abs(f[i] - base * (1 - part + part / factor)) <= 64 * 2.0**-53 * base, i
    assert abs(scale - (1 + math.log(factor) / 10)) <= 2.0**-23 * scale


def test_the_rules_of_yarn_differ():
    """Between the borders alone: of 64 frequencies 16 by more than 1%, the rule by turns up to 42% below the other."""
    args = (128, 1e6), (4.0, 32768, 32.0, 1.0)
    by_turns, by_index = (bd.domino_rope_frequencies(*args[0], k, *args[1])[0] for k in (bd.DOMINO_ROPE_YARN, bd.DOMINO_ROPE_YARN_INDEX))
    far = 1 - by_turns / by_index
    assert (np.abs(far) > 0.01).sum() == 16 and round(far.max(), 2) == 0.42 and (np.abs(far[:24]) < 0.01).all() and (np.abs(far[40:]) < 0.01).all()


@pytest.mark.parametrize("args", [(64, 1e4, 4, 2.0, 0), (64, 1e4, 4, 0.5, 4096), (64, 1e4, 4, 2.0, 4096, 1.0, 1.0), (64, 1e4, 5, 2.0, 4096)])
def test_refusals(args):
    with pytest.raises(bd.DominoError) as e:
        bd.domino_rope_frequencies(*args)
    assert e.value.status == bd.DOMINO_ERR_INVALID_ARG
