"""Distillation over the whole range of temperatures that it takes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import rows_oracle as ro  # noqa: E402
from test_gpu_rows import _check_distill, _distill, _make, _put, _teacher, _values  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1e-30, 2e-30, 1e-25, 1e-18, 1e-16, 3e-14, 1e-12, 1e-8, 1e-4, 1e2, 1e4])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_at_temperatures(T, dtype, rest):
    """Entries t / T apart by up to 1e31 while they are 1e31 themselves: their differences count.  A rest that weighs
    as much as the first entry, where its single precision says so (from 1e-4 up), else far below."""
    rows, V, k, T = 5, 3001, 12, float(np.float32(T))
    ids, vals, tx = _teacher("normal", rows, V, k, seed=12)
    vals[1, 3] = vals[1, 0]         # equal entries
    vals[2] = vals[2, ::-1]         # the largest one last
    vals[3] += 0.1 * np.random.default_rng(0).normal(size=k).astype(np.float32)  # not bf16 values
    ids[4, 5:] = -1
    r = None
    if rest:
        top = vals.max(1).astype(np.float64) / T
        r = (top - (1.0 if T >= 1e-4 else 0.5 / T)).astype(np.float32)
    x = _values(dtype, tx + 0.1 * np.random.default_rng(1).normal(size=tx.shape))
    got = _distill(_put(x, dtype), ids, vals, r, T)
    _check_distill(got, x, ids, vals, r, T, None, 1.0, dtype)
