"""Infinite logits and teacher's values: which outputs they reach, and which not."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from oracle import rows_oracle as ro  # noqa: E402
from test_gpu_rows import _check_distill, _check_rest, _distill, _make, _put, _teacher, _top  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
def test_distill_of_infinities(dtype, weights):
    """A row with a student's logit, a teacher's value or a rest of +inf has no distribution: its loss and every
    gradient of it are NaN, without an error bit, unless it weighs nothing; other rows are as they were."""
    rows, V, k = 9, 5003, 8
    ids, vals, tx = _teacher("normal", rows, V, k, seed=5)
    r = ro.top_logits(tx, k)["rest"].astype(np.float32)
    x = _make("normal", rows, V, dtype, seed=6)
    others = np.setdiff1d(np.arange(V), ids[2])
    x[0, np.setdiff1d(np.arange(V), ids[0])[100]] = np.inf  # a student's logit of no entry
    x[1, ids[1, 3]] = np.inf                              # ... of an entry
    x[2, others], x[2, ids[2, 0]] = -np.inf, np.inf       # ... and every id that is no entry masked
    x[3, ids[3, 0]], x[3, ids[3, 1]] = -np.inf, np.inf    # ... where the one entry that the teacher has is masked
    vals[3, 1:], r[3] = -np.inf, -np.inf
    vals[4, 2] = np.inf                                   # a teacher's value
    r[5] = np.inf                                         # its rest
    ids[6], r[6] = -1, np.inf                             # ... alone
    vals[7, 2], x[7, np.setdiff1d(np.arange(V), ids[7])] = np.inf, -np.inf
    lost = np.arange(rows) < 8
    w = np.where(lost, 0.0, 1.5).astype(np.float32) if weights else None
    loss, row_loss, grad = got = _distill(_put(x, dtype), ids, vals, r, w=w)
    assert np.isnan(row_loss[lost]).all() and np.isfinite(row_loss[~lost]).all()
    if weights:
        assert np.isfinite(loss) and not grad[lost].any() and np.isfinite(grad).all()
    else:
        assert np.isnan(loss) and np.isnan(grad[lost]).all() and np.isfinite(grad[~lost]).all()
    _check_distill(got, x, ids, vals, r, 1.0, w, 1.0, dtype)


def test_distill_of_a_student_of_infinities_without_a_teacher():
    """A row whose teacher says nothing has loss and gradient 0, whatever the student's."""
    x = _make("normal", 2, 300, "f32")
    x[0, 5] = np.inf
    ids, vals = np.full((2, 3), -1), np.zeros((2, 3), np.float32)
    loss, row_loss, grad = _distill(_put(x, "f32"), ids, vals)
    assert loss == 0 and not row_loss.any() and not grad.any()


@pytest.mark.parametrize("V,k,n_inf,dtype", [(40, 3, 4, "f32"), (4099, 64, 65, "bf16"), (50257, 10, 3000, "f32"),
                                             (151936, 1024, 151936, "bf16"), (5000, 200, 200, "f32")])
def test_top_of_more_infinities_than_entries(V, k, n_inf, dtype):
    """More logits of +inf than entries: the entries are the first ids of them, and the rest is +inf."""
    x = _make("normal", 3, V, dtype, seed=8)
    rng = np.random.default_rng(V)
    for row in x:
        row[rng.permutation(V)[:n_inf]] = np.inf
    ids, vals, rest = _top(_put(x, dtype), k)
    want = ro.top_logits(x, k)
    np.testing.assert_array_equal(ids, want["ids"])
    assert np.isposinf(vals).all() and np.isposinf(rest).all() == (n_inf > k)
    _check_rest(rest, want["rest"])


def test_distill_from_a_teacher_of_infinities():
    """The entries of such a row, as domino_top_logits leaves them, give that row's NaN."""
    x = _make("normal", 2, 3000, "f32", seed=4)
    x[0, 7:40] = np.inf
    ids, vals, rest = _top(_put(x, "f32"), 5)
    assert rest[0] == np.inf and np.isfinite(rest[1])
    s = _make("normal", 2, 3000, "f32", seed=9)
    loss, row_loss, grad = _distill(_put(s, "f32"), ids, vals, rest, error=0)
    assert np.isnan(loss) and np.isnan(row_loss[0]) and np.isfinite(row_loss[1])
    assert np.isnan(grad[0]).all() and np.isfinite(grad[1]).all()
