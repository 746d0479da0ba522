"""Pins of the row operators' oracle: closed forms, torch in float64, differences."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro


def test_top_order_with_ties_nan_and_zeros():
    row = np.array([[0.0, 3.0, np.nan, -0.0, 3.0, -np.inf, 1.0]])
    got = ro.top_logits(row, 7)
    assert got["ids"].tolist() == [[1, 4, 6, 0, 3, 2, 5]]
    assert got["rest"][0] == -np.inf
    assert ro.top_logits(row, 2, 2.0)["rest"][0] == pytest.approx(np.log(np.exp(0.5) + 2))
    assert ro.top_logits(np.full((1, 5), -np.inf), 2)["ids"].tolist() == [[0, 1]]


def _entries(rng, V, k, rest):
    t = rng.normal(size=V) * 2
    ids = np.argsort(-t)[:k]
    return t, ids.astype(np.int32), t[ids], (np.log(np.exp(np.delete(t, ids)).sum()) if rest else -np.inf)


def test_distill_is_the_divergence_of_whole_rows_when_every_id_is_an_entry():
    rng = np.random.default_rng(1)
    V, T = 12, 1.7
    t, s = rng.normal(size=V), rng.normal(size=V)
    ids = rng.permutation(V).astype(np.int32)
    got = ro.distill_loss(s[None], ids[None], t[ids][None], temperature=T)
    p, q = torch.softmax(torch.tensor(t) / T, 0), torch.log_softmax(torch.tensor(s) / T, 0)
    want = T * T * torch.nn.functional.kl_div(q, p, reduction="sum")
    assert got["loss"] == pytest.approx(float(want), rel=1e-12)
    np.testing.assert_allclose(got["grad"][0], T * (torch.exp(q) - p).numpy(), atol=1e-14)


def test_distill_of_the_teacher_itself_is_nothing():
    rng = np.random.default_rng(2)
    t, ids, vals, rest = _entries(rng, 50, 6, True)
    got = ro.distill_loss(t[None], ids[None], vals[None], np.array([rest]))
    assert abs(got["loss"]) < 1e-14 and np.abs(got["grad"]).max() < 1e-15


@pytest.mark.parametrize("rest", [False, True])
def test_distill_gradient_against_differences(rest):
    """Central differences of the loss: error h^2 of the third derivative plus rounding 1e-16 / h."""
    rng = np.random.default_rng(3)
    n, V, k, T, h = 3, 40, 5, 1.3, 1e-5
    e = [_entries(rng, V, k, rest) for _ in range(n)]
    ids, vals, r = (np.array([x[j] for x in e]) for j in (1, 2, 3))
    ids[1, 2] = -1                                  # an unused place
    w = np.array([0.5, 2.0, 0.0])
    x = rng.normal(size=(n, V))

    def loss(y):
        return ro.distill_loss(y, ids, vals, r, T, w)["loss"]

    got = ro.distill_loss(x, ids, vals, r, T, w, grad_scale=3.0)
    for i in range(n):
        for v in rng.choice(V, 12, replace=False).tolist() + ids[i][ids[i] >= 0].tolist():
            d = np.zeros_like(x)
            d[i, v] = h
            assert got["grad"][i, v] == pytest.approx(3.0 * (loss(x + d) - loss(x - d)) / (2 * h), abs=1e-9)
    assert np.all(got["grad"][2] == 0)


def test_distill_edges():
    x = np.zeros((1, 4))
    assert ro.distill_loss(x, [[-1, -1]], [[1.0, 2.0]])["loss"] == 0            # the teacher says nothing
    assert np.isnan(ro.distill_loss(x, [[1, 1]], [[1.0, 2.0]])["loss"])         # the same id twice
    low = np.array([[-np.inf, 0.0, 0.0, 0.0]])
    assert ro.distill_loss(low, [[0]], [[1.0]])["loss"] == np.inf               # p > 0 = q
    assert ro.distill_loss(low, [[1]], [[1.0]])["loss"] == pytest.approx(np.log(3))
    assert np.all(np.isfinite(ro.distill_loss(np.full((1, 4), -np.inf), [[0]], [[1.0]])["grad"]))


def test_sample_draws_the_filtered_distribution():
    """Over a fine grid of uniforms each token comes up by its filtered probability."""
    rng = np.random.default_rng(5)
    row = rng.normal(size=9)
    n = 20000
    us = (np.arange(n) + 0.5) / n
    for kw in (dict(), dict(top_k=4), dict(top_p=0.7), dict(min_p=0.3), dict(top_k=6, top_p=0.8, min_p=0.1, T=1.6)):
        T = kw.get("T", 1.0)
        p = np.exp(row / T) / np.exp(row / T).sum()
        by = np.argsort(-p)
        keep = by[:kw.get("top_k", 9)]
        q = p[keep] / p[keep].sum()
        keep = keep[: int(np.sum(np.cumsum(q) - q < kw.get("top_p", 1.0)))]
        keep = keep[p[keep] >= kw.get("min_p", 0.0) * p.max()]
        want = np.zeros(9)
        want[keep] = p[keep] / p[keep].sum()
        got = np.zeros(9)
        for u in us:
            token, lp, kept, _ = ro.sample_row(row, u=u, **kw)
            assert kept == len(keep) and lp == pytest.approx(np.log(want[token]), abs=1e-12)
            got[token] += 1 / n
        assert np.abs(got - want).max() <= 1.5 / n


def test_sample_edges():
    assert ro.sample_row(np.array([1.0, 5.0, 5.0]), T=0, u=0.99)[0] == 1
    assert ro.sample_row(np.array([1.0, 5.0, 5.0]), top_p=0.0, u=0.99)[0] == 1
    assert ro.sample_row(np.full(4, -np.inf))[0] == -1
    assert ro.sample_row(np.array([0.0, np.inf, 1.0, np.inf]), u=0.75)[:2] == (3, -np.log(2))
    assert [ro.sample_row(np.zeros(4), top_p=0.5, u=u)[0] for u in (0.0, 0.49, 0.5, 0.99)] == [0, 0, 1, 1]


def test_distill_of_infinities():
    """+inf in the student's row, the teacher's entries or its rest: NaN, unless the teacher says nothing."""
    x, inf = np.array([[0.0, 1.0, -1.0, 0.5]]), np.inf
    for y, vals, rest in ((np.array([[0.0, inf, -1.0, 0.5]]), [[1.0, 0.0]], None),
                          (np.array([[0.0, -inf, -inf, inf]]), [[1.0, 0.0]], None),
                          (x, [[1.0, inf]], None), (x, [[1.0, 0.0]], [inf])):
        got = ro.distill_loss(y, [[0, 3]], vals, rest)
        assert np.isnan(got["loss"]) and np.isnan(got["grad"]).all()
        got = ro.distill_loss(y, [[0, 3]], vals, rest, weights=[0.0])
        assert got["loss"] == 0 and not got["grad"].any()
    got = ro.distill_loss(np.array([[0.0, inf]]), [[-1]], [[1.0]])
    assert got["loss"] == 0 and not got["grad"].any()
