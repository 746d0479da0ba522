"""Tokens whose uniform, or whose top-p, is the single-precision number next to a border of the running sums.

What decides is a comparison of a running sum with u S (or top_p S).  Both sides of the kernel's are sums of weights,
each off by 2^-38.8 of itself (its polynomial) and by 2^-45 (its rounding to a whole number of 2^-44), where 1 is the
weight of the maximum.  A sum of the first j is so off by j 2^-45 + 2^-38.8 of itself, u S by u V 2^-45 + 2^-38.8
of itself, and the products with u and top_p by 2^-52.  The oracle's sums are in 64-bit mantissas: 2^-46 of a
sum of 2^18.  Farther from a border than all of that together the token is the formula's."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from gpu_helpers import log  # noqa: E402
from oracle import rows_oracle as ro  # noqa: E402
from test_gpu_rows import _make, _put, _sample  # noqa: E402

pytestmark = pytest.mark.gpu


def _sums(x, T):
    """Ids in order and running sums of exp((l - max) / T), of every row."""
    ids = np.stack([ro.order(r) for r in x])
    v = np.take_along_axis(x, ids, 1).astype(np.longdouble)
    return ids, np.cumsum(np.exp((v - v[:, :1]) / np.longdouble(T)), axis=1)


def _off(cum, j, u, V):
    """How far apart the two sides of `cum[j] > u S` may be of the formula's, as a sum."""
    target = np.longdouble(u) * cum[-1]
    return (j + 1 + float(u) * V) * 2.0**-45 + 2 * 2.0**-38.8 * float(target) + 2.0**-45 * float(target)


def _next_to(q):
    """The fp32 numbers around q, from below."""
    f = np.float32(q)
    return [np.nextafter(f, np.float32(-1)), f, np.nextafter(f, np.float32(2))]


CASES = [("normal", 151936, "f32", 1.0), ("normal", 50257, "bf16", 1.3), ("normal", 1000, "f32", 2.0),
         ("zipf", 151936, "bf16", 1.2), ("normal", 32000, "f32", 0.5)]


@pytest.mark.parametrize("upto", [60, 1 << 30])
@pytest.mark.parametrize("kind,V,dtype,T", CASES)
def test_draws_next_to_a_border(kind, V, dtype, T, upto):
    """Without filters, u next to the running sums of the first entries, or of any."""
    n = 48
    x = _make(kind, n, V, dtype, seed=21)
    T = float(np.float32(T))
    ids, cum = _sums(x.astype(np.float64), T)
    rng = np.random.default_rng(V)
    js = rng.integers(0, min(V - 1, upto), n)
    clear_rows = 0
    for c in range(3):
        u = np.array([_next_to(cum[r, js[r]] / cum[r, -1])[c] for r in range(n)], np.float32)
        u = np.clip(u, 0, np.float32(1 - 2.0**-24))
        tok, lp = _sample(_put(x, dtype), u, np.full(n, T, np.float32))
        for r in range(n):
            target = np.longdouble(u[r]) * cum[r, -1]
            near = int(np.argmin(np.abs(cum[r] - target)))
            if abs(cum[r, near] - target) <= _off(cum[r], near, u[r], V):
                continue
            clear_rows += 1
            i = int(np.searchsorted(cum[r], target, side="right"))
            assert tok[r] == ids[r, i], (r, c, js[r], float((cum[r, near] - target) / target))
    log(f"{clear_rows} of {3 * n} draws clear of their border")
    # (behind a peaked row's first entries the steps of u, 2^-24, are wider than the entries' weights: any border is near)
    assert clear_rows >= (2 * n if upto == 60 else n)


@pytest.mark.parametrize("upto", [60, 1000])
@pytest.mark.parametrize("kind,V,dtype,T", CASES)
def test_top_p_next_to_a_border(kind, V, dtype, T, upto):
    """u of the last kept entry tells where top-p ends."""
    n = 48
    x = _make(kind, n, V, dtype, seed=22)
    T = float(np.float32(T))
    ids, cum = _sums(x.astype(np.float64), T)
    rng = np.random.default_rng(V + 1)
    js = rng.integers(0, min(V - 1, upto), n)
    u = np.full(n, 1 - 2.0**-24, np.float32)
    clear_rows = 0
    for c in range(3):
        p = np.array([_next_to(cum[r, js[r]] / cum[r, -1])[c] for r in range(n)], np.float32)
        p = np.clip(p, 0, np.float32(1 - 2.0**-24))
        tok, lp = _sample(_put(x, dtype), u, np.full(n, T, np.float32), top_p=p)
        for r in range(n):
            want = np.longdouble(p[r]) * cum[r, -1]
            near = int(np.argmin(np.abs(cum[r] - want)))
            if abs(cum[r, near] - want) <= _off(cum[r], near, p[r], V):
                continue
            clear_rows += 1
            last = int(np.searchsorted(cum[r], want, side="left"))  # the first whose sum is at least top_p S
            i = int(np.searchsorted(cum[r], np.longdouble(u[r]) * cum[r, last], side="right"))
            if i < last:  # (its weight is less than 2^-24 of the kept sum)
                continue
            assert tok[r] == ids[r, last], (r, c, js[r], float((cum[r, near] - want) / want))
            np.testing.assert_allclose(lp[r], float(np.log((cum[r, last] - (cum[r, last - 1] if last else 0)) / cum[r, last])),
                                       rtol=2.0**-23, atol=4e-6)
    log(f"{clear_rows} of {3 * n} borders clear")
    assert clear_rows >= 2 * n
